"""Host-side refusals of the calls around the adapted projections (no GPU): the
C entries get fake device addresses, which no accepted call of these tests
reaches, and the binding gets tensors that it must refuse before the library."""
import ctypes

import pytest
import torch

P = lambda a: ctypes.c_void_p(a)  # noqa: E731


@pytest.fixture(scope="module")
def ace():
    from paper_2609_06072_amd import ace as mod
    return mod


@pytest.fixture
def no_device():
    if torch.cuda.is_available():
        pytest.skip("fake device addresses are only passed where no kernel can be launched")


def _rt(ace, T=4, k=2, n_keys=4, mode=2, pair_row=0x5000):
    return ace.AceRouting(0x1000, 0x2000, 0x3000, 0x4000, pair_row, 0x6000, 0x7000, 0x8000, n_keys,
                          mode, T, k)


INV, UNS, WSP = -1, -2, -3


@pytest.mark.parametrize("change,want", [
    (dict(dt=2), INV), (dict(im=2), INV), (dict(im=-1), INV), (dict(T=-1), INV),
    (dict(k=0), UNS), (dict(k=33), UNS), (dict(T=1 << 30, k=4), UNS),
    (dict(d_in=60), UNS), (dict(d_out=36), UNS), (dict(dt=0, d_in=62), UNS),
    (dict(d_in=0), INV), (dict(d_out=-8), INV), (dict(E=0), UNS), (dict(E=257), UNS),
    (dict(d_in=1 << 24), UNS), (dict(d_out=1 << 30, E=1, d_in=8, T=1, k=1, rt=dict(n_keys=1)), UNS), (dict(T=1 << 20, k=2, d_out=4096), UNS),
    (dict(T=1 << 20, k=2, d_in=4096), UNS), (dict(d_in=1 << 20, d_out=1 << 20), UNS),
    (dict(acc=2), INV), (dict(rt=None), INV), (dict(E=3), INV),
    (dict(rt=dict(mode=0)), INV), (dict(rt=dict(T=5)), INV), (dict(rt=dict(pair_row=None)), INV),
    (dict(dy=None), INV), (dict(W=None), INV), (dict(dx=None), INV),
    (dict(dy=P(0x1008)), INV), (dict(W=P(0x1004)), INV), (dict(dx=P(0x1002)), INV),
    (dict(ws=None), WSP), (dict(wsb=255), WSP), (dict(ws=P(0x100010)), WSP),
    (dict(im=1, acc=1, ws=None), WSP), (dict(im=1, wsb=255), WSP), (dict(im=1, ws=P(0x100010)), WSP),
])
def test_moe_dx_refusals(ace, no_device, change, want):
    T, k, E = 4, 2, 4
    a = dict(dt=1, im=0, T=T, k=k, d_in=64, d_out=32, E=E, dy=P(0x1000), W=P(0x2000), rt={}, acc=0,
             dx=P(0x3000), ws=P(0x100000), wsb=ace.ace_workspace_bytes(ace.ACE_OP_MOE_DX, T, k, 64, 32, E, 0))
    a.update(change)
    rt = None if a["rt"] is None else ctypes.byref(_rt(ace, **dict(dict(T=a["T"], k=a["k"]), **a["rt"])))
    st = ace.raw_lib().ace_moe_dx(a["dt"], a["im"], a["T"], a["k"], a["d_in"], a["d_out"], a["E"],
                                  a["dy"], a["W"], rt, a["acc"], a["dx"], a["ws"], a["wsb"], None)
    assert st == want, ace.ace_last_error()
    assert ace.ace_last_error()


def test_empty_calls_do_nothing(ace, no_device):
    lib, c = ace.raw_lib(), ctypes.byref(ace.AcePackedAct(None, None))
    rt = ctypes.byref(_rt(ace, T=0))
    assert lib.ace_moe_dx(1, 0, 0, 2, 64, 32, 4, None, P(0x2000), rt, 0, None, None, 0, None) == 0
    assert lib.ace_moe_combine_fwd(1, 0, 2, 64, None, None, rt, None, None) == 0
    assert lib.ace_moe_combine_bwd(1, 0, 2, 64, None, None, None, rt, None, None, None) == 0
    assert lib.ace_act_pack(1, 0, 64, None, c, None) == 0
    assert lib.ace_act_unpack(1, 0, 64, c, None, None) == 0
    assert lib.ace_swiglu_fwd(1, 0, 64, None, None, None, None, None, None) == 0
    assert lib.ace_swiglu_bwd(1, 0, 64, None, None, None, c, c, None, None, None) == 0


def test_workspace_query(ace):
    n = ace.ace_workspace_bytes(ace.ACE_OP_MOE_DX, 100, 3, 40, 64, 5, 0)
    assert n % 256 == 0 and n >= 8 * 100 * 3 * 40 * 4
    assert ace.ace_workspace_bytes(ace.ACE_OP_MOE_DX, 100000, 3, 40, 64, 5, 0) < 2 * 100000 * 3 * 40 * 4
    assert ace.ace_workspace_bytes(ace.ACE_OP_MOE_DX, 0, 3, 40, 64, 5, 0) == 0
    for bad in (dict(d_in=0), dict(T=1 << 30)):
        a = dict(T=100, k=3, d_in=40)
        a.update(bad)
        with pytest.raises(ace.AceError):
            ace.ace_workspace_bytes(ace.ACE_OP_MOE_DX, a["T"], a["k"], a["d_in"], 64, 5, 0)


@pytest.mark.parametrize("change,want", [
    (dict(dt=3), INV), (dict(T=-1), INV), (dict(k=40), UNS), (dict(d=60), UNS), (dict(d=0), INV),
    (dict(dt=0, d=66), UNS), (dict(T=1 << 30, k=2), UNS), (dict(T=1 << 20, k=4, d=4096), UNS),
    (dict(rt=dict(T=5)), INV), (dict(rt=dict(mode=-1)), INV), (dict(rt=dict(pair_row=None)), INV),
    (dict(y=None), INV), (dict(o=None), INV), (dict(y=P(0x1008)), INV), (dict(o=P(0x1004)), INV),
    (dict(w=P(0x1002)), INV),
])
def test_combine_refusals(ace, no_device, change, want):
    a = dict(dt=1, T=4, k=2, d=64, y=P(0x1000), o=P(0x2000), w=P(0x3000), rt={})
    a.update(change)
    rt = ctypes.byref(_rt(ace, **dict(dict(T=a["T"], k=a["k"]), **a["rt"])))
    lib = ace.raw_lib()
    assert lib.ace_moe_combine_fwd(a["dt"], a["T"], a["k"], a["d"], a["y"], a["w"], rt, a["o"], None) == want
    # the same faults in the backward: o is its dout, y with dw its y
    assert lib.ace_moe_combine_bwd(a["dt"], a["T"], a["k"], a["d"], a["o"], a["y"], a["w"], rt,
                                   P(0x4000), P(0x5000), None) == want
    assert lib.ace_moe_combine_bwd(1, 4, 2, 64, P(0x1000), None, None, ctypes.byref(_rt(ace)), None, None, None) == INV
    assert lib.ace_moe_combine_bwd(1, 4, 2, 64, P(0x1000), P(0x1000), None, ctypes.byref(_rt(ace)),
                                   P(0x2000), P(0x2002), None) == INV
    assert lib.ace_moe_combine_fwd(1, 4, 2, 64, P(0x1000), None, None, P(0x2000), None) == INV


@pytest.mark.parametrize("change,want", [
    (dict(dt=9), INV), (dict(rows=-1), INV), (dict(d=0), INV), (dict(d=36), UNS), (dict(dt=0, d=34), UNS),
    (dict(rows=1 << 33, d=8), UNS), (dict(rows=1 << 28), UNS), (dict(d=(1 << 31) - 8), UNS),
    (dict(x=None), INV), (dict(x=P(0x1008)), INV), (dict(c=None), INV),
    (dict(c=(None, 0x2000)), INV), (dict(c=(0x2000, None)), INV), (dict(c=(0x2008, 0x3000)), INV),
])
def test_act_refusals(ace, no_device, change, want):
    a = dict(dt=1, rows=4, d=64, x=P(0x1000), c=(0x2000, 0x3000))
    a.update(change)
    c = None if a["c"] is None else ctypes.byref(ace.AcePackedAct(*a["c"]))
    lib, ok = ace.raw_lib(), ctypes.byref(ace.AcePackedAct(0x2000, 0x3000))
    assert lib.ace_act_pack(a["dt"], a["rows"], a["d"], a["x"], c, None) == want
    assert lib.ace_act_unpack(a["dt"], a["rows"], a["d"], c, a["x"], None) == want
    if change.get("c", 0) is None:
        # one checkpoint without the other
        assert lib.ace_swiglu_fwd(1, 4, 64, a["x"], a["x"], a["x"], ok, None, None) == INV
        assert lib.ace_swiglu_bwd(1, 4, 64, a["x"], None, None, None, ok, a["x"], a["x"], None) == INV
        return
    for i in range(3):      # g, u, a
        t = [P(0x1000)] * 3
        t[i] = a["x"]
        assert lib.ace_swiglu_fwd(a["dt"], a["rows"], a["d"], *t, c, ok, None) == want
    assert lib.ace_swiglu_bwd(a["dt"], a["rows"], a["d"], P(0x1000), None, None, ok, c, a["x"],
                              P(0x1000), None) == want
    assert lib.ace_swiglu_fwd(a["dt"], a["rows"], a["d"], None, None, a["x"], ok, c, None) == want


def test_swiglu_bwd_refusals(ace, no_device):
    lib, x, ok = ace.raw_lib(), P(0x1000), ctypes.byref(ace.AcePackedAct(0x2000, 0x3000))
    f = lambda da, g, u, g8, u8, dg, du: lib.ace_swiglu_bwd(1, 4, 64, da, g, u, g8, u8, dg, du, None)  # noqa: E731
    assert f(None, x, x, None, None, x, x) == INV
    assert f(x, None, x, None, None, x, x) == INV
    assert f(x, x, None, None, None, x, x) == INV
    assert f(x, x, x, None, None, None, x) == INV
    assert f(x, x, x, None, None, x, None) == INV
    assert f(x, x, x, None, None, x, P(0x1008)) == INV
    assert f(x, x, x, ok, ok, x, x) == INV                   # g, u and their checkpoints
    assert f(x, x, None, ok, ok, x, x) == INV
    assert f(x, None, x, ok, ok, x, x) == INV
    fwd = lambda g, u, a, g8, u8: lib.ace_swiglu_fwd(1, 4, 64, g, u, a, g8, u8, None)  # noqa: E731
    assert fwd(x, None, x, ok, ok) == INV
    assert fwd(None, x, x, ok, ok) == INV
    assert fwd(None, None, x, None, None) == INV


def test_binding_refuses_other_devices(ace):
    """Host tensors never reach the library."""
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    W = torch.zeros(4, 64, 64, dtype=torch.bfloat16)
    rt = ace.Routing(2, 2, 4, device="cpu")
    for call in (lambda: ace.ace_moe_dx(x, W, rt, x[:2]), lambda: ace.ace_moe_combine_fwd(x, rt),
                 lambda: ace.ace_moe_combine_bwd(x[:2], rt), lambda: ace.ace_act_pack(x),
                 lambda: ace.ace_act_unpack(ace.PackedAct(4, 64, "cpu")),
                 lambda: ace.ace_swiglu_fwd(x, x), lambda: ace.ace_swiglu_bwd(x, x, x)):
        with pytest.raises(ValueError, match="current GPU"):
            call()


def test_packed_act_shape(ace):
    c = ace.PackedAct(3, 72, "cpu")
    assert c.codes.shape == (3, 72) and c.exps.shape == (3, 3)
