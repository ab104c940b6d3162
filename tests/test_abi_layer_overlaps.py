"""Two outputs in one buffer are refused on the host (no GPU: the C entries get fake
device addresses, which no accepted call of these tests reaches)."""
import ctypes

import pytest
import torch

P = ctypes.c_void_p


@pytest.fixture(scope="module")
def ace():
    if torch.cuda.is_available():
        pytest.skip("fake device addresses are only passed where no kernel can be launched")
    from paper_2609_06072_amd import ace as mod
    return mod


def test_swiglu_outputs(ace):
    lib, x, y = ace.raw_lib(), P(0x10000), P(0x20000)
    c = lambda codes, exps: ctypes.byref(ace.AcePackedAct(codes, exps))  # noqa: E731
    one, codes, exps, two = c(0x30000, 0x40000), c(0x30000, 0x50000), c(0x60000, 0x40000), c(0x60000, 0x70000)
    # dg and du in one buffer, though each may be an input
    for dg, du in ((y, y), (x, x)):
        assert lib.ace_swiglu_bwd(1, 4, 64, x, x, x, None, None, dg, du, None) == -1
        assert "dg" in ace.ace_last_error()
        assert lib.ace_swiglu_bwd(1, 4, 64, x, None, None, one, two, dg, du, None) == -1
    # checkpoints of g and u in one
    for g8, u8 in ((one, one), (one, codes), (one, exps)):
        assert lib.ace_swiglu_fwd(1, 4, 64, x, x, y, g8, u8, None) == -1
        assert "g_packed" in ace.ace_last_error()


def test_combine_gradient_outputs(ace):
    """dy over dout would change what later slots of the token read."""
    lib, x, y = ace.raw_lib(), P(0x10000), P(0x20000)
    rt = ctypes.byref(ace.AceRouting(*[0x1000 * i for i in range(1, 9)], 4, 2, 4, 2))
    assert lib.ace_moe_combine_bwd(1, 4, 2, 64, x, None, None, rt, x, None, None) == -1
    assert lib.ace_moe_combine_bwd(1, 4, 2, 64, x, y, None, rt, x, P(0x30000), None) == -1
    assert lib.ace_moe_combine_fwd(1, 4, 2, 64, x, None, rt, x, None) == -1


def test_input_gradient_over_its_inputs(ace):
    lib, x, w = ace.raw_lib(), P(0x10000), P(0x20000)
    rt = ctypes.byref(ace.AceRouting(*[0x1000 * i for i in range(1, 9)], 4, 2, 4, 2))
    n = ace.ace_workspace_bytes(ace.ACE_OP_MOE_DX, 4, 2, 64, 64, 4, 0)
    f = lambda dy, W, dx, ws: lib.ace_moe_dx(1, 1, 4, 2, 64, 64, 4, dy, W, rt, 0, dx, ws, n if ws else 0, None)  # noqa: E731
    assert f(x, w, x, None) == -1
    assert f(x, w, w, None) == -1
    assert f(x, w, P(0x100000), P(0x100000)) == -1
    assert f(P(0x100000), w, x, P(0x100000)) == -1
