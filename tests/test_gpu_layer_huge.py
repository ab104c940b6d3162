"""The operators between the projections on tensors of more than 2^32 elements, up to
their limit of 2^33: rows at the start, around each power of two and at the end.

Row by row the same bits as a call on a few of the rows alone; the input gradient, whose
rows meet in tiles, on whole numbers, whose sums are exact (test_gpu_layer_exact.py)."""
import numpy as np
import pytest
import torch

import dx_forms as D
from oracle import layer_oracle as L

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def ace():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a HIP device")
    from paper_2609_06072_amd import ace as mod
    return mod


@pytest.fixture(autouse=True)
def _free():
    yield
    torch.cuda.empty_cache()


def normal(seed, *shape, dtype):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.empty(*shape, dtype=DT[dtype], device="cuda").normal_(generator=g)


def whole(seed, *shape, dtype):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-4, 5, shape, generator=g, device="cuda", dtype=torch.int8).to(DT[dtype])


def spans(rows, d, width=70):
    """[first, end) of rows that lie at the start, across every power of two from 2^30
    elements (and bytes of either type) on, and at the end."""
    out = [(0, width)]
    for e in range(28, 34):
        r = (1 << e) // d
        if width < r < rows - width:
            out.append((r - width // 2, r + width // 2))
    return out + [(rows - width, rows)]


@pytest.mark.parametrize("dtype,rows,d", [("bf16", 2080000, 4104), ("f32", 1060000, 4100)])
def test_rows(ace, dtype, rows, d):
    assert rows * d > 1 << 32
    g, u = normal(1, rows, d, dtype=dtype), normal(2, rows, d, dtype=dtype)
    g8, u8 = ace.PackedAct(rows, d), ace.PackedAct(rows, d)
    a = ace.ace_swiglu_fwd(g, u, g_packed=g8, u_packed=u8)
    parts = {}
    for s in spans(rows, d):
        i = slice(*s)
        p8, q8 = ace.ace_act_pack(g[i]), ace.ace_act_pack(u[i])
        parts[s] = (p8, q8)
        assert torch.equal(a[i], ace.ace_swiglu_fwd(g[i], u[i])), s
        for whole_, part in ((g8, p8), (u8, q8)):
            assert torch.equal(whole_.codes[i], part.codes) and torch.equal(whole_.exps[i], part.exps), s
    a.zero_()
    ace.ace_swiglu_fwd(g8, u8, a)
    dg, du = ace.ace_swiglu_bwd(a, g, u)
    for s in spans(rows, d):
        i = slice(*s)
        assert torch.equal(a[i], ace.ace_swiglu_fwd(*parts[s], dtype=DT[dtype])), s
        for x, y in zip((dg, du), ace.ace_swiglu_bwd(a[i], g[i], u[i])):
            assert torch.equal(x[i], y), s
    ace.ace_swiglu_bwd(a, g8, u8, dg, du)
    for s in spans(rows, d):
        i = slice(*s)
        for x, y in zip((dg, du), ace.ace_swiglu_bwd(a[i], *parts[s])):
            assert torch.equal(x[i], y), s
    del dg, du
    alone = ace.ace_act_pack(u, u8)
    ace.ace_act_unpack(alone, a)
    for s in spans(rows, d):
        i = slice(*s)
        assert torch.equal(alone.codes[i], parts[s][1].codes) and torch.equal(alone.exps[i], parts[s][1].exps), s
        assert torch.equal(a[i], ace.ace_act_unpack(parts[s][1], dtype=DT[dtype])), s


@pytest.mark.parametrize("dtype,T,k,d", [("bf16", 261000, 8, 4104), ("f32", 262000, 4, 4100)])
def test_combine(ace, dtype, T, k, d):
    assert T * k * d > 1 << 32
    E = 16
    ids = D.routing("random", T, k, E)
    route = lambda i: ace.ace_group_permute(torch.from_numpy(np.ascontiguousarray(i)).cuda(), E, None, E, ace.ACE_ROWS_EXPERT)  # noqa: E731
    rt = route(ids)
    y, dout, w = normal(1, T * k, d, dtype=dtype), normal(2, T, d, dtype=dtype), torch.rand(T, k, device="cuda")
    out = ace.ace_moe_combine_fwd(y, rt, pair_w=w)
    dy = torch.full_like(y, 3.0)
    dw = torch.empty(T, k, device="cuda")
    ace.ace_moe_combine_bwd(dout, rt, dy, pair_w=w, y=y, dw=dw)
    for s, e in spans(T, k * d, 20):
        t, p = slice(s, e), slice(s * k, e * k)
        part = route(ids[t])
        assert torch.equal(out[t], ace.ace_moe_combine_fwd(y[p], part, pair_w=w[t])), s
        dyp, dwp = torch.full_like(y[p], 3.0), torch.empty(e - s, k, device="cuda")
        ace.ace_moe_combine_bwd(dout[t], part, dyp, pair_w=w[t], y=y[p], dw=dwp)
        assert torch.equal(dy[p], dyp) and torch.equal(dw[t], dwp), s


@pytest.mark.parametrize("dtype,T,k,d_in,d_out,shared", [
    ("bf16", 2090000, 1, 4104, 256, False),     # dx near the limit
    ("bf16", 1050000, 1, 264, 4104, False),     # dy beyond 2^32
    ("bf16", 1030000, 2, 4104, 264, True),      # and the rows that are summed
    ("f32", 1050000, 1, 4100, 260, False),
    ("f32", 1050000, 1, 132, 4100, False),
    ("f32", 525000, 2, 4100, 132, True),
    ("bf16", 16400000, 1, 264, 24, False),      # short contractions: the streaming kernel
])
def test_moe_dx(ace, dtype, T, k, d_in, d_out, shared):
    E = 4
    assert max(T * k * d_in, T * k * d_out) > 1 << 32
    ids = D.routing("even", T, k, E)
    rt = ace.ace_group_permute(torch.from_numpy(ids).cuda(), E, None, E, ace.ACE_ROWS_EXPERT)
    dy, W = whole(2, T * k, d_out, dtype=dtype), whole(3, E, d_out, d_in, dtype=dtype)
    torch.cuda.empty_cache()
    dx = torch.full((T if shared else T * k, d_in), 7.0, dtype=DT[dtype], device="cuda")
    mode = ace.ACE_INPUT_SHARED if shared else ace.ACE_INPUT_PER_PAIR
    ace.ace_moe_dx(dy, W, rt, dx, input_mode=mode)

    def want(s, e):
        p = np.arange(s * k, e * k) if shared else np.arange(s, e)
        rows = torch.from_numpy(L.expert_dx(dy[torch.from_numpy(p).cuda()].double().cpu().numpy(), Wn,
                                            ids.reshape(-1)[p].reshape(-1, 1), E)).cuda()
        return rows.view(-1, k, d_in).sum(1) if shared else rows

    Wn = W.double().cpu().numpy()
    places = {s for n in (d_in, d_out) for s in spans(len(dx), n * (k if shared else 1), 24)}
    for s, e in sorted(places):
        assert torch.equal(dx[s:e], want(s, e).to(dx.dtype)), s
    if shared:
        ace.ace_moe_dx(dy, W, rt, dx, input_mode=mode, accumulate=True)
        for s, e in sorted(places):
            w = want(s, e)
            assert torch.equal(dx[s:e], (w.to(dx.dtype).double() + w).to(dx.dtype)), s
