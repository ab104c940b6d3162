"""The input gradient of the expert projection on whole numbers: with |dy|, |W| <= 4
every product and every sum of them below 2^24 is exact in fp32, in whatever order
they are added.  So a result is the exact sum rounded to its type once, whichever
kernel takes the call and however many blocks share a contraction: bit for bit.
Sums of a token's slots and with what dx holds cancel often, so that a rounding of
the summands shows."""
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


def whole(seed, *shape, dtype, top=4):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-top, top + 1, shape, generator=g, device="cuda", dtype=torch.int8).to(DT[dtype])


def exact_rows(dy, W, ids, E):
    """Per pair W_e^T dy[p] in 64 bits (0 where dropped)."""
    out = torch.zeros(dy.shape[0], W.shape[2], dtype=torch.float64, device="cuda")
    key = np.where(L.routed(ids, E), ids, -1).reshape(-1)
    for e in range(E):
        p = torch.from_numpy(np.nonzero(key == e)[0]).cuda()
        if p.numel():
            out[p] = torch.mm(dy[p].double(), W[e].double())
    assert float(out.abs().max()) < 2 ** 23
    return out


def same(name, got, want):
    want = want.to(got.dtype)
    bad = got != want
    assert not bool(bad.any()), (f"{name}: {int(bad.sum())} of {bad.numel()} off, first at "
                                 f"{bad.nonzero()[0].tolist()}: {float(got[bad][0])} for {float(want[bad][0])}")


def check(ace, T, k, E, d_in, d_out, ids, dtype):
    rt = ace.ace_group_permute(torch.from_numpy(ids).cuda(), E, None, E, ace.ACE_ROWS_EXPERT)
    dy, W = whole(2, T * k, d_out, dtype=dtype), whole(3, E, d_out, d_in, dtype=dtype)
    lost = torch.from_numpy(~L.routed(ids, E).reshape(-1)).cuda()
    rows = exact_rows(dy, W, ids, E)
    sums = rows.view(T, k, d_in).sum(1)
    dx = torch.full((T * k, d_in), 7.0, dtype=DT[dtype], device="cuda")
    ace.ace_moe_dx(dy, W, rt, dx, input_mode=ace.ACE_INPUT_PER_PAIR)
    same("per pair", dx, torch.where(lost[:, None], 7.0, rows))
    same("shared", ace.ace_moe_dx(dy, W, rt), sums)
    base = whole(4, T, d_in, dtype=dtype, top=100)
    acc = base.clone()
    ace.ace_moe_dx(dy, W, rt, acc, accumulate=True)
    same("accumulated", acc, sums + base.double())
    base = whole(5, T * k, d_in, dtype=dtype, top=100)
    acc = base.clone()
    ace.ace_moe_dx(dy, W, rt, acc, input_mode=ace.ACE_INPUT_PER_PAIR, accumulate=True)
    same("accumulated per pair", acc, rows + base.double())


@pytest.mark.parametrize("T,k,E,d_in,d_out", [
    (1, 4, 8, 264, 520), (7, 8, 64, 128, 1032), (300, 2, 3, 520, 328), (200, 8, 16, 1000, 264), (1030, 2, 4, 512, 256),
    (257, 32, 40, 64, 48), (2, 2, 8, 544, 4104), (1000, 2, 64, 328, 136), (750, 3, 32, 328, 136), (3000, 4, 200, 256, 1024),
    (4000, 2, 2, 2056, 640), (1000, 2, 64, 264, 648)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sums_are_rounded_once(ace, T, k, E, d_in, d_out, dtype):
    check(ace, T, k, E, d_in, d_out, D.routing("random", T, k, E), dtype)


@pytest.mark.parametrize("form", D.FORMS, ids=lambda f: "x".join(map(str, f[:5])))
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_forms(ace, form, dtype):
    T, k, E, d_in, d_out, kind = form[:6]
    check(ace, T, k, E, d_in, d_out, D.routing(kind, T, k, E), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_one_workspace_for_smaller_calls(ace, dtype):
    """Sized for the largest batch, used for smaller ones on both sides of the sizes
    from which fewer blocks share a contraction."""
    k, E, d_in, d_out = 1, 4, 2048, 1032
    n = ace.ace_workspace_bytes(ace.ACE_OP_MOE_DX, 2049, k, d_in, d_out, E, 0)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    W = whole(3, E, d_out, d_in, dtype=dtype)
    for T in (2049, 2048, 257, 256, 7, 1):
        ids = D.routing("even", T, k, E)
        rt = ace.ace_group_permute(torch.from_numpy(ids).cuda(), E, None, E, ace.ACE_ROWS_EXPERT)
        dy = whole(2, T, d_out, dtype=dtype)
        rows = exact_rows(dy, W, ids, E)
        same(T, ace.ace_moe_dx(dy, W, rt, ws=ws), rows)
        acc = torch.ones(T, d_in, dtype=DT[dtype], device="cuda")
        ace.ace_moe_dx(dy, W, rt, acc, input_mode=ace.ACE_INPUT_PER_PAIR, accumulate=True, ws=ws)
        same(T, acc, rows + 1)


@pytest.mark.parametrize("form", [f for f in D.FORMS if f[6] == D.LARGE and f[8] >= 2 and f[4] % (128 * f[7])][:6],
                         ids=lambda f: "x".join(map(str, f[:5])))
def test_infinities_between_tiles(ace, form):
    """Blocks of several large tiles with a ragged contraction: infinities and NaN at
    its end reach the pairs that use them, not those of the tiles before and after."""
    T, k, E, d_in, d_out, kind = form[:6]
    ids = D.routing(kind, T, k, E)
    rt = ace.ace_group_permute(torch.from_numpy(ids).cuda(), E, None, E, ace.ACE_ROWS_EXPERT)
    dy, W = whole(2, T * k, d_out, dtype="bf16"), whole(3, E, d_out, d_in, dtype="bf16")
    rows = exact_rows(dy, W, ids, E)
    W[E // 2, d_out - 1, :] = float("nan")
    W[E // 4, 0, :] = float("inf")
    dy[7, d_out - 1] = float("inf")
    dy[T * k // 2, :8] = float("nan")
    dx = torch.zeros(T * k, d_in, dtype=torch.bfloat16, device="cuda")
    n = ace.ace_workspace_bytes(ace.ACE_OP_MOE_DX, T, k, d_in, d_out, E, 0)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    ace.ace_moe_dx(dy, W, rt, dx, input_mode=ace.ACE_INPUT_PER_PAIR, ws=ws)
    ok = L.routed(ids, E).reshape(-1)
    hit = np.isin(ids.reshape(-1), (E // 2, E // 4)) & ok
    hit[[7, T * k // 2]] |= ok[[7, T * k // 2]]
    hit = torch.from_numpy(hit).cuda()
    assert not bool(torch.isfinite(dx[hit]).any())
    same("the other rows", dx[~hit], rows[~hit])


def test_reads_no_more_of_the_routing_than_it_needs(ace):
    """The rows' tokens and slots, which these kernels do not use, may be absent."""
    T, k, E, d_in, d_out = 300, 2, 4, 520, 328
    ids = D.routing("random", T, k, E)
    rt = ace.ace_group_permute(torch.from_numpy(ids).cuda(), E, None, E, ace.ACE_ROWS_EXPERT)
    dy, W = whole(2, T * k, d_out, dtype="bf16"), whole(3, E, d_out, d_in, dtype="bf16")
    want = ace.ace_moe_dx(dy, W, rt)
    rt.c.row_token = rt.c.row_slots = None
    same("without", ace.ace_moe_dx(dy, W, rt), want)
