"""Workspace of the input gradient (no GPU): one that was sized for the largest call
serves every smaller one, though those may share contractions among more blocks."""
import pytest


@pytest.fixture(scope="module")
def ace():
    from paper_2609_06072_amd import ace as mod
    return mod


@pytest.mark.parametrize("k,d_in", [(1, 2048), (8, 2048), (2, 4096), (3, 40), (1, 8)])
def test_size_never_falls(ace, k, d_in):
    # around every power of two of T, and so around every step of T * k * d_in
    sizes = sorted({t for i in range(22) for t in ((1 << i) - 1, 1 << i, (1 << i) + 1, (1 << i) * 1024 // (k * 1000) + 1)})
    need = [ace.ace_workspace_bytes(ace.ACE_OP_MOE_DX, t, k, d_in, 64, 8, 0) for t in sizes if t > 0]
    assert need == sorted(need)
    for t in (100, 5000):
        by_k = [ace.ace_workspace_bytes(ace.ACE_OP_MOE_DX, t, j, d_in, 64, 64, 0) for j in range(1, 33)]
        assert by_k == sorted(by_k)
        by_d = [ace.ace_workspace_bytes(ace.ACE_OP_MOE_DX, t, k, 40 * j, 64, 64, 0) for j in range(1, 120)]
        assert by_d == sorted(by_d)


def test_size_holds_every_share(ace):
    """An fp32 row per pair for each of the blocks that may share a contraction."""
    for elems, blocks in ((1 << 19, 8), ((1 << 19) + 8, 4), (1 << 22, 4), ((1 << 22) + 8, 1), (1 << 28, 1)):
        assert ace.ace_workspace_bytes(ace.ACE_OP_MOE_DX, elems // 8, 1, 8, 64, 8, 0) >= 4 * blocks * elems
    assert ace.ace_workspace_bytes(ace.ACE_OP_MOE_DX, 1 << 25, 1, 8, 64, 8, 0) == 4 << 28
