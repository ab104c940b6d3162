"""The sizes of dx_forms.FORMS reach the launch forms that they are there for (CPU:
the library's own rule, with the 256 CUs that it takes where there is no GPU)."""
import pytest
import torch

import dx_forms as D


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    if torch.cuda.is_available():
        pytest.skip("the forms are named for 256 CUs")
    return D.load_rule(str(tmp_path_factory.mktemp("rule")))


@pytest.mark.parametrize("form", D.FORMS, ids=lambda f: "x".join(map(str, f[:5])))
def test_form(rule, form):
    T, k, E, d_in, d_out, kind, kernel, splits, rounds, parts = form
    for sums in (D.JOINED, D.SUMMED):
        assert D.plan(rule, "bf16", T, k, E, d_in, d_out, sums) == (kernel, splits)
    if kernel == D.LARGE:
        tiles = D.large_tiles(D.expert_rows(D.routing(kind, T, k, E), E), d_in, splits)
        assert (rounds, parts) in tiles, tiles


def test_every_share_of_a_contraction_is_there():
    """Large tiles with 1 to 4 and 6 to 8 splits and tiles of 128 with 3 to 8, some of
    both with whole shares of the contraction and some with ragged ones."""
    seen = {(f[6], f[7], f[4] % (128 * f[7]) == 0) for f in D.FORMS}
    for splits in (1, 2, 3, 4, 8):
        assert {(D.LARGE, splits, True), (D.LARGE, splits, False)} <= seen, splits
    assert {(D.LARGE, s, False) for s in (6, 7)} <= seen
    for splits in range(3, 9):
        assert {(D.TILES, splits, True), (D.TILES, splits, False)} <= seen, splits
    several = {(f[7], f[4] % (128 * f[7]) == 0) for f in D.FORMS if f[6] == D.LARGE and f[8] >= 2}
    assert several >= {(1, True), (1, False), (2, False), (3, True), (3, False), (4, True), (4, False)}
