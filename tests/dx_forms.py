"""Routings of the input gradient's tests."""
import numpy as np


def routing(kind, T, k, E, seed=1):
    """ids [T, k].  even: in turn.  tails: as many experts as possible end in a tile
    with one row.  random: uneven, one pair in twenty dropped."""
    rng = np.random.default_rng(seed)
    if kind == "even":
        return (np.arange(T * k, dtype=np.int32) % E).reshape(T, k)
    if kind == "tails":
        assert k == 1 and T >= E
        more, last = divmod(T - E, 256)
        n = np.full(E, 1 + more // E * 256)
        n[:more % E] += 256
        n[-1] += last
        return rng.permutation(np.repeat(np.arange(E, dtype=np.int32), n)).reshape(T, 1)
    logits = rng.gumbel(size=(T, E)) - 0.5 * np.log(np.arange(1, E + 1))
    ids = np.argsort(-logits, axis=1)[:, :k].astype(np.int32)
    ids[rng.random((T, k)) < 0.05] = -1
    return np.ascontiguousarray(ids)
