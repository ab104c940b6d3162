"""Pins of oracle/layer_oracle.py (CPU): hand-worked values, scalar loops and
central differences."""
import numpy as np
import pytest

from oracle import layer_oracle as L


def test_routed_pairs():
    ids = np.array([[0, 3], [2, 2], [-1, 1], [4, 0]])
    assert L.routed(ids, 4).tolist() == [[True, True], [True, False], [False, True], [False, True]]


def test_expert_dx_by_hand():
    W = np.arange(12.0).reshape(2, 3, 2)            # E=2, d_out=3, d_in=2
    dy = np.array([[1.0, 0.0, 2.0], [0.0, -1.0, 1.0]])
    ids = np.array([[1, 0]])
    # pair 0 -> expert 1: 1*(6,7) + 2*(10,11); pair 1 -> expert 0: -(2,3) + (4,5)
    assert L.expert_dx(dy, W, ids, 2).tolist() == [[26.0, 29.0], [2.0, 2.0]]
    assert L.expert_dx(dy, W, np.array([[1, 1]]), 2).tolist() == [[26.0, 29.0], [0.0, 0.0]]
    assert L.slot_sum(L.expert_dx(dy, W, ids, 2), 2).tolist() == [[28.0, 31.0]]


def test_dx_is_the_gradient_of_the_projection():
    rng = np.random.default_rng(0)
    T, k, E, d_in, d_out = 5, 2, 3, 4, 6
    x, W = rng.normal(size=(T, d_in)), rng.normal(size=(E, d_out, d_in))
    dy = rng.normal(size=(T * k, d_out))
    ids = np.array([[0, 1], [2, 0], [1, 5], [2, 2], [0, 2]])
    ok = L.routed(ids, E)

    def loss(x):
        return sum(dy[t * k + j] @ (W[ids[t, j]] @ x[t]) for t in range(T) for j in range(k) if ok[t, j])

    dx = L.slot_sum(L.expert_dx(dy, W, ids, E), k)
    for t in range(T):
        for c in range(d_in):
            h = np.zeros_like(x)
            h[t, c] = 1.0
            assert dx[t, c] == pytest.approx((loss(x + h) - loss(x - h)) / 2, abs=1e-12)


def test_combine_and_its_gradient():
    rng = np.random.default_rng(1)
    T, k, E, d = 4, 3, 5, 7
    ids = np.array([[0, 1, 2], [3, 3, 4], [9, 0, 1], [2, -1, 2]])
    y, w, dout = rng.normal(size=(T * k, d)), rng.random((T, k)), rng.normal(size=(T, d))
    dy, dw = L.combine_grads(dout, y, w, ids, E)
    f = lambda y, w: float((L.combine(y, w, ids, E) * dout).sum())  # noqa: E731
    for p in range(T * k):
        h = np.zeros_like(y)
        h[p, 2] = 1.0
        assert dy[p, 2] == pytest.approx((f(y + h, w) - f(y - h, w)) / 2, abs=1e-12)
        hw = np.zeros(T * k)
        hw[p] = 1.0
        hw = hw.reshape(T, k)
        assert dw.reshape(-1)[p] == pytest.approx((f(y, w + hw) - f(y, w - hw)) / 2, abs=1e-12)


def test_swiglu_gradient_by_differences():
    rng = np.random.default_rng(2)
    g, u, da = (rng.normal(size=200) * 3 for _ in range(3))
    dg, du = L.swiglu_grads(da, g, u)
    h = 1e-6
    # central differences: h^2/6 |f'''| < 1e-11 and rounding 2^-52 |f| / h < 1e-8
    assert np.allclose(dg, da * (L.swiglu(g + h, u) - L.swiglu(g - h, u)) / (2 * h), rtol=0, atol=1e-7)
    assert np.allclose(du, da * (L.swiglu(g, u + h) - L.swiglu(g, u - h)) / (2 * h), rtol=0, atol=1e-7)
    assert L.swiglu(np.array([-1000.0]), np.array([3.0]))[0] == 0.0


def test_checkpoint_by_hand():
    x = np.zeros((1, 40))
    x[0, :4] = [1.0, -0.5, 127 / 64, 1 / 128]      # 127/64: code 127 at step 1/64
    x[0, 32:34] = [255 / 128, 3.0 / 128]           # 127.5 steps of 1/64: the step doubles
    codes, exps = L.pack(x)
    assert exps.tolist() == [[127, 128]]
    assert codes[0, :4].tolist() == [64, -32, 127, 0]     # half a step: to even
    assert codes[0, 32:34].tolist() == [64, 1]            # 63.75 -> 64, 0.75 -> 1
    assert L.unpack(codes, exps)[0, [0, 2, 32, 33]].tolist() == [1.0, 127 / 64, 2.0, 1 / 32]


def test_checkpoint_bounds_and_fixed_points():
    rng = np.random.default_rng(3)
    x = (rng.normal(size=(50, 100)) * 2.0 ** rng.integers(-30, 30, size=(50, 100))).astype(np.float32)
    x = x.astype(np.float64)
    codes, exps = L.pack(x)
    assert np.abs(codes.astype(int)).max() <= 127
    v = L.unpack(codes, exps)
    for b in range(4):
        blk = slice(32 * b, min(100, 32 * b + 32))
        top = np.abs(x[:, blk]).max(1, keepdims=True)
        assert np.all(np.abs(v - x)[:, blk] <= top / 127.5)
    c2, e2 = L.pack(v)              # what a checkpoint holds is held exactly
    assert np.array_equal(L.unpack(c2, e2), v)


def test_checkpoint_extremes():
    big = float(np.finfo(np.float32).max)
    x = np.zeros((6, 32))
    x[0, 3] = np.nan
    x[1, 5] = -np.inf
    x[2, 0] = big                   # s stays 254: code 127, less than a step off
    x[3, 0] = 2.0 ** -149           # below the smallest step: zero
    x[4, 0] = 2.0 ** -133           # the smallest step
    codes, exps = L.pack(x)
    assert exps[:, 0].tolist() == [255, 255, 254, 0, 0, 0]
    v = L.unpack(codes, exps)
    assert np.isnan(v[:2]).all() and not v[3].any() and not v[5].any()
    assert v[2, 0] == 127 * 2.0 ** 121 and v[4, 0] == 2.0 ** -133
