"""SwiGLU where sigma(g) lies below fp32's normal numbers and its product with u or
da does not.

Tolerance, per element (u = 2^-24): e^-|g| within 2 ulp (4 u), its reciprocal's
factor 1, and at most four products more, each u: 8 u of the result (powers of two
scale exactly); dg adds 2 u for 1 + g (1 - sigma), at |g| > 69 no cancellation: 12 u;
one rounding to the type.  Inputs keep every result and da u a normal number."""
import numpy as np
import pytest
import torch

from oracle import layer_oracle as L

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
H = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


@pytest.fixture(scope="module")
def ace():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a HIP device")
    from paper_2609_06072_amd import ace as mod
    return mod


def f64(t):
    return t.detach().to("cpu", torch.float64).numpy()


def close(name, got, ref, dt):
    assert np.abs(ref).min() > 2.0 ** -125 and np.abs(ref).max() < 2.0 ** 126, name
    err = np.abs(f64(got) - ref) / np.abs(ref)
    assert err.max() <= (12 * U + H[dt]) * (1 + 2 ** -7), (name, err.max(), np.unravel_index(err.argmax(), err.shape))


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_small_sigma_with_large_factors(ace, dt):
    n, d = 64, 64
    rng = np.random.default_rng(1)
    g = -rng.uniform(70.0, 170.0, (n, d))
    # u, da near sqrt(e^|g|): sigma u and sigma da are normal, da u is
    x = np.minimum(-g / np.log(2.0) - 60.0, 120.0)     # exponent of u in a, of da in du
    big = np.exp2(x) * rng.uniform(1.0, 2.0, (n, d)) * rng.choice([-1.0, 1.0], (n, d))
    one = rng.uniform(0.5, 2.0, (n, d))
    to = lambda a: torch.from_numpy(a).to(dt).cuda()  # noqa: E731
    g, big, one = to(g), to(big), to(one)
    for da, u in ((one, big), (big, one)):
        rdg, rdu = L.swiglu_grads(f64(da), f64(g), f64(u))
        dg, du = ace.ace_swiglu_bwd(da, g, u)
        close("dg", dg, rdg, dt)
        if u is big:
            close("a", ace.ace_swiglu_fwd(g, u), L.swiglu(f64(g), f64(u)), dt)
        else:
            close("du", du, rdu, dt)


def test_far_sigma_is_zero(ace):
    """Below 2^-252 sigma counts as 0, and nothing turns into NaN."""
    g = torch.tensor([[-176.0, -200.0, -1000.0, -3e38, 176.0, 1000.0, 3e38, 88.0]], device="cuda")
    u = torch.full_like(g, 1e-3)
    a = ace.ace_swiglu_fwd(g, u)
    assert not bool(a[0, :4].any()) and torch.equal(a[0, 4:], (g * u)[0, 4:])
    dg, du = ace.ace_swiglu_bwd(torch.ones_like(g), g, u)
    assert not bool(dg[0, :4].any()) and torch.equal(dg[0, 4:], u[0, 4:])
    assert not bool(du[0, :4].any()) and torch.equal(du[0, 4:], g[0, 4:])


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_small_sigma_from_checkpoints(ace, dt):
    """The same, g and u read from their checkpoints (of like size in a block)."""
    n, d = 64, 96
    rng = np.random.default_rng(2)
    base = rng.uniform(75.0, 165.0, (n, 1))
    g = -(base + rng.uniform(-4.0, 4.0, (n, d)))
    big = np.exp2(np.minimum(base / np.log(2.0) - 60.0, 118.0)) * rng.uniform(1.0, 2.0, (n, d)) * rng.choice([-1.0, 1.0], (n, d))
    to = lambda a: torch.from_numpy(a).to(dt).cuda()  # noqa: E731
    da = to(rng.uniform(0.5, 2.0, (n, d)))
    g8, u8 = ace.ace_act_pack(to(g)), ace.ace_act_pack(to(big))
    g, u = (L.unpack(*L.pack(f64(x))) for x in (to(g), to(big)))
    close("a", ace.ace_swiglu_fwd(g8, u8, dtype=dt), L.swiglu(g, u), dt)
    dg, _ = ace.ace_swiglu_bwd(da, g8, u8)
    close("dg", dg, L.swiglu_grads(f64(da), g, u)[0], dt)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_elements_do_not_see_their_neighbours(ace, dt):
    """An element's results are the same bits beside small sigma and without any."""
    n, d = 100, 264
    gen = torch.Generator(device="cuda").manual_seed(3)
    g, u, da = (torch.randn(n, d, generator=gen, device="cuda").mul_(s).to(dt) for s in (20.0, 1.0, 1.0))
    g = g.clamp(min=-69.0)
    far = torch.rand(n, d, generator=gen, device="cuda") < 0.2
    mixed = torch.where(far, torch.full_like(g, -120.0), g)
    assert torch.equal(ace.ace_swiglu_fwd(mixed, u)[~far], ace.ace_swiglu_fwd(g, u)[~far])
    for a, b in zip(ace.ace_swiglu_bwd(da, mixed, u), ace.ace_swiglu_bwd(da, g, u)):
        assert torch.equal(a[~far], b[~far])
