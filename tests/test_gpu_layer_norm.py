"""LayerNorm forward and backward against the formulas in 64 bits, against differences, and over widths, types and strides."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def g():
    import paper_2505_01068_b200 as lib
    lib.load()
    return lib


def _type(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _make(B, seg, d, tx, ty, padded, seed=0):
    torch.manual_seed(seed)
    L = sum(seg)
    valid = torch.stack([torch.randint(0, m + 1, (B,)) for m in seg], dim=1).int().cuda() if padded else None
    real = torch.ones((B, L), dtype=torch.bool, device="cuda")
    if padded:
        n = valid[:, torch.repeat_interleave(torch.arange(3), torch.tensor(seg)).cuda()]
        real = torch.cat([torch.arange(m) for m in seg]).cuda()[None, :] < n
    x = (torch.randn((B, L, d), device="cuda") * 1.5 + 3.0).to(tx)
    dy, res = torch.randn((B, L, d), device="cuda").to(ty), torch.randn((B, L, d), device="cuda").to(tx)
    for t in (x, dy, res):
        t[~real] = float("nan")
    return x, dy, res, 1 + 0.2 * torch.randn(d, device="cuda"), 0.2 * torch.randn(d, device="cuda"), valid, real


def _exact(x, dy, res, gamma, beta, real, eps):
    x, dy = (torch.where(real[:, :, None], t.double(), 0.0) for t in (x, dy))
    mean = x.mean(-1, keepdim=True)
    rstd = ((x - mean).square().mean(-1, keepdim=True) + eps) ** -0.5
    h = (x - mean) * rstd
    ga = torch.ones_like(x[0, 0]) if gamma is None else gamma.double()
    y = h * ga + (0.0 if beta is None else beta.double())
    gr = dy * ga
    dx = rstd * (gr - gr.mean(-1, keepdim=True) - h * (gr * h).mean(-1, keepdim=True))
    if res is not None:
        dx = dx + res.double()
    keep = real[:, :, None]
    zero = torch.zeros((), dtype=torch.float64, device="cuda")
    return (torch.where(keep, y, zero), torch.where(keep, mean, zero)[..., 0], torch.where(keep, rstd, zero)[..., 0], torch.where(keep, dx, zero),
            (dy * h).sum((0, 1)), dy.sum((0, 1)))


def _close(got, want, rel, what):
    err = float((got.double() - want).norm())
    assert err <= rel * float(want.norm()) + 1e-30, f"{what}: {err / max(float(want.norm()), 1e-30):.2e}"


WIDTHS = [1, 2, 3, 7, 8, 16, 31, 32, 36, 60, 64, 65, 96, 128, 130, 200, 256, 300, 511, 512, 516, 768, 1000, 1024, 1027, 1536, 2048, 2052, 4096, 5000, 8191, 8192]


@pytest.mark.parametrize("d", WIDTHS)
@pytest.mark.parametrize("types", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16"), ("bf16", "f32")])
def test_widths_and_types(g, d, types):
    """Rounding: float results within some 2^-24 sqrt(d) steps of 64 bits, relative to their norm (x lies around 3, so a centred value
    loses two bits); bf16 results within 2^-9 of it."""
    tx, ty = map(_type, types)
    seg, B = (3, 10, 6), 3
    x, dy, res, gamma, beta, valid, real = _make(B, seg, d, tx, ty, True)
    y, mean, rstd = g.layer_norm_fwd(x, gamma, beta, seg, valid, out_dtype=ty, want_stats=True)
    dx, dgamma, dbeta = g.layer_norm_bwd(dy, x, mean, rstd, gamma, seg, valid, residual=res)
    ey, em, er, edx, ega, ebe = _exact(x, dy, res, gamma, beta, real, 1e-5)
    tol = lambda t: 4e-3 if t == torch.bfloat16 else 3e-6
    if d > 1:   # at width 1 the centred value is zero exactly
        _close(y, ey, tol(ty), "y")
    _close(mean, em, 1e-6, "mean")
    _close(rstd, er, 1e-5, "rstd")
    _close(dbeta, ebe, 3e-6, "dbeta")
    if d > 2:   # a pair's normalised values are +-1 whatever x is, and the gradient cancels to eps
        _close(dx, edx, tol(tx), "dx")
        _close(dgamma, ega, 5e-6, "dgamma")
    pad = ~real
    for t in (y, dx):
        assert not t[pad].float().any() and not torch.signbit(t[pad]).any()
    again = g.layer_norm_bwd(dy, x, mean, rstd, gamma, seg, valid, residual=res)
    assert all(torch.equal(a, b) for a, b in zip(again, (dx, dgamma, dbeta)))
    assert torch.equal(g.layer_norm_bwd(dy, x, mean, rstd, gamma, seg, valid, residual=res, want_params=False), dx)
    assert g.last_device_status() == (0, 0)


@pytest.mark.parametrize("d", [64, 65, 512, 1024])
def test_without_parameters_padding_segments_or_residual(g, d):
    x, dy, _, _, _, _, real = _make(2, (5, 9, 4), d, torch.float32, torch.float32, False, 3)
    y, mean, rstd = g.layer_norm_fwd(x, want_stats=True, eps=0.5)
    dx, dgamma, dbeta = g.layer_norm_bwd(dy, x, mean, rstd)
    for got, want, what in zip((y, mean, rstd, dx, dgamma, dbeta), _exact(x, dy, None, None, None, real, 0.5), ("y", "mean", "rstd", "dx", "dgamma", "dbeta")):
        _close(got, want, 5e-6, what)
    assert torch.equal(g.layer_norm_fwd(x, eps=0.5), y)


@pytest.mark.parametrize("d", [32, 100, 512, 1100])
def test_strided_rows_and_results_in_place(g, d):
    """Rows inside wider buffers (at an offset that allows no vectors, too) give the bits of contiguous ones up to the order of sums;
    dx may take the place of the residual."""
    for off in (0, 1, 4):
        buf = torch.randn((2, 18, 3 * d + 8), device="cuda")
        x, dy, res = (buf[:, :, i * d + off:(i + 1) * d + off] for i in range(3))
        gamma = torch.rand(d, device="cuda") + 0.5
        y, mean, rstd = g.layer_norm_fwd(x, gamma, None, (4, 8, 6), want_stats=True)
        ref = g.layer_norm_fwd(x.contiguous(), gamma, None, (4, 8, 6))
        assert torch.allclose(y, ref, atol=2e-6, rtol=1e-5)
        dx, dgamma, dbeta = g.layer_norm_bwd(dy, x, mean, rstd, gamma, (4, 8, 6), residual=res)
        keep = res.clone()
        got = g.layer_norm_bwd(dy, x, mean, rstd, gamma, (4, 8, 6), residual=res, out=res)
        assert got[0].data_ptr() == res.data_ptr() and torch.equal(res, dx) and torch.equal(got[1], dgamma) and torch.equal(got[2], dbeta)
        res.copy_(keep)


def test_many_rows_add_up(g):
    """More rows than the persistent CTAs take in one turn: the gradients of the parameters hold every row once."""
    x, dy, res, gamma, beta, valid, real = _make(40, (50, 500, 500), 64, torch.float32, torch.bfloat16, True, 5)
    y, mean, rstd = g.layer_norm_fwd(x, gamma, beta, (50, 500, 500), valid, out_dtype=torch.bfloat16, want_stats=True)
    got = g.layer_norm_bwd(dy, x, mean, rstd, gamma, (50, 500, 500), valid, residual=res)
    _, _, _, edx, ega, ebe = _exact(x, dy, res, gamma, beta, real, 1e-5)
    _close(got[0], edx, 3e-6, "dx")
    _close(got[1], ega, 3e-6, "dgamma")
    _close(got[2], ebe, 3e-6, "dbeta")


def test_gradients_are_differences(g):
    """d/dt of <f(x + t e), w> by a centred difference with t = 2^-6, computed from float results in 64-bit sums.  The third derivative
    leaves t^2 / 6 of a term of the size of the first, the rounding of f 2^-24 sqrt(n) / t: together below 1e-3 of |e| |w|."""
    torch.manual_seed(2)
    B, L, d = 2, 40, 48
    x, e, w = (torch.randn((B, L, d), device="cuda") for _ in range(3))
    gamma, beta = torch.rand(d, device="cuda") + 0.5, torch.randn(d, device="cuda")
    eg = torch.randn(d, device="cuda")
    y, mean, rstd = g.layer_norm_fwd(x, gamma, beta, want_stats=True)
    dx, dgamma, dbeta = g.layer_norm_bwd(w, x, mean, rstd, gamma)
    f = lambda x, ga, be: (g.layer_norm_fwd(x, ga, be).double() * w.double()).sum()
    t = 2.0 ** -6
    for step, grad, direction in (((e, 0 * eg, 0 * eg), dx, e), ((0 * e, eg, 0 * eg), dgamma, eg), ((0 * e, 0 * eg, eg), dbeta, eg)):
        up, down = (f(x + s * step[0], gamma + s * step[1], beta + s * step[2]) for s in (t, -t))
        want = float((grad.double() * direction.double()).sum())
        assert abs(float(up - down) / (2 * t) - want) <= 1e-3 * float(direction.norm() * (w.norm() if direction is e else w.norm() * L ** 0.5))


def test_refusals(g):
    x = torch.randn((2, 6, 32), device="cuda")
    y, mean, rstd = g.layer_norm_fwd(x, want_stats=True)
    v = torch.ones(32, device="cuda")
    for args in ((x[0],), (x, v[:31]), (x, v.bfloat16()), (x, v, v, (1, 2, 2)), (x.transpose(1, 2),)):
        with pytest.raises((AssertionError, g.GsitError)):
            g.layer_norm_fwd(*args)
    with pytest.raises(TypeError):
        g.layer_norm_fwd(x.double())
    with pytest.raises(g.GsitError) as e:
        g.layer_norm_fwd(torch.zeros((1, 1, 8196), device="cuda"))
    assert e.value.code == 2
    with pytest.raises(AssertionError):
        g.layer_norm_bwd(x[:, :5], x, mean, rstd)
    with pytest.raises(AssertionError):
        g.layer_norm_bwd(x, x, mean[:1], rstd)
    with pytest.raises(AssertionError):
        g.layer_norm_bwd(x, x, mean, rstd, residual=x.bfloat16())
    with pytest.raises(g.GsitError) as e:
        g.layer_norm_bwd(x, x, mean, rstd, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    assert e.value.code == 3
