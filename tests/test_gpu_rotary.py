"""Rotary positions with several axes, forward and backward, against complex products in 64 bits."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

# One rotated feature is u c - v s with |c|, |s| <= 1: angle to 2^-20 turns (6e-6 rad at the worst, mostly far less), two products and a
# sum in float, then one rounding to the type.  |u| and |v| of N(0, 1) draws stay below 6 here.
TOL = {torch.float32: dict(atol=1e-4, mean=2e-6), torch.bfloat16: dict(atol=6 * 2 ** -8, mean=2 ** -8)}


@pytest.fixture(scope="module")
def g():
    import paper_2505_01068_b200 as lib
    lib.load()
    return lib


def _reference(x, pos, sections, base, interleaved, back, real):
    """x [B, L, H, hd] in float64; pos [axes, B, L]; real [B, L]."""
    n = sum(sections)
    axis = [i for i, m in enumerate(sections) for _ in range(m)]
    angle = np.stack([pos[axis[p]].astype(np.float64) * base ** (-p / n) for p in range(n)], axis=-1)
    turn = np.exp((-1j if back else 1j) * angle)[:, :, None, :]
    y = x.copy()
    if interleaved:
        z = (x[..., 0:2 * n:2] + 1j * x[..., 1:2 * n:2]) * turn
        y[..., 0:2 * n:2], y[..., 1:2 * n:2] = z.real, z.imag
    else:
        z = (x[..., :n] + 1j * x[..., n:2 * n]) * turn
        y[..., :n], y[..., n:2 * n] = z.real, z.imag
    y[~real] = 0
    return y


def _real(seg, valid, B):
    n = np.tile(seg, (B, 1)) if valid is None else valid
    return np.concatenate([np.arange(seg[s])[None, :] < n[:, s:s + 1] for s in range(3)], axis=1)


CASES = [  # dtype, batch, segments, heads, key heads, head_dim, sections, interleaved, far
    ("bf16", 3, (5, 40, 21), 8, 8, 8, (2, 1, 1), False, 0),
    ("bf16", 2, (5, 33, 12), 4, 2, 16, (4, 2, 2), False, 1000),
    ("bf16", 2, (1, 1, 1), 8, 8, 64, (16, 8, 8), False, 100000),
    ("bf16", 1, (7, 0, 30), 3, 1, 64, (32,), True, 0),
    ("bf16", 2, (0, 1, 0), 2, 2, 32, (8, 8), False, 2 ** 31 - 64),
    ("bf16", 2, (9, 17, 5), 2, 2, 8, (4,), True, 5),
    ("bf16", 2, (9, 17, 5), 2, 1, 32, (5, 3, 2), False, 5),       # part of the head, odd sections
    ("f32", 2, (5, 33, 12), 4, 4, 8, (2, 1, 1), False, 0),
    ("f32", 2, (5, 33, 12), 2, 2, 20, (4, 3, 3), True, 1000),
    ("f32", 1, (130, 3, 70), 1, 1, 128, (22, 21, 21), False, 0),
    ("f32", 2, (4, 9, 2), 3, 3, 6, (1, 1, 0), False, 3),          # rows whose addresses allow no vectors
    ("f32", 1, (3, 4, 5), 2, 2, 5, (0, 2, 0), True, 3),
]


@pytest.mark.parametrize("case", CASES, ids=str)
@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("padded", [False, True])
def test_rotation_of_the_fused_buffer(g, case, back, padded):
    dtype, B, seg, H, HK, hd, sections, interleaved, far = case
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    rng, L = np.random.default_rng(7), sum(seg)
    valid = np.stack([rng.integers(0, m + 1, size=B) for m in seg], axis=1).astype(np.int32) if padded else None
    real = _real(seg, valid, B)
    fused = torch.from_numpy(rng.standard_normal((B, L, (H + 2 * HK) * hd), dtype=np.float32)).cuda().to(t)
    fused[torch.from_numpy(~real).cuda()] = float("nan")          # padding is never read
    q = fused[:, :, :H * hd].view(B, L, H, hd)
    k = fused[:, :, H * hd:(H + HK) * hd].view(B, L, HK, hd)
    pos = (rng.integers(0, 50, size=(len(sections), B, L)) + far).astype(np.int32)
    call = g.rotary_bwd if back else g.rotary_fwd
    dev_valid = None if valid is None else torch.from_numpy(valid).cuda()
    got = call(q, k, torch.from_numpy(pos).cuda(), sections, seg, dev_valid, base=500.0, interleaved=interleaved)
    for y, x in zip(got, (q, k)):
        want = _reference(np.nan_to_num(x.float().cpu().numpy().astype(np.float64)), pos, sections, 500.0, interleaved, back, real)
        y = y.float().cpu().numpy()
        assert not np.signbit(y[~real]).any() and not y[~real].any()
        err = np.abs(y - want)
        assert err.max(initial=0) <= TOL[t]["atol"] and err.mean() <= TOL[t]["mean"], (err.max(), err.mean())
    assert g.last_device_status() == (0, 0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_in_place_shared_positions_and_only_q(g, dtype):
    """The same bits in place, out of place, without k, and with one row of positions for all samples."""
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    B, seg, H, hd, sections = 3, (5, 40, 21), 8, 16, (4, 2, 2)
    L = sum(seg)
    torch.manual_seed(0)
    qkv = torch.randn((B, L, 3, H, hd), device="cuda").to(t)
    pos = torch.randint(0, 500, (3, L), device="cuda", dtype=torch.int32)
    q, k = g.rotary_fwd(qkv[:, :, 0], qkv[:, :, 1], pos, sections, seg)
    each = pos[:, None, :].expand(3, B, L).contiguous()
    assert all(torch.equal(x, y) for x, y in zip((q, k), g.rotary_fwd(qkv[:, :, 0], qkv[:, :, 1], each, sections, seg)))
    assert torch.equal(q, g.rotary_fwd(qkv[:, :, 0], None, pos, sections, seg))
    v = qkv[:, :, 2].clone()
    g.rotary_fwd(qkv[:, :, 0], qkv[:, :, 1], pos, sections, seg, out_q=qkv[:, :, 0], out_k=qkv[:, :, 1])
    assert torch.equal(qkv[:, :, 0], q) and torch.equal(qkv[:, :, 1], k) and torch.equal(qkv[:, :, 2], v)


def test_the_backward_pass_is_the_derivative(g):
    """Differences of the forward pass along a direction, in 64-bit sums of float results: the map is linear, so f(x + e) - f(x) = f(e)
    to rounding, and <f(e), w> = <e, f'(w)>."""
    B, seg, H, hd, sections = 2, (5, 30, 20), 4, 32, (8, 4, 4)
    L = sum(seg)
    torch.manual_seed(1)
    x, e, w = (torch.randn((B, L, H, hd), device="cuda") for _ in range(3))
    pos = torch.randint(0, 300, (3, B, L), device="cuda", dtype=torch.int32)
    f = lambda t: g.rotary_fwd(t, None, pos, sections, seg).double()
    left = ((f(x + e) - f(x)) * w.double()).sum()
    right = (e.double() * g.rotary_bwd(w, None, pos, sections, seg).double()).sum()
    assert abs(float(left - right)) <= 1e-6 * float(e.double().norm() * w.double().norm())


def test_refusals(g):
    q = torch.randn((2, 6, 2, 16), device="cuda")
    pos = torch.zeros((3, 2, 6), dtype=torch.int32, device="cuda")
    ok = dict(sections=(4, 2, 2), seg_len=(1, 2, 3))
    g.rotary_fwd(q, q.clone(), pos, **ok)
    for bad in (dict(ok, sections=(4, 4, 2)), dict(ok, sections=(0, 0, 0)), dict(ok, base=0.0), dict(ok, base=float("nan"))):
        with pytest.raises((g.GsitError, AssertionError)):
            g.rotary_fwd(q, None, pos, **bad)
    for bad in (dict(ok, seg_len=(1, 2, 2)), dict(ok, sections=(4, 4)), dict(ok, sections=(8, -1, 1))):
        with pytest.raises(AssertionError):
            g.rotary_fwd(q, None, pos, **bad)
    with pytest.raises(AssertionError):
        g.rotary_fwd(q, None, pos.long(), **ok)
    with pytest.raises(AssertionError):
        g.rotary_fwd(q, q.bfloat16(), pos, **ok)
    with pytest.raises(AssertionError):
        g.rotary_fwd(q.transpose(1, 2), None, pos, **ok)
    with pytest.raises(TypeError):
        g.rotary_fwd(q.double(), None, pos, **ok)
