"""Rotations over more rows than the persistent CTAs take in one turn: every number of pairs that a head may have, in every form of the
kernel, against products in 64 bits.  A CTA then computes the next block's angles while this block's are read."""
import pytest
import torch

pytestmark = pytest.mark.gpu

# u c - v s of N(0, 1) draws (below 8 here) at positions of some hundred: the angle's remainder in float (2^-25 turns), sine, cosine, two
# products and a sum, some 6e-8 each; bf16: one rounding of a result below 16 (half of 2^-4).
ATOL = {torch.float32: 1e-5, torch.bfloat16: 0.04}


@pytest.fixture(scope="module")
def g():
    import paper_2505_01068_b200 as lib
    lib.load()
    return lib


def _turned(x, pos, pairs, interleaved, real):
    """x [1, L, H, hd] in float64 by positions [1, L], base 10000."""
    angle = pos[0].double()[:, None] * 10000.0 ** (-torch.arange(pairs, device="cuda", dtype=torch.float64) / pairs)
    c, s = angle.cos()[None, :, None], angle.sin()[None, :, None]
    x = torch.where(real[None, :, None, None], x.double(), 0.0)
    y = x.clone()
    lo, hi = (x[..., 0:2 * pairs:2], x[..., 1:2 * pairs:2]) if interleaved else (x[..., :pairs], x[..., pairs:2 * pairs])
    a, b = lo * c - hi * s, lo * s + hi * c
    if interleaved:
        y[..., 0:2 * pairs:2], y[..., 1:2 * pairs:2] = a, b
    else:
        y[..., :pairs], y[..., pairs:2 * pairs] = a, b
    return y


def _check(g, dtype, pairs, hd, H, HK, interleaved, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    # three turns and a bit of four CTAs an SM, with as many rows in a block as there can be
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    L = 3 * 4 * sms * min(64, max(1, 256 // pairs)) + 17
    seg = (L // 3, L // 2, L - L // 3 - L // 2)
    valid = torch.tensor([[seg[0] - L // 9, seg[1], seg[2] // 2]], dtype=torch.int32, device="cuda")
    real = torch.cat([torch.arange(m, device="cuda") < n for m, n in zip(seg, valid[0].tolist())])
    q = torch.randn((1, L, H, hd), device="cuda", generator=gen).to(dtype)
    k = torch.randn((1, L, HK, hd), device="cuda", generator=gen).to(dtype) if HK else None
    pos = torch.randint(0, 500, (1, L), device="cuda", generator=gen, dtype=torch.int32)
    for x in (q, k):
        if x is not None:
            x[:, ~real] = float("nan")
    got = g.rotary_fwd(q, k, pos, (pairs,), seg, valid, interleaved=interleaved)
    back = g.rotary_bwd(q, k, -pos, (pairs,), seg, valid, interleaved=interleaved)
    for y, z, x in zip((got,) if k is None else got, (back,) if k is None else back, (q, k)):
        want = _turned(x, pos, pairs, interleaved, real)
        assert float((y.double() - want).abs().max()) <= ATOL[dtype], (pairs, hd, H, HK)
        assert float((z.double() - want).abs().max()) <= ATOL[dtype], (pairs, hd, H, HK)
        assert not y[:, ~real].float().any() and not torch.signbit(y[:, ~real]).any()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("interleaved", [False, True])
def test_every_number_of_pairs(g, dtype, interleaved):
    """One head alone (the most rows in a block), whole and with features that are copied; two heads with one key head."""
    for pairs in range(1, 65):
        _check(g, dtype, pairs, 2 * pairs, 1, 0, interleaved, pairs)
        _check(g, dtype, pairs, 2 * pairs + 1, 1, 0, interleaved, pairs)
        _check(g, dtype, pairs, 2 * pairs, 2, 1, interleaved, pairs)
    assert g.last_device_status() == (0, 0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("hd", [4, 8, 12, 24, 36, 48, 56, 64, 128])
def test_head_widths_of_models(g, dtype, interleaved, hd):
    """Four and eight heads, and as many that a block's units outnumber the offsets that registers hold."""
    for H, HK in ((4, 4), (8, 2), (80, 16)):
        _check(g, dtype, hd // 2, hd, H, HK, interleaved, hd)
    assert g.last_device_status() == (0, 0)
