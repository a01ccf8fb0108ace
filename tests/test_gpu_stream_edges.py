"""Calls on a stream's cache that its own steps do not make: slots that no plan writes; and pasts in which few positions stand out."""
import pytest
import torch

from stream_reference import Streams, bytes_of, open_blocks
from test_gpu_stream import _attention_close, _rows, g, nothing_is_flagged   # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("t", [torch.bfloat16, torch.float32])
def test_a_first_row_without_a_slot(g, t):
    """Rows with a slot behind one that has none: the segment is left out and flagged, the others are taken, and nothing else is written."""
    B, HK, hd, seg = 2, 2, 16, (40, 3, 33)
    gen = torch.Generator().manual_seed(9)
    caches = [g.stream_cache(B, (70, 70, 70), HK, hd, t, times=True) for _ in range(2)]
    k, v = (torch.randn((B, sum(seg), HK, hd), generator=gen).to(t).cuda() for _ in range(2))
    times = torch.rand((B, sum(seg)), generator=gen).cuda()
    for cache in caches:
        cache.times.fill_(-1.0)
    slots = [g.cache_plan(cache, seg) for cache in caches]
    slots[0][0, 0] = -1                     # stream 0, segment 0: its first row
    slots[0][1, 40] = -1                    # stream 1, segment 1
    slots[1][0, :40] = -1                   # the same entries without any row
    slots[1][1, 40:43] = -1
    for cache, at in zip(caches, slots):
        g.cache_append(cache, k, v, at, seg, times)
        torch.cuda.synchronize()
        flag = g.last_device_status()[1]
        assert flag == (g.DEVFLAG_CLAMPED if at is slots[0] else 0)
    for a, b in zip(*caches):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def _even_tail(g, t, held_as, below):
    """Positions that stand out by `below` nats, one in each warp's walk, with values of 0, and 4 100 others with values of 1: what comes out is the tail's weight.
    Streams that a CTA walks alone, and one that is split over many."""
    hd, n = 16, 4100
    for B, HK in ((75, 2), (1, 1)):
        cache = g.stream_cache(B, (0, n, 1), HK, hd, t, held_as)
        k, v = torch.zeros((B, n, HK, hd), device="cuda"), torch.ones((B, n, HK, hd), device="cuda")
        for block in range(0, 128, 4):          # stages of a warp hold four blocks
            if block < 32 or B == 1:
                k[:, 32 * block + 5], v[:, 32 * block + 5] = 1.0, 0.0
        k, v = k.to(t), v.to(t)
        g.cache_append(cache, k, v, g.cache_plan(cache, (0, n, 0)), (0, n, 0))
        q = torch.full((B, 1, HK, hd), 4 * below / hd, device="cuda").to(t)
        out, lse = g.im_cached_attention_fwd(q, cache, (0, 1, 0), phase=g.PHASE_INTRA, want_lse=True)
        K, V = bytes_of(cache, 0, 1, "k"), bytes_of(cache, 0, 1, "v")
        assert K.shape[0] == n
        x = torch.einsum("hc,jhc->hj", q[0, 0].double(), K) * hd ** -0.5
        p = torch.softmax(x, dim=1)
        want, total = torch.einsum("hj,jhc->hc", p, V), torch.logsumexp(x, dim=1)
        # A weight is rounded to 2^-11 of itself or 2^-32 of the largest (float: 2^-22 and 2^-39); a score to 2^-21 of itself and of 8, twice; the result once.
        score = 2.0 ** -21 * (below + 8)
        weight, least = (2.0 ** -11, 2.0 ** -32) if t is torch.bfloat16 else (2.0 ** -22, 2.0 ** -39)
        room = (torch.finfo(t).eps / 2 * 1.01 + weight + 2 * score) * want + n * least
        off = (out[0].double().reshape(HK, hd) - want).abs()
        assert bool((off <= room).all()), (B, float(off.max()), float(room.min()), float(want.max()))
        assert torch.equal(out, out[:1].expand_as(out))
        assert float((lse[0, :, 0].double() - total).abs().max()) <= 2.0 ** -20 * (below + 8)


@pytest.mark.parametrize("below", [10.0, 14.0, 17.4, 21.0])
@pytest.mark.parametrize("held_as, t", [("e4m3", torch.bfloat16), ("int8", torch.float32), ("e4m3", torch.float32)])
def test_a_long_even_tail(g, held_as, t, below):
    _even_tail(g, t, held_as, below)


@pytest.mark.parametrize("below", [10.0, 14.0, 17.4, 21.0])
def test_a_long_even_tail_of_integers(g, below):
    """What stands out has values of 0, so nothing of its weight may be left in the sums."""
    _even_tail(g, torch.bfloat16, "int8", below)


@pytest.mark.parametrize("cap", [1e-3, 1.0, 50.0, 65.0, 1e3, 1e5, 1e9])
@pytest.mark.parametrize("t", [torch.bfloat16, torch.float32])
def test_caps_of_any_size(g, t, cap):
    """A cap far above the scores changes nothing of them; one far below leaves their signs."""
    B, H, HK, hd, seg, gen = 1, 4, 2, 32, (40, 3, 33), torch.Generator().manual_seed(5)
    cache, ref = g.stream_cache(B, seg, HK, hd, t), Streams(B, "int8")
    q, k, v = _rows(gen, B, sum(seg), H, hd, t), _rows(gen, B, sum(seg), HK, hd, t), _rows(gen, B, sum(seg), HK, hd, t)
    g.cache_append(cache, k, v, g.cache_plan(cache, seg), seg)
    ref.step(seg, [seg], k, v)
    got = g.im_cached_attention_fwd(q, cache, seg, phase=g.PHASE_CUSTOM, custom_mask=0x1FF, softcap=cap, want_lse=True)
    want = ref.attention(q, seg, [seg], open_blocks(None, 0x1FF), hd ** -0.5, softcap=cap)
    _attention_close(got, want, t, cap)


@pytest.mark.parametrize("held_as", ["int8", "e4m3"])
@pytest.mark.parametrize("hd", [16, 32, 64])
def test_large_scores_of_float_rows(g, held_as, hd):
    """Queries and keys of one sign, so that nothing cancels and every sum is cut off the same way; log-sum-exps show the scores' errors."""
    t, B, HK, H, seg = torch.float32, 16, 8, 24, (40, 64, 33)
    for seed in range(2):
        gen = torch.Generator().manual_seed(seed)
        q, k, v = (_rows(gen, B, sum(seg), h, hd, t) for h in (H, HK, HK))
        q, k = q.abs(), k.abs()
        cache = g.stream_cache(B, seg, HK, hd, t, held_as)
        g.cache_step(cache, q, k, v, seg)
        _, lse = g.im_cached_attention_fwd(q, cache, seg, phase=g.PHASE_CUSTOM, custom_mask=0x1FF, want_lse=True)
        for b in range(B):
            K = torch.cat([bytes_of(cache, b, s, "k") for s in range(3)]).repeat_interleave(H // HK, dim=1)
            x = torch.einsum("ihc,jhc->hij", q[b].double(), K) * hd ** -0.5
            # A score, relative to itself: 2^-22 by the two terms of a query, 2^-22 by those of open keys, 2^-22 for products that are cut at 2^-23 twice (the
            # terms inside and the sum), 2^-22 for four roundings to float of 2^-24.  Exponentials, sums and logarithm: 2^-20 in all.
            room = 2.0 ** -20 * x.amax(dim=2) + 2.0 ** -20
            off = (lse[b].double() - torch.logsumexp(x, dim=2)).abs()
            assert bool((off <= room).all()), (seed, b, float((off / room).max()), float(x.max()))
