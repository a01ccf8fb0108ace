"""Whole steps of streams: the three calls in one, steps that are refused, streams that find no pages, steps that are taken again."""
import pytest
import torch

from test_gpu_stream import _rows, g, nothing_is_flagged   # noqa: F401

pytestmark = pytest.mark.gpu


def _parts(cache):
    return [t.view(torch.uint8).clone() for t in cache if t is not None]


def _same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b, strict=True))


@pytest.mark.parametrize("t, held_as, hd, table", [(torch.bfloat16, "int8", 64, 0), (torch.float32, "e4m3", 16, 0), (torch.bfloat16, "e4m3", 64, 60000)])
def test_a_step_in_one_call(g, t, held_as, hd, table):
    """The same bits as plan, append and attention one after the other; with long tables (evenly shared blocks), too."""
    B, H, HK, gen = 3, 4, 2, torch.Generator().manual_seed(hd)
    seg = (40, 3, 70)
    caches = [g.stream_cache(B, [max(table, 200)] * 3, HK, hd, t, held_as, pages=60, times=True) for _ in range(2)]
    slopes = torch.rand(H, generator=gen).cuda()
    for i in range(3):
        q, k, v = (_rows(gen, B, sum(seg), h, hd, t) for h in (H, HK, HK))
        times = torch.rand((B, sum(seg)), generator=gen).cuda()
        valid = torch.tensor([[40, 0, 3], [1, 3, 70], [7, 1, 33]], dtype=torch.int32, device="cuda")
        ended = torch.tensor([0, i % 2, 0], dtype=torch.int32, device="cuda")
        rule = dict(phase=g.PHASE_CUSTOM, custom_mask=0x1FF, softcap=30.0, slopes=slopes, causal=True)
        slots = g.cache_plan(caches[0], seg, valid, ended)
        g.cache_append(caches[0], k, v, slots, seg, times)
        want = g.im_cached_attention_fwd(q, caches[0], seg, valid, times=times, **rule)
        given = torch.empty_like(want), torch.empty_like(slots)
        got = g.cache_step(caches[1], q, k, v, seg, valid, ended, times=times, **rule, **(dict(out=given[0], slots=given[1]) if i == 2 else {}))
        assert torch.equal(got[0], want) and torch.equal(got[1], slots) and (i < 2 or got[0].data_ptr() == given[0].data_ptr() and got[1].data_ptr() == given[1].data_ptr())
        assert _same(_parts(caches[0]), _parts(caches[1]))


@pytest.mark.parametrize("timed", [False, True])
def test_a_refused_step_changes_nothing(g, timed):
    """The layer's cache is as it was, bit by bit, and the corrected step is the one that would have been."""
    torch.manual_seed(3)
    B, D, most, seg = 2, 64, (70, 70, 70), (20, 33, 1)
    layer = g.ImEncoderLayer(D, 4, most, kv_heads=2)
    caches = [layer.open_cache(B, most, times=timed) for _ in range(2)]
    x = torch.randn((2, B, sum(seg), D), device="cuda")
    times = torch.rand((B, sum(seg)), device="cuda") if timed else None
    moments = torch.rand((B, sum(seg)), device="cuda")
    good = dict(times=times, causal=True)
    for cache in caches:
        layer.step(cache, x[0], seg, **good)
    before = _parts(caches[0])
    bad = [dict(good, softcap=float("nan")), dict(good, phase=17), dict(good, custom_mask=0x200, phase=g.PHASE_CUSTOM), dict(good, documents=None), dict(good, prefix=moments[0]),
           dict(good, slope=2.0), dict(good, slopes=torch.ones(3, device="cuda")), dict(good, slopes=torch.ones(4)), dict(good, workspace=torch.empty(8)),
           dict(good, ended=torch.zeros(1, dtype=torch.int32, device="cuda")), dict(good, times=moments[:, 1:]),
           dict(good, times=None) if timed else dict(good, times=moments)]
    for kw in bad:
        with pytest.raises((AssertionError, TypeError, g.GsitError)):
            layer.step(caches[0], x[1], seg, **kw)
        torch.cuda.synchronize()
        assert _same(_parts(caches[0]), before), kw
    assert torch.equal(layer.step(caches[0], x[1], seg, **good), layer.step(caches[1], x[1], seg, **good))
    assert _same(_parts(caches[0]), _parts(caches[1]))


@pytest.mark.parametrize("padded", [False, True])
def test_streams_that_find_no_pages(g, padded):
    """Rows that did not join the cache are +0, whether or not lengths are given, and the others are what they are with pages for all."""
    torch.manual_seed(5)
    B, D, most, seg = 3, 32, (64, 64, 64), (33, 2, 40)
    layer = g.ImEncoderLayer(D, 4, most)
    few, many = layer.open_cache(B, most, pages=9), layer.open_cache(B, most)
    x = torch.randn((B, sum(seg), D), device="cuda")
    valid = torch.tensor([list(seg)] * B, dtype=torch.int32, device="cuda") if padded else None
    rule = dict(phase=g.PHASE_INTRA)
    want = layer.step(many, x, seg, valid, **rule)
    assert g.last_device_status() == (0, 0)
    got = layer.step(few, x, seg, valid, **rule)
    torch.cuda.synchronize()
    assert g.last_device_status()[1] == g.DEVFLAG_FULL
    # five blocks a stream: the first stream's, the second's first two segments; its third finds one page, and nothing behind it is taken
    real = torch.zeros((B, sum(seg), 1), dtype=torch.bool, device="cuda")
    real[0], real[1, :35] = True, True
    assert few.lengths.cpu().tolist() == [[33, 2, 40], [33, 2, 0], [0, 0, 0]]
    assert torch.equal(got, torch.where(real, want, 0.0)) and not torch.signbit(got[~real.expand_as(got)]).any() and bool(want[~real.expand_as(got)].any())


def test_a_layers_step_taken_again(g):
    """A step with other rows from the lengths before it: as if the first one had never been."""
    torch.manual_seed(6)
    B, D, most, seg = 2, 32, (80, 80, 80), (3, 32, 1)
    layer = g.ImEncoderLayer(D, 4, most)
    x = torch.randn((4, B, sum(seg), D), device="cuda")
    caches = [layer.open_cache(B, most) for _ in range(2)]
    for cache in caches:
        layer.step(cache, x[0], seg)
    held = caches[0].lengths.clone()
    layer.step(caches[0], x[1], seg)
    for i, kw in ((2, dict(held=held)), (3, {})):
        assert torch.equal(layer.step(caches[0], x[i], seg, **kw), layer.step(caches[1], x[i], seg))
    assert torch.equal(caches[0].lengths, caches[1].lengths)
    assert all(torch.equal(a, b) for a, b in zip(g.cache_read(caches[0], most), g.cache_read(caches[1], most)))
