"""Calls on a stream's cache that its own steps do not make: slots that no plan writes."""
import pytest
import torch

from test_gpu_stream import g, nothing_is_flagged   # noqa: F401

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
