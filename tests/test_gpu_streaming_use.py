"""The streaming calls together, as a program uses them: a layer's steps against the same layer over rows, captured, with streams that end; and the example."""
import sys
from pathlib import Path

import pytest
import torch

pytestmark = pytest.mark.gpu
sys.path.insert(0, str(Path(__file__).resolve().parent.parent / "examples"))


@pytest.fixture(scope="module")
def g():
    import paper_2505_01068_b200 as lib
    lib.load()
    return lib


@pytest.fixture(autouse=True)
def nothing_is_flagged(g):
    """No test leaves a flag behind that it has not looked at."""
    yield
    assert g.last_device_status() == (0, 0)


@pytest.mark.parametrize("qk_norm", [False, True])
def test_a_layer_over_streams(g, qk_norm):
    """In float: while blocks are open nothing is lost, so the first steps are those of the layer over rows; behind them, those of the layer's attention over
    what the cache gives back."""
    torch.manual_seed(2)
    B, D, H, HK, most = 3, 64, 4, 2, (40, 70, 90)
    layer = g.ImEncoderLayer(D, H, most, kv_heads=HK, sections=(4, 2, 2), dtype=torch.float32, qk_norm=qk_norm)
    cache = layer.open_cache(B, most, held_as="int8", times=True)
    rule = dict(phase=g.PHASE_CUSTOM, custom_mask=0x1FF, causal=True, softcap=20.0)
    L = sum(most)
    x = torch.randn((B, L, D), device="cuda")
    place, seg = layer.place, layer.segment
    when = (place * torch.tensor([1.0, 0.5, 0.4], device="cuda")[seg]).float().expand(B, L).contiguous()
    pos = torch.stack([place, place // 3, place % 3]).int()[:, None].expand(3, B, L).contiguous()
    first = [0, most[0], most[0] + most[1]]
    held = [0, 0, 0]
    with torch.no_grad():
        q, k, v = layer.project(x, None, pos)
        for i, step in enumerate([(1, 2, 3), (9, 0, 20), (1, 1, 1), (0, 28, 7), (20, 30, 40), (1, 1, 1), (2, 3, 4)]):
            at = torch.cat([first[s] + held[s] + torch.arange(step[s], device="cuda") for s in range(3)])
            y = layer.step(cache, x[:, at], step, None, pos[:, :, at].contiguous(), when[:, at], **rule)
            held = [a + b for a, b in zip(held, step)]
            valid = torch.tensor([held] * B, dtype=torch.int32, device="cuda")
            keys, values = (k, v) if max(held) < 32 else g.cache_read(cache, most)
            att = g.im_scored_attention_fwd(q[:, at].contiguous(), keys, values, most, valid, q_len=step, times=when, **rule)
            want = layer.finish(x[:, at], att, None, step)
            # float all the way: attention as in the other tests, then a norm and products of 64 and 256 terms: 1e-4 of values of size 1 to 5 is 2^-13
            assert float((y - want).abs().max()) <= 2e-4, i
    assert cache.lengths.cpu().tolist() == [held] * B and g.last_device_status() == (0, 0)


def test_streams_that_end(g):
    """Streams that begin anew in the place of others are as if they had been alone."""
    torch.manual_seed(4)
    B, D, step = 4, 32, (2, 3, 1)
    layer = g.ImEncoderLayer(D, 4, (80, 80, 80), dtype=torch.bfloat16, qk_norm=True)
    both, alone = layer.open_cache(B, (80, 80, 80), "e4m3"), layer.open_cache(B, (80, 80, 80), "e4m3")
    x = torch.randn((24, B, 6, D), device="cuda")
    stop = torch.tensor([0, 1, 0, 1], dtype=torch.int32, device="cuda")
    for i in range(24):
        y = layer.step(both, x[i], step, phase=g.PHASE_INTER_FWD, ended=stop if i == 12 else None)
        if i >= 12:
            z = layer.step(alone, x[i], step, phase=g.PHASE_INTER_FWD)
            assert torch.equal(y[stop.bool()], z[stop.bool()])
            assert not torch.equal(y[0], z[0])


def test_the_example(g):
    import stream_encoder
    for held_as in ("int8", "e4m3"):
        worst, held, pages, rows = stream_encoder.run(4, 40, held_as)
        assert held > 0 and 0 < pages and worst == worst
