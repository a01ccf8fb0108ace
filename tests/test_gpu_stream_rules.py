"""Attention over a cache under every rule: by the index inside the segment, and over evenly shared blocks with moments, several rows a segment and blocks with NaN;
rows read into given results."""
import ctypes
import math

import pytest
import torch

from stream_reference import Streams, bytes_of, open_blocks
from test_gpu_stream import _attention_close, _rows, _valid, g, nothing_is_flagged   # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("t, held_as, hd, H, HK", [(torch.bfloat16, "int8", 64, 4, 2), (torch.bfloat16, "e4m3", 8, 6, 2), (torch.float32, "int8", 16, 4, 4), (torch.float32, "e4m3", 32, 4, 1)])
def test_rules_by_index(g, t, held_as, hd, H, HK):
    """A cache without moments: causality and slopes go by the index inside the segment, also between segments of unlike lengths."""
    B, gen = 2, torch.Generator().manual_seed(hd + H)
    cache, ref = g.stream_cache(B, (110, 160, 120), HK, hd, t, held_as), Streams(B, held_as)
    for seg in ((33, 90, 64), (1, 1, 1), (20, 3, 40), (2, 5, 0)):
        valid = _valid(gen, seg, B)
        q, k, v = (_rows(gen, B, sum(seg), h, hd, t) for h in (H, HK, HK))
        g.cache_append(cache, k, v, g.cache_plan(cache, seg, valid), seg)
        ref.step(seg, valid.cpu(), k, v)
        for rule in (dict(phase=g.PHASE_CUSTOM, custom_mask=0x1FF, causal=True), dict(phase=g.PHASE_INTRA, causal=True, softcap=9.0), dict(phase=g.PHASE_INTER_FWD, slopes=True),
                     dict(phase=g.PHASE_CUSTOM, custom_mask=0x0E6, slopes=True, causal=True)):
            rule = dict(rule)
            if rule.pop("slopes", False):
                rule["slopes"] = torch.rand(H, generator=gen).cuda()
            got = g.im_cached_attention_fwd(q, cache, seg, valid, want_lse=True, **rule)
            pairs = open_blocks(rule.pop("phase"), rule.pop("custom_mask", 0))
            _attention_close(got, ref.attention(q, seg, valid.cpu(), pairs, hd ** -0.5, **rule), t, (seg, rule))


def _needs_workspace(g, cache, seg, H, hd, t, rule):
    from test_ops_refusals import Rule
    from test_stream_refusals import Cache
    fn = g.load().gsit_cached_attention_workspace
    fn.restype = ctypes.c_size_t
    B = cache.tables.shape[0]
    c = Cache(1 if cache.keys.dtype is torch.float8_e4m3fn else 0, g.DTYPE_BF16 if t is torch.bfloat16 else g.DTYPE_F32, B, cache.open_keys.shape[3], hd, cache.free.numel(),
              cache.tables.shape[2], *[x.data_ptr() for x in (cache.keys, cache.values, cache.key_scale, cache.value_scale)], None if cache.times is None else cache.times.data_ptr(),
              *[x.data_ptr() for x in (cache.open_keys, cache.open_values, cache.tables, cache.lengths, cache.free, cache.n_free)])
    shape = g.make_shape(B, seg, H * hd, H, None, c.dtype, g.PHASE_CUSTOM, 0x1FF)
    r = Rule(0.0, int(bool(rule.get("causal"))), 0, None, None, None, None, 0, (ctypes.c_int32 * 3)())
    return fn(ctypes.byref(shape), ctypes.byref(r), ctypes.byref(c))


# lengths of the streams, table's positions, rows of the step, heads, key heads, width, held as, type, moments
SHARED = [([(700, 2500, 90), (33, 0, 64), (3, 900, 1000)], 60000, (1, 2, 1), 4, 2, 64, "int8", torch.bfloat16, True),
          ([(3000, 70, 800)], 30000, (4, 2, 2), 4, 2, 64, "e4m3", torch.bfloat16, True),
          ([(100, 1500, 33), (640, 32, 31)], 60000, (1, 1, 2), 6, 2, 32, "e4m3", torch.float32, True),
          ([(900, 1500, 33), (40, 64, 31)], 300000, (2, 1, 1), 2, 2, 8, "int8", torch.float32, False),
          ([(64, 2100, 600), (1, 1, 1)], 100000, (1, 2, 2), 2, 2, 16, "int8", torch.bfloat16, False)]


@pytest.mark.parametrize("case", SHARED, ids=lambda c: "-".join(str(x) for x in c[1:]).replace(" ", ""))
@pytest.mark.parametrize("broken", [False, True])
def test_shares_under_rules(g, case, broken):
    """Rows that see nothing, rows that see what some of the CTAs walk and nothing of the others', cap and slopes; with `broken`, full blocks of NaN keys and of NaN values."""
    lengths, table, seg, H, HK, hd, held_as, t, timed = case
    B, gen = len(lengths), torch.Generator().manual_seed(hd)
    most = [max(n[s] for n in lengths) for s in range(3)]
    pages = sum((m + 70) // 32 for m in most) * B
    cache = g.stream_cache(B, (table, table, table), HK, hd, t, held_as, pages=pages, times=timed)
    k, v = (_rows(gen, B, sum(most), HK, hd, t, 0.3) for _ in range(2))
    if broken:
        k[0, 40, 0, 1] = float("nan")              # stream 0, its first segment's second block, or (short ones) the next segment's rows
        v[B - 1, most[0] + 5, HK - 1, 0] = float("inf")
    n = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    # moments of a segment run from 0 to 100 in order, those of the rows lie before all of them, among them and behind
    place = torch.cat([torch.arange(m) * (100.0 / max(m, 1)) for m in most])
    moments = place.expand(B, -1).contiguous().cuda() if timed else None
    g.cache_append(cache, k, v, g.cache_plan(cache, most, n), most, moments)
    L = sum(seg)
    q, nk, nv = _rows(gen, B, L, H, hd, t, 0.3), _rows(gen, B, L, HK, hd, t, 0.3), _rows(gen, B, L, HK, hd, t, 0.3)
    when = (torch.tensor([-1.0, 31.0, 57.5, 200.0, 88.0, 12.0, 99.0, 64.0])[:L].expand(B, -1).contiguous().cuda()) if timed else None
    late = None if when is None else torch.full_like(when, 300.0)   # the step's own keys are nobody's: every row is earlier
    slots = g.cache_plan(cache, seg)
    g.cache_append(cache, nk, nv, slots, seg, late)
    now = cache.lengths.cpu()
    rules = [dict(causal=True), dict(causal=True, slopes=torch.rand(H, generator=gen) / 20, softcap=30.0), dict(slopes=torch.rand(H, generator=gen)), dict(softcap=4.0)]
    for mask in (0x1FF, 0x062):
        for rule in rules:
            rule = dict(rule)
            slopes = rule.get("slopes")
            if slopes is not None:
                rule["slopes"] = slopes.cuda()
            assert _needs_workspace(g, cache, seg, H, hd, t, rule) > 0
            got = g.im_cached_attention_fwd(q, cache, seg, phase=g.PHASE_CUSTOM, custom_mask=mask, times=when, want_lse=True, **rule)
            again = g.im_cached_attention_fwd(q, cache, seg, phase=g.PHASE_CUSTOM, custom_mask=mask, times=when, want_lse=True, **rule)
            assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(got, again))
            ref, size = (torch.zeros((B, L, H, hd), dtype=torch.float64) for _ in range(2))
            lse, scores = torch.full((B, H, L), -math.inf, dtype=torch.float64), torch.zeros((B, H, L), dtype=torch.float64)
            for b in range(B):
                keys, values = ([bytes_of(cache, b, s, name) for s in range(3)] for name in "kv")
                theirs = [cache.times[cache.tables[b, s, :(int(now[b, s]) + 31) // 32].long()].flatten()[:int(now[b, s])].double() if timed
                          else torch.arange(int(now[b, s]), device="cuda").double() for s in range(3)]
                row = 0
                for s in range(3):
                    over = [r for r in range(3) if mask >> (3 * s + r) & 1]
                    for i in range(seg[s]):
                        K, V = (torch.cat([x[r] for r in over]).repeat_interleave(H // HK, dim=1) for x in (keys, values))
                        at = torch.cat([theirs[r] for r in over])
                        mine = when[b, row].double() if timed else torch.tensor(float(now[b, s]) - seg[s] + i, device="cuda", dtype=torch.float64)
                        x = torch.einsum("hc,jhc->hj", q[b, row].double(), K) * hd ** -0.5
                        if "softcap" in rule:
                            x = torch.tanh(x / rule["softcap"]) * rule["softcap"]
                        if slopes is not None:
                            x = x - slopes.cuda().double()[:, None] * (mine - at).abs()
                        sees = at <= mine if rule.get("causal") else torch.ones_like(at, dtype=torch.bool)
                        if sees.any():
                            x, V = x[:, sees], V[sees]
                            total = torch.logsumexp(x, dim=1)
                            p = torch.exp(x - total[:, None])
                            ref[b, row] = torch.einsum("hj,jhc->hc", p, V).cpu()
                            size[b, row] = torch.einsum("hj,jhc->hc", p, V.abs()).amax(dim=1, keepdim=True).expand(H, hd).cpu()
                            lse[b, :, row], scores[b, :, row] = total.cpu(), x.abs().amax(dim=1).cpu()
                        row += 1
            _attention_close(got, (ref, lse, size, scores), t, (mask, rule))
            if broken and mask == 0x1FF and not rule.get("causal"):
                assert torch.isnan(got[0][0]).any() and (lengths[B - 1][1] < 32 or torch.isnan(got[0][B - 1]).any())   # (a shorter one does not hold the row)


@pytest.mark.parametrize("t", [torch.bfloat16, torch.float32])
def test_rows_into_given_results(g, t):
    """cache_read into parts of wider rows: what lies beside them stays, and rows behind the last one held are +0."""
    B, HK, hd, seg, gen = 2, 2, 16, (40, 3, 64), torch.Generator().manual_seed(8)
    cache = g.stream_cache(B, seg, HK, hd, t)
    k, v = (_rows(gen, B, sum(seg), HK, hd, t) for _ in range(2))
    g.cache_append(cache, k, v, g.cache_plan(cache, seg, torch.tensor([[40, 3, 64], [32, 0, 33]], dtype=torch.int32, device="cuda")), seg)
    want = g.cache_read(cache, seg)
    wide = torch.full((B, sum(seg), 3 * HK, hd), 7.0, dtype=t, device="cuda")
    got = g.cache_read(cache, seg, wide[:, :, :HK], wide[:, :, 2 * HK:])
    assert got[0].data_ptr() == wide.data_ptr() and torch.equal(wide[:, :, :HK], want[0]) and torch.equal(wide[:, :, 2 * HK:], want[1])
    assert bool((wide[:, :, HK:2 * HK] == 7.0).all()) and not want[0][1, 40:].narrow(0, 0, 3).any() and not torch.signbit(want[0][1, 32:40]).any()
    for bad in (wide[:, 1:, :HK], wide[:, :, :HK].float() if t is torch.bfloat16 else wide[:, :, :HK].bfloat16(), torch.empty((B, sum(seg), HK, hd), dtype=t)):
        with pytest.raises((AssertionError, TypeError, g.GsitError)):
            g.cache_read(cache, seg, bad, wide[:, :, 2 * HK:])
