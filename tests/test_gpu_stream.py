"""A stream's cache in 8 bits, its tables and attention over it, step by step against plain lists of rows in 64 bits."""
import numpy as np
import pytest
import torch

from stream_reference import BLOCK, Streams, bytes_of, open_blocks

pytestmark = pytest.mark.gpu


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


def _rows(gen, B, L, H, hd, t, spread=1.0):
    x = torch.randn((B, L, H, hd), generator=gen) * torch.exp(spread * torch.randn((B, 1, H, hd), generator=gen))
    return x.to(t).cuda()


def _check_plan(g, cache, slots, seg, valid, old, ref):
    """Slots, lengths and tables fit together, and no page has two blocks."""
    tables, lengths, slots = cache.tables.cpu().numpy(), cache.lengths.cpu().numpy(), slots.cpu().numpy()
    first = np.concatenate([[0], np.cumsum(seg)])
    used = tables[tables >= 0]
    n_free = int(cache.n_free)
    assert len(set(used.tolist())) == len(used) and n_free + len(used) == cache.free.numel()
    assert sorted(used.tolist() + cache.free[:n_free].cpu().tolist()) == list(range(cache.free.numel()))
    for b in range(len(ref.rows)):
        for s in range(3):
            n = int(valid[b][s])
            assert lengths[b, s] == old[b][s] + n
            at = np.arange(old[b][s], old[b][s] + n)
            assert (slots[b, first[s]:first[s] + n] == tables[b, s, at // BLOCK] * BLOCK + at % BLOCK).all()
            assert (slots[b, first[s] + n:first[s + 1]] == -1).all()
            assert ((tables[b, s] >= 0).sum() == (lengths[b, s] + BLOCK - 1) // BLOCK)


# dtype, held as, head width, heads, key heads, batch, steps (rows of each segment)
STREAMS = [
    ("bf16", "int8", 64, 4, 2, 2, [(1, 1, 1), (33, 70, 5), (0, 31, 32), (1, 1, 1), (3, 0, 2)]),
    ("bf16", "e4m3", 64, 8, 8, 3, [(40, 64, 1), (1, 1, 1), (7, 129, 33)]),
    ("f32", "int8", 16, 4, 4, 2, [(5, 90, 32), (1, 1, 1), (20, 100, 70), (2, 3, 4)]),
    ("f32", "e4m3", 64, 3, 1, 1, [(32, 96, 31), (1, 1, 1)]),
    ("f32", "int8", 64, 2, 2, 2, [(1, 66, 30), (2, 2, 2)]),
    ("bf16", "int8", 8, 8, 8, 4, [(10, 33, 65), (1, 1, 1), (22, 70, 90)]),
    ("bf16", "e4m3", 8, 6, 2, 2, [(1, 40, 100), (4, 5, 6)]),
    ("f32", "e4m3", 8, 8, 1, 2, [(70, 40, 10), (1, 1, 1)]),
    ("bf16", "int8", 16, 4, 4, 2, [(64, 32, 96), (32, 1, 33)]),
    ("bf16", "e4m3", 32, 8, 1, 2, [(35, 70, 5), (1, 40, 1)]),
    ("f32", "int8", 32, 16, 8, 1, [(1, 300, 200), (1, 1, 1)]),
]


def _attention_close(got, want, t, what):
    """out: one rounding to its type, weights in f16 where it is bf16 (each 2^-11 off, all one way at worst), and scores that are off by some
    roundings to float: 2^-21 of the largest score and of 1, which moves a weight by as much, twice (its own and the sum's).  lse likewise."""
    (out, lse), (ref, ref_lse, size, most) = got, want
    out, lse = out.double().cpu(), lse.double().cpu()
    ref, size = ref.flatten(2), size.flatten(2)
    score = 2.0 ** -21 * (most + 8).transpose(1, 2)[..., None].expand(-1, -1, -1, size.shape[2] // most.shape[1]).flatten(2)
    weight = 2.0 ** -11 if t is torch.bfloat16 else 2.0 ** -21
    room = torch.finfo(t).eps / 2 * 1.01 * ref.abs() + (weight + 2 * score) * size
    nan = torch.isnan(ref)
    assert torch.equal(torch.isnan(out), nan), what
    off = ((out - ref).abs() - room)[~nan]
    assert off.numel() == 0 or float(off.max()) <= 0, (what, float(off.max()))
    fine = torch.isfinite(ref_lse)
    assert torch.equal(torch.isneginf(lse), torch.isneginf(ref_lse)) and torch.equal(torch.isnan(lse), torch.isnan(ref_lse)), what
    off = ((lse - ref_lse).abs() - 2.0 ** -20 * (most + 8))[fine]
    assert off.numel() == 0 or float(off.max()) <= 0, (what, "lse", float(off.max()))


def _valid(gen, seg, B):
    v = torch.stack([torch.randint((n + 1) // 2, n + 1, (B,), generator=gen) for n in seg], dim=1)
    v[0] = torch.tensor(seg)
    return v.int().cuda()


@pytest.mark.parametrize("case", STREAMS, ids=lambda c: "-".join(str(x) for x in c[:6]))
def test_steps(g, case):
    """Plans, appended rows (all of them read back, bit by bit), and attention under one rule after the other."""
    dtype, held_as, hd, H, HK, B, steps = case
    t, gen = torch.bfloat16 if dtype == "bf16" else torch.float32, torch.Generator().manual_seed(hd * H + B)
    most = [sum(st[s] for st in steps) + 5 for s in range(3)]
    cache = g.stream_cache(B, most, HK, hd, t, held_as, pages=sum((m + 31) // 32 + 1 for m in most) * B + 3, times=True)
    ref = Streams(B, held_as)
    rules = [dict(phase=g.PHASE_INTER_FWD), dict(phase=g.PHASE_CUSTOM, custom_mask=0x1FF, softcap=5.0, causal=True), dict(phase=g.PHASE_INTRA, scale=0.3),
             dict(phase=g.PHASE_CUSTOM, custom_mask=0x0A1, slopes=True), dict(phase=g.PHASE_INTER_BWD, slopes=True, causal=True, softcap=20.0)]
    clock = 0.0
    for i, seg in enumerate(steps):
        valid = _valid(gen, seg, B)
        old = [[ref.length(b, s) for s in range(3)] for b in range(B)]
        qkv = _rows(gen, B, sum(seg), H + 2 * HK, hd, t)
        q, k, v = qkv[:, :, :H], qkv[:, :, H:H + HK], qkv[:, :, H + HK:]
        times = (clock + 3 * torch.rand((sum(seg), B), generator=gen)).cuda().t()   # rows of a column-major matrix
        clock += 2.0
        slots = g.cache_plan(cache, seg, valid)
        g.cache_append(cache, k, v, slots, seg, times)
        ref.step(seg, valid.cpu(), k, v, times)
        _check_plan(g, cache, slots, seg, valid.cpu(), old, ref)
        whole = tuple(m + 40 for m in most)
        got = g.cache_read(cache, whole)
        first = np.concatenate([[0], np.cumsum(whole)])
        for name, x in zip("kv", got):
            want = torch.zeros((B, sum(whole), HK, hd), dtype=t)
            for b in range(B):
                for s in range(3):
                    if ref.length(b, s):
                        want[b, first[s]:first[s] + ref.length(b, s)] = ref.held(b, s, name, exactly=False)
            assert torch.equal(x.cpu(), want), (name, i)
        for rule in rules:
            rule = dict(rule)
            if rule.pop("slopes", False):
                rule["slopes"] = torch.rand(H, generator=gen).cuda()
            got = g.im_cached_attention_fwd(q, cache, seg, valid, times=times, want_lse=True, **rule)
            pairs = open_blocks(rule.pop("phase"), rule.pop("custom_mask", 0))
            want = ref.attention(q, seg, valid.cpu(), pairs, rule.pop("scale", hd ** -0.5), times=times, **rule)
            _attention_close(got, want, t, (i, rule))
    assert g.last_device_status() == (0, 0)


def test_ended_streams_and_a_full_pool(g):
    """Pages go back and come out again in order; what finds none is left out whole, and says so."""
    B, seg = 3, (40, 40, 40)
    cache = g.stream_tables(B, 4, 14)
    full = torch.tensor([seg] * B, dtype=torch.int32, device="cuda")
    slots = g.cache_plan(cache, seg, full)            # 18 blocks wanted, 14 there: the first seven segments
    assert g.last_device_status()[1] == g.DEVFLAG_FULL
    lengths = cache.lengths.cpu().flatten()
    assert lengths.tolist() == [40] * 7 + [0] * 2 and int(cache.n_free) == 0
    assert cache.tables.cpu().flatten(0, 1)[:7, :2].flatten().tolist() == list(range(14))
    assert (slots.cpu().reshape(9, 40)[7:] == -1).all() and (slots.cpu().reshape(9, 40)[:7] >= 0).all()
    # rows that fit the open blocks are taken although the list is empty; a table's end is an end
    slots = g.cache_plan(cache, (24, 0, 89), torch.tensor([[24, 0, 88], [24, 0, 0], [24, 0, 1]], dtype=torch.int32, device="cuda"))
    assert cache.lengths.cpu().tolist() == [[64, 40, 40], [64, 40, 40], [64, 0, 0]] and g.last_device_status()[1] == g.DEVFLAG_FULL
    # stream 1 ends and begins anew: its six pages come back in order
    ended = torch.tensor([0, 1, 0], dtype=torch.int32, device="cuda")
    before = cache.tables.clone()
    slots = g.cache_plan(cache, (1, 33, 64), torch.tensor([[0, 0, 0], [1, 33, 64], [0, 0, 0]], dtype=torch.int32, device="cuda"), ended=ended)
    assert g.last_device_status() == (0, 0) and cache.lengths.cpu().tolist() == [[64, 40, 40], [1, 33, 64], [64, 0, 0]]
    old = before[1].cpu()
    pages = [p for p in old.flatten().tolist() if p >= 0]
    assert [p for p in cache.tables[1].cpu().flatten().tolist() if p >= 0] == pages[:5] and int(cache.n_free) == 1
    assert torch.equal(cache.tables[0], before[0]) and torch.equal(cache.tables[2], before[2])
    # everything ends: the pool is whole again
    g.cache_plan(cache, (1, 0, 0), torch.zeros((3, 3), dtype=torch.int32, device="cuda"), ended=torch.ones(3, dtype=torch.int32, device="cuda"))
    assert int(cache.n_free) == 14 and sorted(cache.free.cpu().tolist()) == list(range(14)) and not cache.lengths.any() and (cache.tables == -1).all()


@pytest.mark.parametrize("B", [1, 70, 1000])
def test_plans_of_many_streams(g, B):
    """Against a plan made entry by entry: one CTA and several, long rows of a table, streams that end."""
    rng, blocks = np.random.default_rng(B), 45
    cache = g.stream_tables(B, blocks, 3 * B * 30)
    tables, free, held = np.full((3 * B, blocks), -1), list(range(3 * B * 30 - 1, -1, -1)), np.zeros(3 * B, dtype=int)
    for step in range(4):
        seg = (1, 1, 1) if step == 2 else (70, 400, 33)
        valid = np.stack([rng.integers(0, n + 1, size=B) for n in seg], axis=1)
        ended = (rng.random(B) < 0.3).astype(np.int32) if step else np.zeros(B, dtype=np.int32)
        slots = g.cache_plan(cache, seg, torch.from_numpy(valid.astype(np.int32)).cuda(), ended=torch.from_numpy(ended).cuda()).cpu().numpy()
        back = []
        for e in range(3 * B):
            if ended[e // 3]:
                back += [p for p in tables[e] if p >= 0]
                tables[e], held[e] = -1, 0
        free += back[::-1]
        avail, run, used = len(free), 0, 0
        for e in range(3 * B):
            n = int(valid[e // 3, e % 3])
            to = (held[e] + n + 31) // 32
            if n == 0 or to > blocks:
                continue
            need = [j for j in range(held[e] // 32, to) if tables[e, j] < 0]
            run += len(need)
            if need and run > avail:
                continue
            for i, j in enumerate(need):
                tables[e, j] = free[avail - 1 - (run - len(need) + i)]
            used = run if need else used
            at = np.arange(held[e], held[e] + n)
            row = sum(seg[:e % 3])
            assert (slots[e // 3, row:row + n] == tables[e, at // 32] * 32 + at % 32).all()
            held[e] += n
        free = free[:avail - used]
        assert (cache.tables.cpu().numpy().reshape(3 * B, -1) == tables).all() and (cache.lengths.cpu().numpy().flatten() == held).all()
        assert cache.free[:int(cache.n_free)].cpu().tolist() == free
    g.last_device_status()


def test_a_step_taken_again(g):
    """A guess that is taken back: plan from the lengths before it, other rows, the same cache as if the guess had never been."""
    B, HK, hd, gen = 2, 2, 32, torch.Generator().manual_seed(1)
    caches = [g.stream_cache(B, (100, 100, 100), HK, hd) for _ in range(2)]
    start = _rows(gen, B, 90, HK, hd, torch.bfloat16), _rows(gen, B, 90, HK, hd, torch.bfloat16)
    guess, real = [(_rows(gen, B, 60, HK, hd, torch.bfloat16), _rows(gen, B, 60, HK, hd, torch.bfloat16)) for _ in range(2)]
    for cache, steps in zip(caches, ([guess, real], [real])):
        g.cache_append(cache, *start, g.cache_plan(cache, (20, 30, 40)), (20, 30, 40))
        held = cache.lengths.clone()
        for k, v in steps:
            g.cache_append(cache, k, v, g.cache_plan(cache, (32, 8, 20), held=held), (32, 8, 20))
    a, b = (g.cache_read(c, (100, 100, 100)) for c in caches)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and torch.equal(caches[0].lengths, caches[1].lengths) and int(caches[0].n_free) == int(caches[1].n_free)


@pytest.mark.parametrize("held_as", ["int8", "e4m3"])
@pytest.mark.parametrize("t", [torch.bfloat16, torch.float32])
def test_values_at_the_edges(g, held_as, t):
    """Blocks of zeros, of one value, of values that lie between two of the 8-bit ones, of almost nothing and of almost everything."""
    most, hd = (127.0 if held_as == "int8" else 448.0), 16
    gen = torch.Generator().manual_seed(3)
    big = float(torch.finfo(t).max)
    ramp = torch.arange(BLOCK * hd).float().reshape(BLOCK, hd) / 4
    ties = torch.where(torch.arange(BLOCK * hd).reshape(BLOCK, hd) == 0, torch.tensor(most), (ramp % most))       # quarters under a scale of 1
    kinds = [torch.zeros(BLOCK, hd), torch.full((BLOCK, hd), -3.7), ties, -ties, ties * 2.0 ** -60, torch.full((BLOCK, hd), 2.0 ** -120), torch.full((BLOCK, hd), big),
             torch.randn((BLOCK, hd), generator=gen) * 1e30, torch.randn((BLOCK, hd), generator=gen) * 2.0 ** -40, ties * 3.0]
    x = torch.stack(kinds, dim=1)[None].to(t).cuda()      # [1, 32, heads, hd]
    cache, ref = g.stream_cache(1, (32, 0, 0), len(kinds), hd, t, held_as), Streams(1, held_as)
    g.cache_append(cache, x, -x, g.cache_plan(cache, (32, 0, 0)), (32, 0, 0))
    ref.step((32, 0, 0), [[32, 0, 0]], x, -x)
    for name, got in zip("kv", g.cache_read(cache, (32, 0, 0))):
        assert torch.equal(got[0].cpu(), ref.held(0, 0, name, exactly=False)), name


def test_nan_and_inf(g):
    """A block and head with NaN or Inf reads as NaN: rows that see it, and no others; what stands behind the last position held reaches nothing."""
    B, H, hd, t, gen = 1, 2, 64, torch.bfloat16, torch.Generator().manual_seed(4)
    seg = (40, 70, 33)
    k, v, q = (_rows(gen, B, sum(seg), H, hd, t) for _ in range(3))
    k[0, 40 + 5, 0, 3] = float("inf")       # segment 1, first block, keys of head 0
    v[0, 110 + 32, 1, 0] = float("nan")     # segment 2, open block, values of head 1
    v[0, 35, 0, 1] = float("nan")           # segment 0, open block, head 0
    cache, ref = g.stream_cache(B, seg, H, hd, t, times=True), Streams(B, "int8")
    cache.open_keys.fill_(float("nan"))
    cache.open_values.fill_(float("nan"))
    times = torch.arange(sum(seg), device="cuda").float()[None] - torch.tensor([0.0] * 40 + [40.0] * 70 + [110.0] * 33, device="cuda")
    g.cache_append(cache, k, v, g.cache_plan(cache, seg), seg, times)
    ref.step(seg, [seg], k, v, times)
    for rule in (dict(phase=g.PHASE_INTRA), dict(phase=g.PHASE_INTER_FWD), dict(phase=g.PHASE_CUSTOM, custom_mask=0x1FF, causal=True), dict(phase=g.PHASE_INTER_BWD, causal=True)):
        got = g.im_cached_attention_fwd(q, cache, seg, times=times, want_lse=True, **rule)
        want = ref.attention(q, seg, [seg], open_blocks(rule.pop("phase"), rule.pop("custom_mask", 0)), hd ** -0.5, times=times, **rule)
        _attention_close(got, want, t, rule)
    # a query with NaN, and one with Inf: their own rows
    clean = g.stream_cache(B, seg, H, hd, t)
    k, v = (torch.nan_to_num(x, 0.0, 0.0, 0.0) for x in (k, v))
    g.cache_append(clean, k, v, g.cache_plan(clean, seg), seg)
    want = g.im_cached_attention_fwd(q, clean, seg, phase=g.PHASE_INTRA)
    dirty = q.clone()
    dirty[0, 3, 0, 7], dirty[0, 50, 1, 7] = float("nan"), float("inf")
    got = g.im_cached_attention_fwd(dirty, clean, seg, phase=g.PHASE_INTRA)
    bad = torch.zeros_like(want, dtype=torch.bool)
    bad[0, 3, :64], bad[0, 50, 64:] = True, True
    assert torch.equal(torch.isnan(got), bad) and torch.equal(got[~bad], want[~bad])


def test_no_rows_no_keys(g):
    """Streams that hold nothing, segments that no key is open to, steps in which a stream has no rows."""
    B, H, hd = 3, 4, 16
    cache = g.stream_cache(B, (64, 64, 64), H, hd)
    q = torch.randn((B, 3, H, hd), device="cuda").bfloat16()
    valid = torch.zeros((B, 3), dtype=torch.int32, device="cuda")
    valid[1] = 1
    slots = g.cache_plan(cache, (1, 1, 1), valid)
    assert (slots[0] == -1).all() and (slots[1] >= 0).all()
    g.cache_append(cache, q, q, slots, (1, 1, 1))
    out, lse = g.im_cached_attention_fwd(q, cache, (1, 1, 1), valid, phase=g.PHASE_INTRA, want_lse=True)
    assert torch.equal(out[1], q[1].flatten(1)) and not out[0].any() and not out[2].any() and torch.isneginf(lse[0]).all() and torch.isfinite(lse[1]).all()
    out, lse = g.im_cached_attention_fwd(q, cache, (1, 1, 1), valid, phase=g.PHASE_CUSTOM, custom_mask=0, want_lse=True)
    assert not out.any() and torch.isneginf(lse).all()
    k, v = g.cache_read(cache, (1, 0, 2))
    assert k.shape == (B, 3, H, hd) and torch.equal(k[1, 0], q[1, 0]) and torch.equal(v[1, 1], q[1, 2]) and not k[0].any() and not k[1, 2].any()


def test_streams_graphs_and_bits(g):
    """A step captured once and replayed while the streams grow, against the same steps called one by one; on a stream of its own, behind late writes."""
    B, H, HK, hd, seg, gen = 3, 4, 2, 64, (1, 2, 3), torch.Generator().manual_seed(6)
    caches = [g.stream_cache(B, (40, 80, 120), HK, hd) for _ in range(2)]
    rows = [_rows(gen, B, 6, H + 2 * HK, hd, torch.bfloat16) for _ in range(36)]
    valid = torch.tensor([[1, 2, 3], [0, 1, 3], [1, 0, 2]], dtype=torch.int32, device="cuda")
    x = torch.zeros_like(rows[0])
    slots, out = torch.empty((B, 6), dtype=torch.int32, device="cuda"), torch.empty((B, 6, H * hd), device="cuda", dtype=torch.bfloat16)

    def step(cache, x):
        g.cache_plan(cache, seg, valid, slots=slots)
        g.cache_append(cache, x[:, :, H:H + HK], x[:, :, H + HK:], slots, seg)
        return g.im_cached_attention_fwd(x[:, :, :H], cache, seg, valid, phase=g.PHASE_CUSTOM, custom_mask=0x1FF, out=out)

    side = torch.cuda.Stream()
    want = []
    with torch.cuda.stream(side):
        for r in rows:
            x.zero_()
            g.late_write(x, r)
            want.append(step(caches[0], x).clone())
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    keep = [t.clone() for t in caches[1] if t is not None]
    with torch.cuda.graph(graph):
        step(caches[1], x)
    for t, k in zip([t for t in caches[1] if t is not None], keep):
        assert torch.equal(t, k)   # capturing runs nothing
    for r, w in zip(rows, want):
        x.copy_(r)
        graph.replay()
        assert torch.equal(out, w)
    for a, b in zip(g.cache_read(caches[0], (40, 80, 120)), g.cache_read(caches[1], (40, 80, 120))):
        assert torch.equal(a, b)
    again = [g.im_cached_attention_fwd(x[:, :, :H], caches[1], seg, valid) for _ in range(4)]
    assert all(torch.equal(a, again[0]) for a in again)


@pytest.mark.parametrize("case", [(1, (40, 3000, 900), 8, 8, 64, "int8", torch.bfloat16), (2, (600, 1500, 2500), 8, 1, 64, "e4m3", torch.bfloat16),
                                  (1, (100, 5000, 60), 4, 4, 8, "int8", torch.float32), (1, (33, 6000, 64), 16, 2, 32, "int8", torch.float32),
                                  (40, (64, 200, 300), 4, 4, 16, "e4m3", torch.bfloat16)])
def test_long_pasts(g, case):
    """Keys split over many CTAs, against attention over the bytes as they lie in the pages."""
    B, n, H, HK, hd, held_as, t = case
    gen = torch.Generator(device="cuda").manual_seed(hd)
    cache = g.stream_cache(B, [m + 1 for m in n], HK, hd, t, held_as)
    k, v = (torch.randn((B, sum(n), HK, hd), device="cuda", generator=gen).to(t) for _ in range(2))
    g.cache_append(cache, k, v, g.cache_plan(cache, n), n)
    q = 2 * torch.randn((B, 3, H, hd), device="cuda", generator=gen)
    q, nk, nv = q.to(t), q[:, :, :HK].to(t), -q[:, :, H - HK:].to(t)
    g.cache_append(cache, nk, nv, g.cache_plan(cache, (1, 1, 1)), (1, 1, 1))
    got = g.im_cached_attention_fwd(q, cache, (1, 1, 1), phase=g.PHASE_CUSTOM, custom_mask=0x1FF, want_lse=True)
    ref, lse, size, most = [], [], [], []
    for b in range(B):
        K, V = (torch.cat([bytes_of(cache, b, s, name) for s in range(3)]).repeat_interleave(H // HK, dim=1) for name in "kv")
        assert K.shape[0] == sum(n) + 3
        x = torch.einsum("ihc,jhc->hij", q[b].double(), K) * hd ** -0.5
        p = torch.softmax(x, dim=2)
        ref.append(torch.einsum("hij,jhc->ihc", p, V))
        size.append(torch.einsum("hij,jhc->ihc", p, V.abs()).amax(dim=2, keepdim=True).expand_as(ref[-1]))
        lse.append(torch.logsumexp(x, dim=2))
        most.append(x.abs().amax(dim=2))
    _attention_close(got, [torch.stack(x).cpu() for x in (ref, lse, size, most)], t, case)
