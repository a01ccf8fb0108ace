"""Attention over a cache whose blocks are shared out evenly to all CTAs, which long tables ask for: ragged and empty streams, fewer blocks than CTAs,
streams in several rounds of the scan, workspaces."""
import ctypes

import pytest
import torch

from stream_reference import bytes_of
from test_gpu_stream import _attention_close, g, nothing_is_flagged   # noqa: F401

pytestmark = pytest.mark.gpu

# streams, longest lengths, table's positions, heads, key heads, width, held as, type
CASES = [(1, (3, 40, 0), 9000, 8, 8, 64, "int8", torch.bfloat16),            # a handful of blocks for all CTAs
         (1, (9000, 50, 8000), 9000, 8, 8, 64, "e4m3", torch.bfloat16),
         (3, (700, 2000, 90), 30000, 4, 1, 64, "int8", torch.float32),
         (7, (100, 3000, 33), 80000, 12, 4, 32, "e4m3", torch.bfloat16),
         (2, (64, 32, 31), 40000, 6, 2, 16, "int8", torch.bfloat16),
         (2, (500, 1000, 1), 200000, 2, 2, 8, "e4m3", torch.float32),
         (300, (40, 70, 100), 2000, 4, 2, 64, "int8", torch.bfloat16),
         (520, (33, 0, 64), 2000, 2, 2, 32, "e4m3", torch.float32)]


def _filled(g, case, seed=0):
    B, most, table, H, HK, hd, held_as, t = case
    gen = torch.Generator().manual_seed(seed + hd)
    n = torch.stack([torch.randint(0, m + 1, (B,), generator=gen) for m in most], dim=1).int()
    n[0] = torch.tensor(most)
    if B > 2:
        n[B // 2] = 0   # a stream that holds nothing
    blocks = (torch.tensor(most).sum() + 3) // 32 + 6
    cache = g.stream_cache(B, (table, table, table), HK, hd, t, held_as, pages=int(blocks) * B)
    dev = torch.Generator(device="cuda").manual_seed(seed)
    k, v = (torch.randn((B, sum(most), HK, hd), device="cuda", generator=dev).to(t) for _ in range(2))
    g.cache_append(cache, k, v, g.cache_plan(cache, most, n.cuda()), most)
    valid = torch.randint(0, 2, (B, 3), generator=gen).int()
    valid[0] = 1
    q = (2 * torch.randn((B, 3, H, hd), device="cuda", generator=dev)).to(t)
    new = (torch.randn((B, 3, HK, hd), device="cuda", generator=dev).to(t) for _ in range(2))
    g.cache_append(cache, *new, g.cache_plan(cache, (1, 1, 1), valid.cuda()), (1, 1, 1))
    return cache, q, valid


def _workspace(g, cache, q, **kw):
    """What the call asks for; more than 0: the blocks are shared out."""
    fn = g.load().gsit_cached_attention_workspace
    fn.restype = ctypes.c_size_t
    from test_ops_refusals import Rule
    from test_stream_refusals import Cache
    B, _, H, hd = q.shape
    c = Cache(1 if cache.keys.dtype is torch.float8_e4m3fn else 0, g.DTYPE_BF16 if q.dtype is torch.bfloat16 else g.DTYPE_F32, B, cache.open_keys.shape[3], hd, cache.free.numel(),
              cache.tables.shape[2], *[t.data_ptr() for t in (cache.keys, cache.values, cache.key_scale, cache.value_scale)], None,
              *[t.data_ptr() for t in (cache.open_keys, cache.open_values, cache.tables, cache.lengths, cache.free, cache.n_free)])
    shape = g.make_shape(B, (1, 1, 1), H * hd, H, None, c.dtype, g.PHASE_CUSTOM, 0x1FF)
    return fn(ctypes.byref(shape), ctypes.byref(Rule(0.0, 0, 0, None, None, None, None, 0, (ctypes.c_int32 * 3)())), ctypes.byref(c))


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(x) for x in c).replace(" ", ""))
@pytest.mark.parametrize("mask", [0x1FF, 0x062])   # all blocks; the forward ring
def test_shares(g, case, mask):
    B, most, table, H, HK, hd, held_as, t = case
    cache, q, valid = _filled(g, case)
    assert _workspace(g, cache, q) > 0
    got = g.im_cached_attention_fwd(q, cache, (1, 1, 1), valid.cuda(), phase=g.PHASE_CUSTOM, custom_mask=mask, want_lse=True)
    again = g.im_cached_attention_fwd(q, cache, (1, 1, 1), valid.cuda(), phase=g.PHASE_CUSTOM, custom_mask=mask, want_lse=True)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])
    ref, size = (torch.zeros((B, 3, H, hd), dtype=torch.float64) for _ in range(2))
    lse, scores = torch.full((B, H, 3), float("-inf"), dtype=torch.float64), torch.zeros((B, H, 3), dtype=torch.float64)
    for b in range(B):
        rows = {n: [bytes_of(cache, b, s, n) for s in range(3)] for n in "kv"} if valid[b].any() else None
        for s in range(3):
            over = [r for r in range(3) if mask >> (3 * s + r) & 1]
            if not valid[b, s] or sum(rows["k"][r].shape[0] for r in over) == 0:
                continue
            K, V = (torch.cat([rows[n][r] for r in over]).repeat_interleave(H // HK, dim=1) for n in "kv")
            x = torch.einsum("hc,jhc->hj", q[b, s].double(), K) * hd ** -0.5
            p = torch.softmax(x, dim=1)
            ref[b, s], size[b, s] = torch.einsum("hj,jhc->hc", p, V).cpu(), torch.einsum("hj,jhc->hc", p, V.abs()).amax(dim=1, keepdim=True).expand(H, hd).cpu()
            lse[b, :, s], scores[b, :, s] = torch.logsumexp(x, dim=1).cpu(), x.abs().amax(dim=1).cpu()
    _attention_close(got, (ref, lse, size, scores), t, case)


def test_workspaces(g):
    """Host memory, gaps and too little are refused; what stands in it does not matter; two captured graphs may share one, one after the other."""
    case = CASES[3]
    cache, q, valid = _filled(g, case)
    call = lambda **kw: g.im_cached_attention_fwd(q, cache, (1, 1, 1), valid.cuda(), phase=g.PHASE_CUSTOM, custom_mask=0x1FF, **kw)
    want, need = call(), _workspace(g, cache, q)
    for bad in (torch.empty(need, dtype=torch.uint8), torch.empty(2 * need, dtype=torch.uint8, device="cuda")[::2]):
        with pytest.raises(AssertionError):
            call(workspace=bad)
    for bad in (torch.empty(need - 1, dtype=torch.uint8, device="cuda"), torch.empty(need + 16, dtype=torch.uint8, device="cuda")[4:]):
        with pytest.raises(g.GsitError):
            call(workspace=bad)
    space = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    assert torch.equal(call(workspace=space), want)
    on_device = valid.cuda()
    graphs, outs = [], []
    for mask in (0x1FF, 0x062):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(g.im_cached_attention_fwd(q, cache, (1, 1, 1), on_device, phase=g.PHASE_CUSTOM, custom_mask=mask, workspace=space))
        graphs.append(graph)
    for _ in range(3):
        for graph in graphs:
            graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want) and torch.equal(outs[1], g.im_cached_attention_fwd(q, cache, (1, 1, 1), on_device, phase=g.PHASE_CUSTOM, custom_mask=0x062))
