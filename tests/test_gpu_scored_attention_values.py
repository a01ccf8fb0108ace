"""Scored attention where single values decide."""
import math

import pytest
import torch

from test_gpu_scored_attention import TOL, Problem, _check, _close

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def g():
    import paper_2505_01068_b200 as lib
    lib.load()
    return lib


# ---- moments of -0.0 and +0.0 are one moment ----

def _ages(p, seg):
    """Segment 0 timed by its age, so that its newest position has -0.0; the others start at +0.0."""
    t = torch.cat([-1.0 * torch.arange(seg[0] - 1, -1, -1, dtype=torch.float32), torch.arange(seg[1]).float() * 0.25, torch.arange(seg[2]).float() * 0.5])
    p.times = t.cuda().expand(p.B, -1).contiguous()
    assert float(p.times[0, seg[0] - 1]) == 0.0 and bool(torch.signbit(p.times[0, seg[0] - 1]))


@pytest.mark.parametrize("dtype,hd,seg", [("bf16", 8, (20, 90, 45)), ("bf16", 16, (20, 90, 45)), ("bf16", 32, (70, 64, 300)), ("bf16", 64, (70, 41, 60)),
                                          ("bf16", 64, (130, 300, 257)), ("f32", 16, (20, 90, 45)), ("f32", 64, (70, 200, 3)), ("f32", 96, (20, 90, 45))])
@pytest.mark.parametrize("rule", [dict(), dict(cap=20.0, slopes=True), dict(docs=-1)], ids=str)
def test_moments_of_either_zero_are_equal(g, dtype, hd, seg, rule):
    """The newest position of segment 0 sees the first key of segment 1 and nothing else: its result is that key's value."""
    p = Problem(dtype, 2, seg, 2, 1, hd, "fwd", padded=False, causal=True, **rule)
    _ages(p, seg)
    out, lse = _check(g, p)
    row = out[:, seg[0] - 1].view(2, 2, hd)
    assert torch.equal(row, p.v[:, seg[0]].expand(2, 2, hd)) and bool(torch.isfinite(lse[:, :, seg[0] - 1]).all())


@pytest.mark.parametrize("dtype,hd,seg", [("bf16", 16, (20, 900, 45)), ("bf16", 64, (130, 300, 257)), ("f32", 16, (20, 90, 45)), ("f32", 24, (20, 90, 45))])
def test_moments_of_either_zero_are_equal_to_the_newest_position(g, dtype, hd, seg):
    p = Problem(dtype, 2, seg, 2, 1, hd, "fwd", padded=False, causal=True, q_len=(1, 1, 1))
    _ages(p, seg)
    out, _ = _check(g, p, grads=False)
    assert torch.equal(out[:, 0].view(2, 2, hd), p.v[:, seg[0]].expand(2, 2, hd))


# ---- NaN in a stream's rows ----

STREAMS = [("bf16", 8, 4, 2, (1, 1, 1)), ("bf16", 16, 2, 2, (1, 1, 1)), ("bf16", 32, 4, 1, (1, 0, 1)), ("bf16", 64, 4, 2, (2, 1, 1)), ("f32", 8, 1, 1, (1, 0, 0)),
           ("f32", 16, 2, 2, (1, 1, 1)), ("f32", 32, 4, 2, (1, 1, 1)), ("f32", 64, 2, 2, (1, 1, 1)), ("f32", 24, 2, 1, (1, 1, 1))]
SEG = (100, 500, 300)


@pytest.mark.parametrize("rule", [dict(), dict(cap=20.0), dict(slopes=True, docs=-3, causal=True)], ids=str)
@pytest.mark.parametrize("stream", STREAMS, ids=str)
def test_nan_reaches_the_newest_rows_that_it_is_open_to(g, stream, rule):
    """NaN in a query, in an open key, in an open value: NaN in what depends on it, other rows to rounding."""
    dtype, hd, H, HK, q_len = stream
    make = lambda: Problem(dtype, 2, SEG, H, HK, hd, "intra", padded=False, q_len=q_len, **rule)
    base, blse = make().forward(g)
    base = base.view(2, sum(q_len), H, hd)
    last = q_len[0] - 1                      # the newest row of segment 0, position 99
    for what in ("q", "k", "v"):
        p = make()
        if what == "q":
            p.q[0, last, 0, 1] = float("nan")
            hit = [0]
        else:
            getattr(p, what)[0, 99, 0, 1] = float("nan")
            hit = list(range(H // HK))
        out, lse = p.forward(g)
        out = out.view(2, sum(q_len), H, hd)
        broken = torch.zeros_like(out, dtype=torch.bool)
        rows = [last] if what == "q" or rule.get("causal") else list(range(last + 1))   # without causality every query of segment 0 sees key 99
        for i in rows:
            broken[0, i, hit] = True
        if what == "v":
            broken[..., :1] = broken[..., 2:] = False
        assert bool(out[broken].isnan().all()), what
        _close(torch.where(broken, 0.0, out.float()), torch.where(broken, 0.0, base.double()), TOL[dtype]["out"], what)
        lse_broken = torch.zeros_like(lse, dtype=torch.bool)
        if what != "v":
            for i in rows:
                lse_broken[0, hit, i] = True
        assert bool(lse[lse_broken].isnan().all()) and torch.allclose(lse[~lse_broken], blse[~lse_broken], atol=2e-5, rtol=2e-5), what
    assert g.last_device_status() == (0, 0)


@pytest.mark.parametrize("fill", [float("nan"), float("inf"), -3.38e38])
@pytest.mark.parametrize("stream", STREAMS, ids=str)
def test_what_stands_in_closed_keys_does_not_reach_the_newest_rows(g, stream, fill):
    """Keys of another document, and keys past the valid ones."""
    dtype, hd, H, HK, q_len = stream
    p = Problem(dtype, 2, SEG, H, HK, hd, "all", q_len=q_len, docs=-3, causal=True, seed=4)
    base = p.forward(g)
    for t in (p.k, p.v):
        t[p.padding()] = fill
    got = p.forward(g)
    assert torch.equal(got[0], base[0]) and torch.equal(got[1], base[1])
    shut = p.docs == 1
    assert bool((shut & ~p.padding()).any())
    keep = torch.zeros(2, sum(q_len), dtype=torch.bool, device="cuda")   # rows whose own document is another
    first = (0, SEG[0], SEG[0] + SEG[1])
    for b in range(2):
        i = 0
        for s in range(3):
            for r in range(q_len[s]):
                at = int(p.n[b, s]) - q_len[s] + r
                keep[b, i] = at >= 0 and int(p.docs[b, first[s] + at]) != 1
                i += 1
    assert bool(keep.any())
    for t in (p.k, p.v):
        t[shut] = fill
    out, lse = p.forward(g)
    _close(out[keep], base[0][keep].double(), TOL[dtype]["out"], "out")
    assert torch.allclose(lse.transpose(1, 2)[keep], base[1].transpose(1, 2)[keep], atol=2e-5, rtol=2e-5)


# ---- rows beside a tile's real ones ----

@pytest.mark.parametrize("seg", [(130, 300, 257), (100, 200, 192)], ids=str)
@pytest.mark.parametrize("phase", ["intra", "all"])
def test_other_rows_of_a_tile_leave_a_rows_bits(g, seg, phase):
    """head_dim 64, scores without a cap: padded queries, and the queries of the next segment and of the next sample, which a tile's load
    brings along, may hold large values that outgrow their references late; the bits of the other rows stay."""
    p = Problem("bf16", 3, seg, 2, 2, 64, phase, seed=11)
    pad, L = p.padding(), sum(seg)
    large = (torch.randn(p.q.shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3)) * 100).bfloat16()
    q = p.q.clone()
    p.q = torch.where(pad[:, :, None, None], 0.0, q)
    out, lse = p.forward(g)
    p.q = torch.where(pad[:, :, None, None], large, q)
    got = p.forward(g)
    assert torch.equal(got[0], out) and torch.equal(got[1], lse)
    p.q = q.clone()
    p.q[:, seg[0]:] = large[:, seg[0]:]
    got = p.forward(g)
    assert torch.equal(got[0][:, :seg[0]], out[:, :seg[0]]) and torch.equal(got[1][:, :, :seg[0]], lse[:, :, :seg[0]])
    p.q = q.clone()
    p.q[1:] = large[1:]
    got = p.forward(g)
    assert torch.equal(got[0][0], out[0]) and torch.equal(got[1][0], lse[0])
    assert g.last_device_status() == (0, 0)


# ---- single precision of a capped score ----

@pytest.mark.parametrize("hd,tail", [(8, False), (16, False), (64, False), (96, False), (8, True), (64, True)])
@pytest.mark.parametrize("cap", [1.0, 50.0])
def test_a_capped_float_score_has_floats_accuracy(g, hd, tail, cap):
    """One key to a query: the log-sum-exp is the score, cap tanh(s / cap), for arguments s / cap from 1/100 to 4.  Between the exact dot and
    it there are six roundings (of 1 / cap, of the cap and of the two constants of base 2, and their products) and the tanh; the same in
    32-bit torch operations has four and the tanh: the root mean square of the relative error may be sqrt(6 / 4) of theirs, 1.5 with some room."""
    n = 4096
    s = torch.logspace(-2, math.log10(4.0), n, device="cuda") * cap
    q = torch.zeros((n, 1, 1, hd), device="cuda")
    q[:, 0, 0, 0] = s
    k = torch.zeros((n, 1, 1, hd), device="cuda")
    k[:, 0, 0, 0] = 1.0
    more = dict(q_len=(1, 0, 0)) if tail else {}
    _, lse = g.im_scored_attention_fwd(q, k, k, (1, 0, 0), None, g.PHASE_INTRA, scale=1.0, softcap=cap, want_lse=True, **more)
    want = cap * torch.tanh(s.double() / cap)
    plain = cap * torch.tanh(s / cap)
    rms = lambda x: float(((x.double() - want) / want).square().mean().sqrt())
    assert rms(lse.flatten()) <= 1.5 * rms(plain), (rms(lse.flatten()), rms(plain))
