"""Scored attention where single values decide."""
import math

import pytest
import torch

from test_gpu_scored_attention import Problem, _check

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
