"""Scored attention at head_dim 64 on both sides of the line between the tcgen05 kernels and the mma.sync tiles: long walks over well
filled tiles take the former, short or ragged ones the latter.  Every rule and block pattern on either side, against 64 bits."""
import math

import pytest
import torch

from test_gpu_scored_attention import RULES, TOL, Problem, _check, _close

pytestmark = pytest.mark.gpu
LONG, SHORT = (130, 300, 257), (70, 41, 60)


@pytest.fixture(scope="module")
def g():
    import paper_2505_01068_b200 as lib
    lib.load()
    return lib


@pytest.mark.parametrize("seg", [LONG, SHORT], ids=str)
@pytest.mark.parametrize("rule", RULES, ids=str)
@pytest.mark.parametrize("phase", ["fwd", "intra", "all"])
def test_rules(g, seg, rule, phase):
    i = RULES.index(rule)
    _check(g, Problem("bf16", 2, seg, 4, (4, 2, 1)[i % 3], 64, phase, seed=i, **rule))


@pytest.mark.parametrize("seg", [LONG, SHORT, (128, 256, 64), (1, 700, 129), (0, 400, 400), (513, 0, 0)], ids=str)
@pytest.mark.parametrize("phase", ["fwd", "bwd", "intra", "all", "first", "none"])
def test_block_patterns(g, seg, phase):
    _check(g, Problem("bf16", 3, seg, 2, 2, 64, phase, cap=30.0))


@pytest.mark.parametrize("amplitude", [0.01, 4.0, 9.0])
@pytest.mark.parametrize("cap", [0.0, 2.0, 60.0])
def test_small_and_large_scores(g, amplitude, cap):
    """The gradient's terms are as large as its inputs, so only the forward pass is held to the relative bound where they are not of order one."""
    _check(g, Problem("bf16", 2, LONG, 2, 2, 64, "all", cap=cap, amplitude=amplitude), grads=False)


@pytest.mark.parametrize("seg", [(60, 250, 190), SHORT], ids=str)
@pytest.mark.parametrize("fill", [float("nan"), float("inf"), -3.38e38])
def test_what_stands_in_padding_and_in_closed_documents_never_matters(g, seg, fill):
    p = Problem("bf16", 2, seg, 2, 1, 64, "all", docs=-3, causal=True, seed=5, cap=20.0)
    base = p.forward(g)
    clean = p.backward(g, *base)
    pad, other = p.padding(), p.docs == 1
    for t in (p.q, p.k, p.v, p.dout):
        t[pad] = fill
    out, lse = p.forward(g)
    assert torch.equal(out, base[0]) and torch.equal(lse, base[1])
    assert all(torch.equal(x, y) for x, y in zip(p.backward(g, out, lse), clean))
    for t in (p.q, p.k, p.v, p.dout):
        t[other & ~pad] = fill
    out, lse = p.forward(g)
    keep = ~other
    _close(out[keep], base[0][keep].double(), TOL["bf16"]["out"], "out")
    for x, y in zip(p.backward(g, out, lse), clean):
        _close(x[keep], y[keep].double(), TOL["bf16"]["grad"], "grad")
    assert g.last_device_status() == (0, 0)


def test_warps_of_uneven_speed(g):
    """Large values in one document send some warps of a tile through the form of the cap for any argument, others not: whoever is ahead
    must not take a result before it is whole."""
    p = Problem("bf16", 2, (60, 250, 190), 2, 1, 64, "all", docs=-3, causal=True, seed=5, cap=20.0)
    base = p.forward(g)
    clean = p.backward(g, *base)
    other = p.docs == 1
    for t in (p.q, p.k, p.v, p.dout):
        t[other] = 1e15
    keep = ~other & ~p.padding()
    for _ in range(40):
        out, lse = p.forward(g)
        _close(out[keep], base[0][keep].double(), TOL["bf16"]["out"], "out")
        for x, y in zip(p.backward(g, out, lse), clean):
            _close(x[keep], y[keep].double(), TOL["bf16"]["grad"], "grad")
    assert g.last_device_status() == (0, 0)


@pytest.mark.parametrize("q_len", [(40, 200, 100), (130, 300, 257), (0, 150, 129)])
def test_many_newest_positions(g, q_len):
    _check(g, Problem("bf16", 2, LONG, 2, 1, 64, "all", q_len=q_len, cap=30.0, causal=True, slopes=True), grads=False)


def test_rows_that_see_nothing(g):
    p = Problem("bf16", 2, LONG, 2, 2, 64, "fwd", docs=2, causal=True, times="seconds")
    p.docs[:, 5:11] = 77
    p.times[0, :20] = -5.0
    out, lse = _check(g, p)
    assert bool((lse[:, :, 5:11] == -math.inf).all()) and not out[:, 5:11].float().any() and bool((lse[0, :, :20] == -math.inf).all())
    dq, dk, dv = p.backward(g, out, lse)
    assert not dq[:, 5:11].float().any() and not torch.signbit(dq[:, 5:11]).any()


def test_views_of_fused_buffers(g):
    p = Problem("bf16", 2, LONG, 2, 2, 64, "fwd", cap=30.0)
    out, lse = p.forward(g)
    grads = p.backward(g, out, lse)
    L = sum(p.seg)
    buf = torch.randn((2, L, 3 * 128 + 32), device="cuda").bfloat16()
    views = [buf[:, :, 128 * i + 8:128 * i + 136].view(2, L, 2, 64) for i in range(3)]
    for x, t in zip(views, (p.q, p.k, p.v)):
        x.copy_(t)
    q = Problem("bf16", 2, LONG, 2, 2, 64, "fwd", cap=30.0)
    q.q, q.k, q.v = views
    o2, l2 = q.forward(g)
    assert torch.equal(o2, out) and torch.equal(l2, lse)
    wide = torch.full((2, L, 3, 2, 64), 5.0, device="cuda").bfloat16()
    q.backward(g, o2, l2, grads=tuple(wide[:, :, i] for i in range(3)))
    assert all(torch.equal(wide[:, :, i], grads[i]) for i in range(3))


@pytest.mark.parametrize("dtype,hd,seg", [("bf16", 8, SHORT), ("bf16", 32, SHORT), ("bf16", 64, SHORT), ("bf16", 64, LONG), ("f32", 16, SHORT)])
def test_caps_of_almost_nothing(g, dtype, hd, seg):
    """A cap far below the scores leaves equal weights, for rows whose scores are zero as well."""
    p = Problem(dtype, 2, seg, 2, 2, hd, "all", cap=1e-12)
    p.q[:, ::2] = 0
    out, lse = _check(g, p, grads=False)
    assert bool(torch.isfinite(out.float()).all())
    assert all(bool(torch.isfinite(x.float()).all()) for x in p.backward(g, out, lse))
