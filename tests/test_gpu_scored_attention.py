"""Attention with a rule on its scores -- cap, bias by distance in time, documents, causality, shared key heads, newest positions only --
forward and backward, against the definition in 64 bits with automatic differentiation, pair by pair."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

# Norm of the error of a whole result.  bf16: the weights (and the score gradients) are rounded once, 2^-9 relative, and the result once
# more; float: sums of up to some thousand products, each 2^-24.  What cancels in a score gradient (p (dP - delta)) leaves an error of
# the size of its terms, which for N(0, 1) inputs are of order one: the second part, per element.
TOL = {"f32": dict(out=1e-5, grad=1e-5), "bf16": dict(out=4e-3, grad=8e-3)}
FLOOR = 0.2


@pytest.fixture(scope="module")
def g():
    import paper_2505_01068_b200 as lib
    lib.load()
    return lib


OPEN = {"fwd": [(0, 1), (1, 2), (2, 0)], "bwd": [(0, 2), (1, 0), (2, 1)], "intra": [(0, 0), (1, 1), (2, 2)],
        "all": [(s, r) for s in range(3) for r in range(3)], "first": [(0, 1), (0, 2)], "none": []}


def _phase(g, name):
    if name in ("fwd", "bwd", "intra"):
        return dict(phase={"fwd": g.PHASE_INTER_FWD, "bwd": g.PHASE_INTER_BWD, "intra": g.PHASE_INTRA}[name])
    return dict(phase=g.PHASE_CUSTOM, custom_mask=sum(1 << (3 * s + r) for s, r in OPEN[name]))


class Problem:
    def __init__(self, dtype, B, seg, H, HK, hd, phase, padded=True, cap=0.0, slopes=False, times=None, docs=0, causal=False, prefix=False, seed=0, q_len=None,
                 amplitude=1.0):
        self.dtype, self.B, self.seg, self.H, self.HK, self.hd, self.phase, self.cap, self.causal = dtype, B, seg, H, HK, hd, phase, cap, causal
        t = torch.float32 if dtype == "f32" else torch.bfloat16
        gen = torch.Generator(device="cuda").manual_seed(seed)
        rng, L = np.random.default_rng(seed), sum(seg)
        randn = lambda *s: torch.randn(s, device="cuda", generator=gen)
        self.q_len = q_len
        self.q = (randn(B, L if q_len is None else sum(q_len), H, hd) * amplitude).to(t)
        self.k, self.v = (randn(B, L, HK, hd) * amplitude).to(t), randn(B, L, HK, hd).to(t)
        self.dout = randn(B, self.q.shape[1], H * hd).to(t)
        n = np.stack([rng.integers(0, m + 1, size=B) for m in seg], axis=1).astype(np.int32) if padded else np.tile(np.array(seg, np.int32), (B, 1))
        if padded and B > 1:
            n[0] = seg
        self.n = n
        self.valid = torch.from_numpy(n).cuda() if padded else None
        self.slopes = torch.tensor([0.5 ** (i + 1) for i in range(H)], device="cuda") if slopes else None
        self.times = None
        place = np.concatenate([np.arange(m) for m in seg])
        if times == "seconds":
            step = np.concatenate([np.full(m, 10.0 / max(m, 1)) for m in seg])
            self.times = torch.from_numpy(np.tile((place * step).astype(np.float32), (B, 1))).cuda()
        elif times == "shuffled":   # moments in no order, far from zero
            self.times = torch.from_numpy((rng.permuted(np.tile(place, (B, 1)), axis=1) * 0.25 + 1000.0).astype(np.float32)).cuda()
        self.docs = torch.from_numpy(rng.integers(0, docs, size=(B, L)).astype(np.int32)).cuda() if docs > 0 else None
        if docs < 0:   # contiguous documents
            self.docs = torch.from_numpy(np.tile(place * -docs // (max(seg) + 1), (B, 1)).astype(np.int32)).cuda()
        self.prefix = (torch.rand(B, device="cuda", generator=gen) * 4.0 + (1000.0 if times == "shuffled" else 0.0)) if prefix else None
        self.place = torch.from_numpy(place).cuda().float()

    def rule(self, g):
        return dict(_phase(g, self.phase), softcap=self.cap, slopes=self.slopes, times=self.times, documents=self.docs, causal=self.causal, prefix=self.prefix)

    def forward(self, g, **kw):
        return g.im_scored_attention_fwd(self.q, self.k, self.v, self.seg, self.valid, q_len=self.q_len, want_lse=True, **self.rule(g), **kw)

    def backward(self, g, out, lse, **kw):
        return g.im_scored_attention_bwd(self.dout, self.q, self.k, self.v, out, lse, self.seg, self.valid, **self.rule(g), **kw)

    def exact(self, grads=True):
        """out, lse and the gradients in float64; rows that are padding or see nothing: 0 / -inf."""
        q, k, v = (t.double().nan_to_num(7.0, 7.0, 7.0).requires_grad_() for t in (self.q, self.k, self.v))
        off = np.concatenate([[0], np.cumsum(self.seg)[:2]])
        q_len = self.q_len or self.seg
        q_off = np.concatenate([[0], np.cumsum(q_len)[:2]])
        out, lse = torch.zeros_like(q), torch.full((self.B, self.H, q.shape[1]), -math.inf, dtype=torch.float64, device="cuda")
        total = torch.zeros((), dtype=torch.float64, device="cuda")
        do = self.dout.double().view_as(q)
        for b in range(self.B):
            t = (self.place if self.times is None else self.times[b]).double()
            for s in range(3):
                n = int(self.n[b, s])
                shift = 0 if self.q_len is None else n - q_len[s]
                rows = torch.arange(max(0, -shift), n - shift, device="cuda")
                keys = torch.cat([torch.arange(off[r], off[r] + self.n[b, r], device="cuda") for x, r in OPEN[self.phase] if x == s]
                                 or [torch.zeros(0, dtype=torch.long, device="cuda")]).long()
                if rows.numel() == 0 or keys.numel() == 0:
                    continue
                pos = (rows + shift + off[s]).long()
                rows = (rows + q_off[s]).long()
                kk, vv = (x[b, keys].repeat_interleave(self.H // self.HK, dim=1) for x in (k, v))
                x = torch.einsum("ihc,jhc->hij", q[b, rows], kk) / math.sqrt(self.hd)
                if self.cap:
                    x = self.cap * torch.tanh(x / self.cap)
                if self.slopes is not None:
                    x = x - self.slopes.double()[:, None, None] * (t[pos][:, None] - t[keys][None]).abs()
                ok = torch.ones(x.shape[1:], dtype=torch.bool, device="cuda")
                if self.docs is not None:
                    ok &= self.docs[b, pos][:, None] == self.docs[b, keys][None]
                if self.causal:
                    see = t[keys][None] <= t[pos][:, None]
                    ok &= see if self.prefix is None else see | (t[keys] < self.prefix[b].double())[None]
                some = ok.any(dim=1)
                if not some.any():
                    continue
                x = torch.where(ok[some][None], x[:, some], -math.inf)
                o = torch.einsum("hij,jhc->ihc", torch.softmax(x, dim=2), vv)
                out.data[b, rows[some]] = o.detach()
                lse[b][:, rows[some]] = torch.logsumexp(x, dim=2).detach()
                total = total + (o * do[b, rows[some]]).sum()
        out = out.detach().reshape(self.B, q.shape[1], -1)
        if not grads:
            return out, lse
        if total.grad_fn is None:
            return (out, lse) + tuple(torch.zeros_like(x) for x in (q, k, v))
        return (out, lse) + tuple(x if x is not None else 0 for x in torch.autograd.grad(total, (q, k, v), allow_unused=True))

    def padding(self):
        """Truth values [B, L] of the padded positions."""
        place = torch.cat([torch.arange(m) for m in self.seg]).cuda()
        n = torch.from_numpy(self.n).cuda()[:, torch.repeat_interleave(torch.arange(3), torch.tensor(self.seg)).cuda()]
        return place[None] >= n


def _close(got, want, tol, what):
    assert got.shape == want.shape
    got = got.double()
    assert bool(torch.isfinite(got).all()), what
    err, norm = float((got - want).norm()), float(want.norm())
    assert err <= tol * (norm + FLOOR * math.sqrt(want.numel())), f"{what}: {err:.3e} of {norm:.3e}"


def _check(g, p, grads=True):
    out, lse = p.forward(g)
    want = p.exact(grads)
    _close(out, want[0], TOL[p.dtype]["out"], "out")
    inf = want[1] == -math.inf
    assert torch.equal(torch.isneginf(lse), inf)
    got, ref = lse[~inf].double(), want[1][~inf]
    assert float((got - ref).abs().max() if ref.numel() else 0.0) <= 2e-5 * (1.0 + float(ref.abs().max() if ref.numel() else 0.0))
    if grads:
        res = p.backward(g, out, lse)
        for x, y, what in zip(res, want[2:], ("dq", "dk", "dv")):
            _close(x, y, TOL[p.dtype]["grad"], what)
        pad = p.padding()
        for x in res + (out,):
            assert not x[pad].float().any() and not torch.signbit(x[pad]).any()
        again = p.backward(g, *p.forward(g))
        assert all(torch.equal(x, y) for x, y in zip(res, again))
    assert g.last_device_status() == (0, 0)
    return out, lse


SHAPES = [(2, (8, 12, 10)), (3, (1, 1, 1)), (2, (0, 5, 17)), (2, (50, 375, 130)), (1, (200, 64, 65)), (2, (3, 600, 33)), (1, (1, 130, 0))]
RULES = [dict(), dict(cap=5.0), dict(cap=30.0, slopes=True), dict(slopes=True, times="seconds"), dict(docs=3), dict(docs=-4, cap=20.0), dict(causal=True),
         dict(causal=True, prefix=True, times="shuffled", slopes=True), dict(docs=-3, causal=True, prefix=True, cap=50.0, slopes=True, times="seconds")]


@pytest.mark.parametrize("rule", RULES, ids=str)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rules_over_shapes(g, dtype, shape, rule):
    heads = {"8": (4, 4), "16": (4, 2), "32": (2, 2), "64": (3, 1)}
    i = (SHAPES.index(shape) + RULES.index(rule)) % 4
    hd = (8, 16, 32, 64)[i]
    phase = ("fwd", "bwd", "intra", "all")[(i + RULES.index(rule) // 2) % 4]
    H, HK = heads[str(hd)]
    _check(g, Problem(dtype, shape[0], shape[1], H, HK, hd, phase, seed=i, **rule))


@pytest.mark.parametrize("hd", [8, 16, 32, 64])
@pytest.mark.parametrize("phase", ["fwd", "bwd", "intra", "all", "first", "none"])
def test_head_widths_and_block_patterns(g, hd, phase):
    _check(g, Problem("bf16", 3, (40, 150, 77), 4, 2, hd, phase, cap=25.0, slopes=True, seed=hd))
    _check(g, Problem("bf16", 2, (40, 150, 277), 2, 2, hd, phase, padded=False, seed=hd + 1))


@pytest.mark.parametrize("hd", [1, 5, 24, 40, 100, 128])
def test_float_takes_any_head_width(g, hd):
    _check(g, Problem("f32", 2, (7, 70, 33), 3, 1, hd, "all", cap=10.0, slopes=True, docs=2, causal=True, seed=hd))


@pytest.mark.parametrize("heads", [(8, 8), (8, 4), (8, 1), (6, 3), (5, 5), (16, 2), (1, 1)])
@pytest.mark.parametrize("dtype,hd", [("bf16", 8), ("bf16", 64), ("f32", 16)])
def test_shared_key_heads_add_their_gradients(g, dtype, hd, heads):
    _check(g, Problem(dtype, 2, (20, 90, 45), heads[0], heads[1], hd, "bwd", cap=30.0, seed=sum(heads)))


@pytest.mark.parametrize("amplitude", [0.01, 4.0, 9.0])
@pytest.mark.parametrize("dtype,hd", [("bf16", 8), ("bf16", 16), ("bf16", 64), ("f32", 32)])
@pytest.mark.parametrize("cap", [0.0, 2.0, 60.0])
def test_small_and_large_scores(g, dtype, hd, amplitude, cap):
    """Scores of some hundred: one key takes all of the softmax, and the cap is reached.  In bf16 the result is held to the forward
    tolerance only: where scores saturate, a gradient is what is left of terms that cancel."""
    p = Problem(dtype, 2, (30, 140, 80), 2, 2, hd, "all", cap=cap, amplitude=amplitude)
    out, lse = p.forward(g)
    want = p.exact()
    _close(out, want[0], max(TOL[dtype]["out"], 4e-4 if dtype == "f32" and amplitude > 1 else 0.0), "out")
    for x, y in zip(p.backward(g, out, lse), want[2:]):
        assert bool(torch.isfinite(x).all())
        assert float((x.double() - y).norm()) <= 2e-2 * (float(y.norm()) + amplitude * math.sqrt(y.numel()))


def test_far_moments_leave_the_nearest_key(g):
    """Biases of up to 2 10^7: every weight but the nearest key's vanishes (the next one is 2^-400 at the least), and none is lost to
    underflow: the result is that key's value, the log-sum-exp its bias to float rounding.  Of two keys at the same distance the scores
    differ by less than their own rounding, so that such rows are only held to be a mean of the two values."""
    seg, slopes = (10, 300, 40), (300.0, 1e4)
    at = torch.cat([torch.arange(10) * 100.0 + 7.0, torch.arange(300) * 1.0 - 2000.0, torch.arange(40) * 3.0]).cuda().float()
    first = (0, 10, 310)
    for dtype in ("f32", "bf16"):
        p = Problem(dtype, 2, seg, 2, 2, 8, "fwd", slopes=True, padded=False)
        p.slopes = torch.tensor(slopes, device="cuda")
        p.times = at.expand(2, 350).contiguous()
        out, lse = p.forward(g)
        out, ties = out.view(2, 350, 2, 8).float(), 0
        for s, r in OPEN["fwd"]:
            rows, keys = (slice(first[x], first[x] + seg[x]) for x in (s, r))
            far, which = torch.topk((at[rows][:, None] - at[keys][None]).abs(), 2, dim=1, largest=False)
            v = p.v[:, keys].float()
            near, next_ = v[:, which[:, 0]], v[:, which[:, 1]]
            unique = far[:, 1] > far[:, 0]
            assert torch.equal(out[:, rows][:, unique], near[:, unique])
            lo, hi = torch.minimum(near, next_), torch.maximum(near, next_)
            assert bool(((out[:, rows] >= lo - 0.05) & (out[:, rows] <= hi + 0.05)).all())
            bias = far[:, 0] * p.slopes[:, None]
            assert bool(((lse[:, :, rows] + bias).abs() <= 20.0 + 2.0 ** -21 * bias).all())
            ties += int((~unique).sum())
        assert ties > 0
        for x in p.backward(g, *p.forward(g)):
            assert bool(torch.isfinite(x).all())


@pytest.mark.parametrize("dtype,hd", [("bf16", 8), ("bf16", 16), ("bf16", 32), ("bf16", 64), ("f32", 16)])
@pytest.mark.parametrize("fill", [float("nan"), float("inf"), -3.38e38])
def test_what_stands_in_padding_and_in_closed_documents_never_matters(g, dtype, hd, fill):
    seg = (20, 130, 70)
    p = Problem(dtype, 2, seg, 2, 1, hd, "all", docs=-3, causal=True, seed=5, cap=20.0)
    clean = p.backward(g, *p.forward(g))
    base = p.forward(g)
    pad, other = p.padding(), p.docs == 1
    for t in (p.q, p.k, p.v, p.dout):
        t[pad] = fill
    out, lse = p.forward(g)
    assert torch.equal(out, base[0]) and torch.equal(lse, base[1])
    assert all(torch.equal(x, y) for x, y in zip(p.backward(g, out, lse), clean))
    for t in (p.q, p.k, p.v, p.dout):      # one document is broken: the others' rows do not notice, to rounding
        t[other & ~pad] = fill
    out, lse = p.forward(g)
    keep = ~other
    _close(out[keep], base[0][keep].double(), TOL[dtype]["out"], "out")
    for x, y in zip(p.backward(g, out, lse), clean):
        _close(x[keep], y[keep].double(), TOL[dtype]["grad"], "grad")
    assert g.last_device_status() == (0, 0)


@pytest.mark.parametrize("hd", [8, 64])
def test_warps_of_uneven_speed(g, hd):
    """Large values in one document send some warps of a tile through the form of the cap for any argument, others not: whoever is ahead
    must not take a result before it is whole.  The other documents' rows keep their values on every one of many runs."""
    p = Problem("bf16", 2, (20, 130, 70), 2, 1, hd, "all", docs=-3, causal=True, seed=5, cap=20.0)
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


def test_rows_that_see_nothing(g):
    """Documents without a key, and moments before every key: +0, -inf and no gradient."""
    for dtype in ("f32", "bf16"):
        p = Problem(dtype, 2, (20, 90, 30), 2, 2, 16, "fwd", docs=2, causal=True, times="seconds")
        p.docs[:, 5:11] = 77
        p.times[0, :20] = -5.0
        out, lse = _check(g, p)
        assert bool((lse[:, :, 5:11] == -math.inf).all()) and not out[:, 5:11].float().any() and bool((lse[0, :, :20] == -math.inf).all())
        dq, dk, dv = p.backward(g, out, lse)
        assert not dq[:, 5:11].float().any() and not torch.signbit(dq[:, 5:11]).any()


@pytest.mark.parametrize("q_len", [(1, 1, 1), (0, 1, 0), (2, 3, 1), (5, 0, 17), (20, 90, 45)])
@pytest.mark.parametrize("dtype,hd,HK", [("bf16", 8, 4), ("bf16", 16, 2), ("bf16", 32, 1), ("bf16", 64, 4), ("f32", 24, 2)])
@pytest.mark.parametrize("rule", [dict(), dict(cap=30.0, causal=True, slopes=True), dict(docs=-3, causal=True, prefix=True, times="seconds")], ids=str)
def test_newest_positions_only(g, q_len, dtype, hd, HK, rule):
    _check(g, Problem(dtype, 3, (20, 90, 45), 4, HK, hd, "all", q_len=q_len, **rule), grads=False)


@pytest.mark.parametrize("q_len", [(1, 1, 1), (2, 0, 1)])
@pytest.mark.parametrize("hd,H,HK", [(8, 4, 2), (16, 2, 2), (32, 4, 2), (64, 3, 3)])
@pytest.mark.parametrize("rule", [dict(), dict(cap=30.0, causal=True, slopes=True), dict(docs=-3, causal=True, prefix=True, times="seconds")], ids=str)
def test_newest_positions_of_streams_that_have_run_for_long(g, q_len, hd, H, HK, rule):
    _check(g, Problem("bf16", 2, (301, 450, 270), H, HK, hd, "all", q_len=q_len, **rule), grads=False)


@pytest.mark.parametrize("dtype,hd", [("bf16", 8), ("bf16", 64), ("f32", 32)])
def test_newest_position_over_long_keys(g, dtype, hd):
    p = Problem(dtype, 2, (5, 5000, 3001), 4, 2, hd, "all", q_len=(1, 1, 1), cap=30.0, slopes=True, times="seconds", causal=True)
    _check(g, p, grads=False)
    q = Problem(dtype, 2, (5, 5000, 3001), 4, 2, hd, "all", q_len=(1, 1, 1), docs=-7)
    _check(g, q, grads=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_views_of_fused_buffers(g, dtype):
    """q, k, v inside one projection buffer, the gradients written into another, in rows that are longer than needed."""
    p = Problem(dtype, 2, (20, 70, 35), 4, 4, 16, "fwd", cap=30.0)
    out, lse = p.forward(g)
    grads = p.backward(g, out, lse)
    L = sum(p.seg)
    buf = torch.randn((2, L, 3 * 64 + 32), device="cuda").to(p.q.dtype)
    views = [buf[:, :, 64 * i + 8:64 * i + 72].view(2, L, 4, 16) for i in range(3)]
    for x, t in zip(views, (p.q, p.k, p.v)):
        x.copy_(t)
    q = Problem(dtype, 2, (20, 70, 35), 4, 4, 16, "fwd", cap=30.0)
    q.q, q.k, q.v = views
    o2, l2 = q.forward(g)
    assert torch.equal(o2, out) and torch.equal(l2, lse)
    wide = torch.full((2, L, 3, 4, 16), 5.0, device="cuda").to(p.q.dtype)
    res = q.backward(g, o2, l2, grads=tuple(wide[:, :, i] for i in range(3)))
    for i in range(3):
        assert torch.equal(wide[:, :, i], grads[i]) and res[i].data_ptr() == wide[:, :, i].data_ptr()
    given = torch.empty_like(out)
    assert p.forward(g, out=given)[0].data_ptr() == given.data_ptr() and torch.equal(given, out)


def test_rows_further_apart_than_32_bits_count(g):
    """Offsets beyond 2^31 elements: keys and values in the rows of a cache with room for many more features."""
    p = Problem("bf16", 1, (4, 600, 0), 1, 1, 8, "fwd", padded=False)
    stride = 2 ** 22
    if torch.cuda.mem_get_info()[0] < 12 << 30:
        pytest.skip("needs 12 GB")
    room = torch.empty((604 * stride,), dtype=torch.bfloat16, device="cuda")
    k = room.as_strided((1, 604, 1, 8), (604 * stride, stride, 8, 1))
    v = room.as_strided((1, 604, 1, 8), (604 * stride, stride, 8, 1), 64)
    k.copy_(p.k)
    v.copy_(p.v)
    out, lse = p.forward(g)
    grads = p.backward(g, out, lse)
    p.k, p.v = k, v
    o2, l2 = p.forward(g)
    assert torch.equal(o2, out) and torch.equal(l2, lse)
    assert all(torch.equal(x, y) for x, y in zip(p.backward(g, o2, l2), grads))


@pytest.mark.parametrize("rule", [dict(cap=3.0, slopes=True), dict(docs=2, causal=True, prefix=True, times="seconds")], ids=str)
def test_gradients_are_differences(g, rule):
    """d/dt <f(q + t e, ...), w> by centred differences of the float kernel's results, t = 2^-7, summed in 64 bits.  The third derivative
    leaves t^2 / 6 of a term of the size of the first, rounding 2^-23 |f| |w| / t: below 2e-3 of |e| |w| / sqrt(n)."""
    p = Problem("f32", 2, (15, 40, 25), 4, 2, 16, "all", **rule)
    out, lse = p.forward(g)
    grads = p.backward(g, out, lse)
    w, t = p.dout.double(), 2.0 ** -7
    for name, grad in zip("qkv", grads):
        x = getattr(p, name)
        e = torch.randn_like(x)
        val = []
        for s in (t, -t):
            setattr(p, name, x + s * e)
            val.append(float((p.forward(g)[0].double() * w).sum()))
        setattr(p, name, x)
        want = float((grad.double() * e.double()).sum())
        assert abs((val[0] - val[1]) / (2 * t) - want) <= 2e-3 * float(e.norm() * w.norm()) / math.sqrt(e.numel()) * 4


def test_other_streams(g):
    """Calls on a stream of their own, behind inputs written there."""
    p = Problem("bf16", 2, (20, 90, 45), 4, 4, 16, "fwd", cap=30.0, docs=2)
    want = p.forward(g)
    grads = p.backward(g, *want)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    q = p.q.clone()
    with torch.cuda.stream(st):
        p.q = (q * 2) / 2
        got = p.forward(g)
        res = p.backward(g, *got)
    st.synchronize()
    assert torch.equal(got[0], want[0]) and all(torch.equal(x, y) for x, y in zip(res, grads))


def test_refusals(g):
    p = Problem("bf16", 2, (6, 10, 8), 4, 2, 16, "fwd", padded=False)
    out, lse = p.forward(g)
    call = lambda q=p.q, k=p.k, v=p.v, seg=p.seg, **kw: g.im_scored_attention_fwd(q, k, v, seg, **kw)
    for kw in (dict(k=p.k.float()), dict(k=p.k[:, :23]), dict(v=p.v[:, :, :1]), dict(seg=(6, 10, 7)), dict(slopes=torch.ones(3, device="cuda")),
               dict(times=torch.ones((2, 24), device="cuda").double()), dict(documents=torch.ones((2, 24), device="cuda")), dict(q_len=(1, 1, 1)),
               dict(prefix=torch.ones(3, device="cuda"), causal=True), dict(out=out[:, :5]), dict(q=p.q.transpose(1, 2))):
        with pytest.raises(AssertionError):
            call(**kw)
    k3 = torch.zeros((2, 24, 3, 16), device="cuda", dtype=torch.bfloat16)
    buf = torch.zeros((2, 24, 4 * 16 + 4), device="cuda", dtype=torch.bfloat16)
    for kw, code in ((dict(k=k3, v=k3), 1), (dict(softcap=float("nan")), 1), (dict(custom_mask=0x200, phase=g.PHASE_CUSTOM), 1),
                     (dict(q=buf[:, :, :64].view(2, 24, 4, 16)), 1)):
        with pytest.raises(g.GsitError) as e:
            call(**kw)
        assert e.value.code == code
    q24 = torch.zeros((2, 24, 2, 24), device="cuda", dtype=torch.bfloat16)
    with pytest.raises(g.GsitError) as e:
        call(q=q24, k=q24, v=q24)
    assert e.value.code == 2
    with pytest.raises(g.GsitError) as e:
        g.im_scored_attention_bwd(p.dout, p.q, p.k, p.v, out, lse, p.seg, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    assert e.value.code == 3
    with pytest.raises(AssertionError):
        g.im_scored_attention_bwd(p.dout, p.q, p.k, p.v, out, lse, p.seg, grads=(p.q, p.k))
    with pytest.raises(TypeError):
        call(q=p.q.half(), k=p.k.half(), v=p.v.half())
