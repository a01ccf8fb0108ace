"""Norms of heads with the rotation in the same pass, and their gradients, against the definition in 64 bits."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

# dtype, batch, segments, heads, key heads, head width, sections, interleaved, padding
CASES = [
    ("bf16", 2, (8, 12, 10), 4, 4, 8, (2, 1, 1), False, True),
    ("bf16", 3, (5, 0, 17), 3, 1, 16, (4, 2, 2), False, True),
    ("bf16", 1, (1, 1, 1), 8, 8, 64, (16, 8, 8), False, False),
    ("bf16", 5, (7, 40, 33), 8, 2, 64, (16, 8, 8), True, True),
    ("bf16", 2, (9, 30, 2), 8, 8, 128, (64,), False, True),
    ("bf16", 2, (9, 30, 2), 20, 3, 128, (30, 34), True, True),       # more heads than a warp's lanes take at once
    ("bf16", 4, (6, 5, 4), 4, 4, 64, (8, 8), False, True),           # the first half of a head rotates, whole pieces of it
    ("bf16", 4, (6, 5, 4), 4, 2, 64, (5, 4), False, True),           # no whole pieces
    ("bf16", 4, (6, 5, 4), 4, 2, 64, (5, 4), True, True),
    ("bf16", 2, (11, 3, 6), 5, 5, 24, (12,), False, True),
    ("bf16", 2, (3, 3, 6), 2, 1, 256, (32, 16, 16), True, True),
    ("bf16", 64, (50, 100, 100), 8, 8, 8, (2, 1, 1), False, True),
    ("f32", 2, (8, 12, 10), 4, 4, 8, (2, 1, 1), False, True),
    ("f32", 3, (5, 1, 17), 6, 3, 16, (8,), True, True),
    ("f32", 2, (30, 48, 23), 8, 8, 32, (8, 4, 4), False, True),
    ("f32", 2, (13, 4, 9), 16, 1, 64, (16, 8, 8), False, False),
    ("f32", 2, (13, 4, 9), 2, 2, 128, (16, 8, 8), False, True),
    ("f32", 2, (4, 4, 9), 2, 1, 7, (2, 1), False, True),
    ("f32", 2, (4, 4, 9), 3, 3, 1, None, False, True),
    ("f32", 1, (1, 0, 0), 1, 1, 33, (16,), True, False),
    ("bf16", 2, (8, 12, 10), 4, 4, 32, None, False, True),
    ("bf16", 2, (8, 12, 10), 4, 4, 32, (0, 0), False, True),
]


@pytest.fixture(scope="module")
def g():
    import paper_2505_01068_b200 as lib
    lib.load()
    return lib


def _inputs(dtype, B, seg, H, HK, hd, sections, padding, seed=0, far=True):
    gen = torch.Generator().manual_seed(seed)
    t, L = torch.bfloat16 if dtype == "bf16" else torch.float32, sum(seg)
    r = lambda *s: torch.randn(s, generator=gen)
    qkv = (r(B, L, H + 2 * HK, hd) * torch.exp(r(H + 2 * HK, 1))).to(t).cuda()
    s = {"q": qkv[:, :, :H], "k": qkv[:, :, H:H + HK], "dq": r(B, L, H, hd).to(t).cuda(), "dk": r(B, L, HK, hd).to(t).cuda(),
         "gq": (1 + 0.3 * r(hd)).cuda(), "gk": (1 + 0.3 * r(hd)).cuda(), "pos": None, "valid": None}
    if sections is not None:
        s["pos"] = torch.randint(-1000, 2 ** 31 - 1 if far else 1000, (len(sections), B, L), generator=gen).int().cuda()
    if padding:
        s["valid"] = torch.stack([torch.randint(0, n + 1, (B,), generator=gen) for n in seg], dim=1).int().cuda()
        s["valid"][0] = torch.tensor(seg, dtype=torch.int32)
    return s


def _real(seg, valid, B):
    n = torch.tensor(seg).expand(B, 3) if valid is None else valid.cpu().long()
    return torch.cat([torch.arange(m)[None] < n[:, i:i + 1] for i, m in enumerate(seg)], dim=1).cuda()


def _rotate(x, pos, sections, interleaved, base, sign):
    if pos is None or sum(sections) == 0:
        return x
    n = sum(sections)
    axis = [a for a, m in enumerate(sections) for _ in range(m)]
    angle = torch.stack([pos[axis[p]].double() * base ** (-p / n) for p in range(n)], dim=-1)[:, :, None]
    z = torch.complex(x[..., 0:2 * n:2], x[..., 1:2 * n:2]) if interleaved else torch.complex(x[..., :n], x[..., n:2 * n])
    z = z * torch.polar(torch.ones_like(angle), sign * angle)
    y = torch.view_as_real(z).flatten(-2) if interleaved else torch.cat([z.real, z.imag], dim=-1)
    return torch.cat([y, x[..., 2 * n:]], dim=-1)


def _reference(x, gamma, dy, pos, sections, interleaved, real, base, eps):
    """(y, dx, dgamma) in 64 bits, and what the errors of each are measured by: the size of the terms that meet in a value."""
    keep = real[:, :, None, None]
    x, dy, gamma = torch.where(keep, x.double(), 0.0), torch.where(keep, dy.double(), 0.0), gamma.double()
    r = (x.square().mean(dim=3, keepdim=True) + eps) ** -0.5
    h = x * r
    y = torch.where(keep, _rotate(h * gamma, pos, sections, interleaved, base, 1), 0.0)
    u = _rotate(dy, pos, sections, interleaved, base, -1)
    gr = u * gamma
    dx = torch.where(keep, r * (gr - h * (gr * h).mean(dim=3, keepdim=True)), 0.0)
    y_size = (h * gamma).abs().amax(dim=3, keepdim=True)
    big = u.abs().amax(dim=3, keepdim=True) * gamma.abs().max()
    dx_size = r * (big + h.abs() * (big * h.abs()).mean(dim=3, keepdim=True))
    return y, dx, (u * h).sum(dim=(0, 1, 2)), y_size, dx_size, (dy.abs().amax(dim=3, keepdim=True) * math.sqrt(2) * h.abs()).sum(dim=(0, 1, 2))


def _close(got, want, size, steps, what):
    """One rounding to the result's type, and `steps` roundings to float of terms of this size."""
    half = torch.finfo(got.dtype).eps / 2
    off = (got.double() - want).abs() - half * 1.01 * want.abs() - steps * 2.0 ** -24 * size
    assert float(off.max()) <= 0, (what, float(off.max()), float((got.double() - want).abs().max()))


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(x) for x in c).replace(" ", ""))
def test_against_the_definition(g, case):
    dtype, B, seg, H, HK, hd, sections, interleaved, padding = case
    s, base, eps = _inputs(dtype, B, seg, H, HK, hd, sections, padding), 10000.0, 1e-6
    args = (s["gq"], s["gk"], s["pos"], sections, seg, s["valid"], base, interleaved, eps)
    got = g.head_norm_rotary_fwd(s["q"], s["k"], *args) + g.head_norm_rotary_bwd(s["dq"], s["dk"], s["q"], s["k"], *args)
    real = _real(seg, s["valid"], B)
    # roundings on the way to a value: the sum of hd squares (their errors are halved by the root), the root's 2 ulp, three products, cosine and sine 4 ulp
    # of angles that are right to 2^-25 turns (10 more); backward twice the sums.  A weight's gradient: one lane adds at most 64 terms here, then 5 + 8 + 32 partial ones.
    fwd, bwd = hd / 2 + 24, 2 * hd + 48
    for i, n in enumerate(("q", "k")):
        y, dx, dg, ys, dxs, dgs = _reference(s[n], s["g" + n], s["d" + n], s["pos"], sections, interleaved, real, base, eps)
        _close(got[i], y, ys, fwd, n)
        _close(got[2 + i], dx, dxs, bwd, "d" + n)
        _close(got[4 + i], dg, dgs, 64 + 64 + hd, "gamma of " + n)
        assert not got[i][~real].any() and not got[2 + i][~real].any()


def test_gradients_against_differences(g):
    """Of the formula itself: along a direction, in float, by central differences of 64 bits' worth of outputs."""
    dtype, B, seg, H, HK, hd, sections = "f32", 2, (4, 6, 5), 2, 1, 16, (4, 2, 2)
    s = _inputs(dtype, B, seg, H, HK, hd, sections, True, far=False)
    args = (s["pos"], sections, seg, s["valid"])
    dq, dk, dgq, dgk = g.head_norm_rotary_bwd(s["dq"], s["dk"], s["q"], s["k"], s["gq"], s["gk"], *args)
    gen = torch.Generator().manual_seed(5)
    way = {n: torch.randn(s[n].shape, generator=gen).cuda() for n in ("q", "k", "gq", "gk")}
    loss = lambda t: sum(float((o.double() * d.double()).sum()) for o, d in
                         zip(g.head_norm_rotary_fwd(s["q"] + t * way["q"], s["k"] + t * way["k"], s["gq"] + t * way["gq"], s["gk"] + t * way["gk"], *args), (s["dq"], s["dk"])))
    step = 2.0 ** -9
    slope = (loss(step) - loss(-step)) / (2 * step)
    terms = [(dq.double() * way["q"].double()), (dk.double() * way["k"].double()), dgq.double() * way["gq"].double(), dgk.double() * way["gk"].double()]
    want = sum(float(t.sum()) for t in terms)
    # outputs of some 500 terms of size 5, each right to 2^-21, over a step of 2^-8: 500^0.5 * 5 * 2^-21 * 2^8 = 0.014; curvature: step^2 / 6 of third derivatives of size
    # 6 |way / x|^3, of which small heads (|x| 0.2) have the most: 2^-18 / 6 * 6 * 125 * 500^0.5 = 0.011.  Four times their sum
    assert abs(slope - want) <= 0.1, (slope, want)


@pytest.mark.parametrize("dtype,hd,sections", [("bf16", 64, (16, 8, 8)), ("f32", 24, (3, 2))])
def test_padding_place_strides_and_bits(g, dtype, hd, sections):
    B, seg, H, HK = 3, (9, 20, 11), 4, 2
    s = _inputs(dtype, B, seg, H, HK, hd, sections, True)
    args = (s["gq"], s["gk"], s["pos"], sections, seg, s["valid"])
    bwd = lambda q, k, dq, dk, **kw: g.head_norm_rotary_bwd(dq, dk, q, k, *args, **kw)
    want = g.head_norm_rotary_fwd(s["q"], s["k"], *args) + bwd(s["q"], s["k"], s["dq"], s["dk"])
    real = _real(seg, s["valid"], B)[:, :, None, None]
    # what stands in padded rows reaches nothing
    dirt = {n: torch.where(real, s[n], float("nan")) for n in ("q", "k", "dq", "dk")}
    got = g.head_norm_rotary_fwd(dirt["q"], dirt["k"], *args) + bwd(dirt["q"], dirt["k"], dirt["dq"], dirt["dk"])
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    # in place, in a buffer with rows further apart, and with weights of their own
    wide = torch.zeros((B, sum(seg), H + 3 * HK, hd), dtype=s["q"].dtype, device="cuda")
    q, k = wide[:, :, :H], wide[:, :, H:H + HK]
    q.copy_(s["q"]); k.copy_(s["k"])
    ret = g.head_norm_rotary_fwd(q, k, *args, out_q=q, out_k=k)
    assert ret[0].data_ptr() == q.data_ptr() and torch.equal(q, want[0]) and torch.equal(k, want[1]) and not wide[:, :, H + HK:].any()
    dq, dk = s["dq"].clone(), s["dk"].clone()
    bwd(s["q"], s["k"], dq, dk, out_q=dq, out_k=dk, workspace=torch.empty(1 << 21, dtype=torch.uint8, device="cuda"))
    assert torch.equal(dq, want[2]) and torch.equal(dk, want[3])
    # an address between the widest loads'
    odd = torch.zeros(s["q"].numel() + 1, dtype=s["q"].dtype, device="cuda")[1:].view(B, sum(seg), H, hd)
    odd.copy_(s["q"])
    y, _ = g.head_norm_rotary_fwd(odd, s["k"], *args)
    assert float((y.double() - want[0].double()).abs().max()) <= 2 * torch.finfo(y.dtype).eps * float(want[0].abs().max())
    # q alone, rows alone, and the gradients of rows alone
    assert torch.equal(g.head_norm_rotary_fwd(s["q"], None, s["gq"], None, *args[2:]), want[0])
    alone = g.head_norm_rotary_bwd(s["dq"], None, s["q"], None, s["gq"], None, *args[2:])
    assert torch.equal(alone[0], want[2]) and float((alone[1] - want[4]).abs().max()) <= 1e-5 * float(want[4].abs().max())
    assert all(torch.equal(a, b) for a, b in zip(bwd(s["q"], s["k"], s["dq"], s["dk"], want_params=False), want[2:4]))
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(bwd(s["q"], s["k"], s["dq"], s["dk"]), want[2:]))


def test_heads_of_zeros_and_of_nan(g):
    """A head of zeros is normalised by eps alone; NaN stays in its head."""
    q = torch.randn((1, 6, 4, 64), device="cuda").bfloat16()
    q[0, 1, 2] = 0
    q[0, 2, 1, 5] = float("nan")
    pos = torch.arange(6, device="cuda", dtype=torch.int32)[None]
    y = g.head_norm_rotary_fwd(q, None, None, None, pos, (32,), (6, 0, 0))
    dq, dg = g.head_norm_rotary_bwd(torch.ones_like(q), None, q, None, None, None, pos, (32,), (6, 0, 0))
    bad = torch.zeros_like(q, dtype=torch.bool)
    bad[0, 2, 1] = True
    assert not y[0, 1, 2].any() and torch.equal(torch.isnan(y), bad) and torch.equal(torch.isnan(dq), bad) and torch.isnan(dg).all()
    assert torch.isfinite(dq[0, 1, 2]).all() and float(dq[0, 1, 2].abs().max()) > 100   # 1 / sqrt(eps)


def test_streams_and_graphs(g):
    """Behind a kernel that writes the inputs late, on a stream of its own, and captured."""
    B, seg, H, hd = 4, (20, 30, 10), 4, 64
    s = _inputs("bf16", B, seg, H, H, hd, (16, 8, 8), True)
    q, k = s["q"].contiguous(), s["k"].contiguous()
    args = (s["gq"], s["gk"], s["pos"], (16, 8, 8), seg, s["valid"])
    want = g.head_norm_rotary_fwd(q, k, *args) + g.head_norm_rotary_bwd(s["dq"], s["dk"], q, k, *args)
    side = torch.cuda.Stream()
    late = torch.zeros_like(q)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        g.late_write(late, q)
        got = g.head_norm_rotary_fwd(late, k, *args)
        late.zero_()
        g.late_write(late, q)
        got += g.head_norm_rotary_bwd(s["dq"], s["dk"], late, k, *args)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = g.head_norm_rotary_fwd(late, k, *args) + g.head_norm_rotary_bwd(s["dq"], s["dk"], late, k, *args)
    late.zero_()
    graph.replay()
    late.copy_(q)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_differentiable(g):
    from paper_2505_01068_b200.training import ImEncoderLayer, head_norm_rotary
    B, seg, H, HK, hd, sections = 2, (5, 8, 6), 4, 2, 16, (4, 2, 2)
    s = _inputs("f32", B, seg, H, HK, hd, sections, True)
    leaves = [s[n].clone().requires_grad_() for n in ("q", "k", "gq", "gk")]
    q, k = head_norm_rotary(*leaves, s["pos"], sections, seg, s["valid"])
    got = torch.autograd.grad((q, k), leaves, (s["dq"], s["dk"]))
    want = g.head_norm_rotary_bwd(s["dq"], s["dk"], s["q"], s["k"], s["gq"], s["gk"], s["pos"], sections, seg, s["valid"])
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    only = head_norm_rotary(leaves[0], None, None, None, s["pos"], sections, seg, s["valid"])
    assert torch.equal(torch.autograd.grad(only, leaves[0], s["dq"])[0],
                       g.head_norm_rotary_bwd(s["dq"], None, s["q"], None, None, None, s["pos"], sections, seg, s["valid"])[0])
    # an encoder layer with it: same as without where the weights do nothing, gradients for both weights
    torch.manual_seed(3)
    layer = ImEncoderLayer(64, 4, seg, sections=sections, dtype=torch.float32, qk_norm=True)
    x = torch.randn((B, sum(seg), 64), device="cuda", requires_grad=True)
    layer(x, s["valid"], s["pos"]).square().sum().backward()
    assert all(p.grad is not None and torch.isfinite(p.grad).all() and p.grad.any() for p in layer.parameters())
    plain = ImEncoderLayer(64, 4, seg, sections=sections, dtype=torch.float32)
    assert "q_g" not in dict(plain.named_parameters()) and len(list(plain.parameters())) == len(list(layer.parameters())) - 2


def test_refuses(g):
    q = torch.zeros((2, 6, 4, 64), device="cuda").bfloat16()
    pos = torch.zeros((1, 6), dtype=torch.int32, device="cuda")
    gamma = torch.ones(64, device="cuda")
    call = lambda q=q, k=None, gq=gamma, gk=None, pos=pos, sections=(32,), seg=(1, 2, 3), **kw: g.head_norm_rotary_fwd(q, k, gq, gk, pos, sections, seg, **kw)
    call()
    for kw in (dict(q=q.cpu()), dict(gq=gamma[:32]), dict(gq=gamma.bfloat16()), dict(gq=gamma.cpu()), dict(pos=None), dict(pos=pos.long()), dict(pos=pos[:, :5]),
               dict(sections=None), dict(sections=(32, 0)), dict(sections=(-1,)), dict(seg=(1, 2, 2)), dict(gk=gamma), dict(k=q[:, :5]), dict(k=q.float()),
               dict(out_q=q[:1]), dict(out_q=q.float())):
        with pytest.raises((AssertionError, TypeError)):
            call(**kw)
    for kw in (dict(sections=(33,)), dict(base=0.0), dict(eps=float("nan"))):
        with pytest.raises(g.GsitError):
            call(**kw)
    with pytest.raises(TypeError):
        call(q=q.half())
    for ws in (torch.empty(1 << 21, dtype=torch.uint8), torch.empty(1 << 22, dtype=torch.uint8, device="cuda")[::2]):
        with pytest.raises(AssertionError):
            g.head_norm_rotary_bwd(q, None, q, None, gamma, None, pos, (32,), (1, 2, 3), workspace=ws)
    with pytest.raises(g.GsitError):
        g.head_norm_rotary_bwd(q, None, q, None, gamma, None, pos, (32,), (1, 2, 3), workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))
