"""What the speed of the framework's training operators is judged by: rotary positions with several axes, layer norm with its
gradients, and interlaced-mask attention whose scores are capped, biased by distance in time and masked by document or by time --
as one training step of an encoder layer, or one step of a stream that receives a new position per modality, calls them.  Shapes
follow the workloads of this repository (aligned and unaligned MOSI / MOSEI, CH-SIMS, MIntRec, a scaled stress shape); `draw`
spreads over the ranges between them.

Kinds of case (the `kind` of a case):
  rotary   q and k of a fused projection rotated (back = False), or their gradients rotated back
  norm     layer norm and its backward pass: result, statistics, gradients of input, weight and bias
  train    attention and its backward pass: result, log-sum-exp, gradients of q, k and v
  stream   attention of the newest position of each segment against all keys

`own` = False computes every operator in plain 32-bit torch operations, True through the framework's calls.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_OPEN = {"fwd": ((0, 1), (1, 2), (2, 0)), "bwd": ((0, 2), (1, 0), (2, 1)), "intra": ((0, 0), (1, 1), (2, 2)),
         "all": tuple((s, r) for s in range(3) for r in range(3))}
_BASE = 10000.0


def _case(kind, dtype, batch, seg, d, heads, padding="half", **more):
    c = {"kind": kind, "dtype": dtype, "batch": batch, "seg0": seg[0], "seg1": seg[1], "seg2": seg[2], "d": d, "heads": heads, "padding": padding}
    if kind == "rotary":
        c |= {"back": False, "axes": 3, "interleaved": False, "far": 0}
    if kind in ("train", "stream"):
        c |= {"kv_heads": heads, "phase": "fwd", "cap": 0.0, "slopes": False, "docs": 0, "causal": False, "prefix": False}
    return c | more


def listed():
    mosei, scaled = (50, 500, 500), (128, 1024, 1024)
    named = {
        # a new position per modality of 32 streams that have run for long: nothing but latency
        "rotary_stream_step": _case("rotary", "bf16", 32, (1, 1, 1), 512, 8, "none", far=100000),
        # queries and keys of an unaligned MOSEI batch, straight out of the fused projection
        "rotary_mosei": _case("rotary", "bf16", 64, mosei, 64, 8),
        # the gradients of the scaled model's queries and keys on their way back to the projection
        "rotary_scaled_back": _case("rotary", "bf16", 128, scaled, 512, 8, "quarter", back=True),
        # one utterance through a layer's norm and back: launches and the reduction's latency
        "norm_one_utterance": _case("norm", "bf16", 1, mosei, 64, 8),
        # the norm of a ring encoder's layer on a MOSEI batch
        "norm_mosei": _case("norm", "bf16", 64, mosei, 64, 8),
        # the norm of the scaled model: the largest activations there are
        "norm_scaled": _case("norm", "bf16", 128, scaled, 512, 8, "quarter"),
        # a toy problem in single precision with every rule but the masks: what a unit test or a notebook calls
        "scores_toy_f32": _case("train", "f32", 2, (8, 12, 10), 32, 4, "none", cap=20.0, slopes=True),
        # the newest position of each modality of 32 streams against everything the stream has seen
        "scores_stream_step": _case("stream", "bf16", 32, scaled, 512, 8, phase="all", cap=50.0, causal=True),
        # cross-modal attention of a MOSEI batch, capped, nearer moments weighted higher
        "scores_mosei": _case("train", "bf16", 64, mosei, 64, 8, cap=30.0, slopes=True),
        # intra-modal attention over rows that hold several utterances each, causal behind a prompt, two heads to a key head
        "scores_chsims_packed": _case("train", "bf16", 32, (39, 55, 400), 128, 4, kv_heads=2, phase="intra", docs=4, causal=True, prefix=True),
        # the unmasked graph in single precision (evaluation of a float model's gradients)
        "scores_mintrec_f32": _case("train", "f32", 8, (30, 480, 230), 128, 8, phase="all", slopes=True),
        # long sequences, wide heads: where the products count
        "scores_scaled": _case("train", "bf16", 32, scaled, 512, 8, "quarter", cap=50.0),
    }
    return [dict(c, name=n) for n, c in named.items()]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the same ranges: batches of 1 to 128, segments of 1 to 1024 steps, widths 32 to 512 with heads of 8 to 64
    (norms: any width of 17 to 2048), every rule on scores alone and together, every kind of padding."""
    kind = rng.choice(("rotary", "norm", "train", "train", "train", "stream"))
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    hd = rng.choice((8, 16, 32, 64))
    widths = [w for w in ((32, 64, 128) if dtype == "f32" and kind == "train" else (32, 64, 96, 128, 192, 256, 512)) if hd <= w <= 16 * hd and w % hd == 0]
    d = rng.choice(widths)
    heads = d // hd
    if kind == "norm":
        d, heads = _log_int(rng, 17, 2048) if rng.random() < 0.5 else rng.choice((32, 64, 128, 256, 512)), 1
    seg = [_log_int(rng, 1, 128), _log_int(rng, 8, 1024), _log_int(rng, 8, 1024)]
    if rng.random() < 0.25:
        rng.shuffle(seg)
    case = _case(kind, dtype, _log_int(rng, 1, 128), seg, d, heads, rng.choice(("half", "half", "quarter", "stats", "none")))
    if kind == "rotary":
        case |= {"back": rng.random() < 0.5, "axes": rng.choice((1, 2, 3, 3)), "interleaved": rng.random() < 0.3, "far": rng.choice((0, 0, 1000, 100000) if dtype == "bf16" else (0, 0, 1000))}   # in 32 bits a far angle is not known well
    if kind in ("train", "stream"):
        case |= {"kv_heads": heads // rng.choice([n for n in (1, 1, 2, 4) if heads % n == 0]), "phase": rng.choice(("fwd", "bwd", "intra", "all")),
                 "cap": rng.choice((0.0, 20.0, 30.0, 50.0)), "slopes": rng.random() < 0.5, "docs": rng.choice((0, 0, 2, 5)),
                 "causal": rng.random() < 0.4}
        case["prefix"] = case["causal"] and rng.random() < 0.5
    while case["batch"] > 1 and _cost(case) > _most(case):
        case["batch"] = max(1, case["batch"] * 3 // 4)
    return case


def _cost(case):
    """About what a pass costs in either form, in seconds."""
    L, es = sum(_seg(case)), 4 if case["dtype"] == "f32" else 2
    c = 8.0 * case["batch"] * L * case["d"] * es / 5e12
    if case["kind"] in ("train", "stream"):
        c += 60.0 * case["batch"] * case["heads"] * L * (L if case["kind"] == "train" else 3) / 5e12
    return c


def _most(case):
    name = {"rotary": "rotary_scaled_back", "norm": "norm_scaled", "stream": "scores_stream_step"}.get(case["kind"])
    name = name or ("scores_mintrec_f32" if case["dtype"] == "f32" else "scores_scaled")
    return _cost(next(c for c in listed() if c["name"] == name))


def _seg(case):
    return (case["seg0"], case["seg1"], case["seg2"])


def _lengths(case, seed):
    """Valid lengths [B, 3]: uniform between half and full, every fourth sample at half, or clipped normals around the averages
    of the MOSEI training split (in proportion to the maxima); None where nothing is padded."""
    rng, seg, b = np.random.default_rng(int(seed) + 17), np.asarray(_seg(case)), case["batch"]
    if case["padding"] == "none":
        return None
    if case["padding"] == "half":
        return np.stack([rng.integers((n + 1) // 2, n + 1, size=b) for n in seg], axis=1).astype(np.int32)
    if case["padding"] == "quarter":
        n = np.tile(seg, (b, 1))
        n[np.arange(b) % 4 == 3] = np.maximum(1, seg // 2)
        return n.astype(np.int32)
    share, spread = np.array([24 / 50, 149 / 500, 94 / 500]), np.array([148 ** 0.5 / 50, 8105 ** 0.5 / 500, 5115 ** 0.5 / 500])
    return np.clip(np.rint(rng.normal(share * seg, spread * seg, size=(b, 3))), 1, seg).astype(np.int32)


def _times(case):
    """Time stamps [L] in seconds: every modality is sampled evenly over the same ten seconds."""
    return np.concatenate([np.arange(n) * (10.0 / max(n, 1)) for n in _seg(case)]).astype(np.float32)


def _documents(case, seed):
    """Document numbers [B, L]: each sample's time axis is cut into `docs` utterances at random moments."""
    rng, t = np.random.default_rng(int(seed) + 29), _times(case)
    cuts = np.sort(rng.uniform(0.5, 9.5, size=(case["batch"], case["docs"] - 1)), axis=1)
    return (t[None, :, None] >= cuts[:, None, :]).sum(axis=2).astype(np.int32)


def _prefix(case, seed):
    """Moment [B] up to which every position may be seen: up to a fifth of the sample."""
    return np.random.default_rng(int(seed) + 31).uniform(0.0, 2.0, size=case["batch"]).astype(np.float32)


def _sections(case):
    """How many of a head's frequencies belong to each axis: half of them to time, the rest to height and width."""
    n = case["d"] // case["heads"] // 2
    return {1: (n,), 2: (n - n // 2, n // 2), 3: (n - 2 * (n // 4), n // 4, n // 4)}[case["axes"]]


# ---------------------------------------------------------------------------------------------------------- inputs

def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    b, d, h, seg, L = case["batch"], case["d"], case["heads"], _seg(case), sum(_seg(case))
    hd, t = d // h, torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    randn = lambda *shape: torch.randn(shape, device="cuda", generator=gen)
    n = _lengths(case, seed)
    s = {"case": case, "seg": seg, "valid": None if n is None else torch.from_numpy(n).cuda()}
    if case["kind"] == "rotary":
        if case["back"]:   # as the attention's backward pass leaves them
            s["q"], s["k"] = randn(b, L, h, hd).to(t), randn(b, L, h, hd).to(t)
        else:              # views of the fused projection
            qkv = randn(b, L, 3, h, hd).to(t)
            s["q"], s["k"] = qkv[:, :, 0], qkv[:, :, 1]
        # text and audio move along all axes together; video frames are grids of 5 x 5 patches
        i = np.concatenate([np.arange(m) for m in seg])
        video = np.arange(L) >= seg[0] + seg[1]
        pos = np.stack([np.where(video, i // 25, i), np.where(video, i // 5 % 5, i), np.where(video, i % 5, i)])[:case["axes"]]
        start = np.random.default_rng(int(seed)).integers(0, case["far"] + 1, size=(1, b, 1))
        s["pos"] = torch.from_numpy((pos[:, None, :] + start).astype(np.int32)).cuda()
        s["sections"] = _sections(case)
        return s
    if case["kind"] == "norm":
        s["x"] = randn(b, L, d) * 1.5 + randn(1, 1, d) * 0.3       # the residual stream, float
        s["gamma"], s["beta"] = 1 + 0.1 * randn(d), 0.1 * randn(d)
        s["dy"] = randn(b, L, d).to(t)                               # from the projection behind the norm, in its type
        s["residual"] = randn(b, L, d)                               # from the layer's residual branch
        return s
    kv = case["kv_heads"]
    rows = 3 if case["kind"] == "stream" else L
    s["q"], s["k"], s["v"] = randn(b, rows, h, hd).to(t), randn(b, L, kv, hd).to(t), randn(b, L, kv, hd).to(t)
    if case["kind"] == "train":
        s["dout"] = randn(b, L, d).to(t)
    s["scale"], s["cap"] = hd ** -0.5, case["cap"]
    s["slopes"] = torch.tensor([2.0 ** (-4.0 * (i + 1) / h) for i in range(h)], device="cuda") if case["slopes"] else None
    s["times"] = torch.from_numpy(_times(case)).cuda().expand(b, L).contiguous() if case["slopes"] or case["causal"] else None
    s["docs"] = torch.from_numpy(_documents(case, seed)).cuda() if case["docs"] else None
    s["prefix"] = torch.from_numpy(_prefix(case, seed)).cuda() if case["prefix"] else None
    return s


# ---------------------------------------------------------------------------------------------------------- one pass

def run(s):
    kind = s["case"]["kind"]
    if own:
        return {"rotary": _own_rotary, "norm": _own_norm}.get(kind, _own_attention)(s)
    return {"rotary": _plain_rotary, "norm": _plain_norm}.get(kind, _plain_attention)(s)


def _own_rotary(s):
    import paper_2505_01068_b200 as g
    call = g.rotary_bwd if s["case"]["back"] else g.rotary_fwd
    return call(s["q"], s["k"], s["pos"], s["sections"], s["seg"], s["valid"], base=_BASE, interleaved=s["case"]["interleaved"])


def _own_norm(s):
    import paper_2505_01068_b200 as g
    y, mean, rstd = g.layer_norm_fwd(s["x"], s["gamma"], s["beta"], s["seg"], s["valid"], out_dtype=s["dy"].dtype, want_stats=True)
    dx, dgamma, dbeta = g.layer_norm_bwd(s["dy"], s["x"], mean, rstd, s["gamma"], s["seg"], s["valid"], residual=s["residual"])
    return {"y": y, "mean": mean, "rstd": rstd, "dx": dx, "dgamma": dgamma, "dbeta": dbeta}


def _own_attention(s):
    import paper_2505_01068_b200 as g
    c = s["case"]
    phase = {"fwd": g.PHASE_INTER_FWD, "bwd": g.PHASE_INTER_BWD, "intra": g.PHASE_INTRA, "all": g.PHASE_CUSTOM}[c["phase"]]
    rule = {"phase": phase, "custom_mask": 0x1FF if c["phase"] == "all" else 0, "softcap": s["cap"], "slopes": s["slopes"], "times": s["times"],
            "documents": s["docs"], "causal": c["causal"], "prefix": s["prefix"]}
    if c["kind"] == "stream":
        return g.im_scored_attention_fwd(s["q"], s["k"], s["v"], s["seg"], s["valid"], q_len=(1, 1, 1), **rule)
    out, lse = g.im_scored_attention_fwd(s["q"], s["k"], s["v"], s["seg"], s["valid"], want_lse=True, **rule)
    dq, dk, dv = g.im_scored_attention_bwd(s["dout"], s["q"], s["k"], s["v"], out, lse, s["seg"], s["valid"], **rule)
    return {"out": out, "lse": lse, "dq": dq, "dk": dk, "dv": dv}


def _real(s):
    """Truth values [B, L] of the positions that are not padding, and the segment [L] of each."""
    seg = torch.tensor(s["seg"], device="cuda")
    which = torch.repeat_interleave(torch.arange(3, device="cuda"), seg)
    place = torch.arange(which.numel(), device="cuda") - (torch.cumsum(seg, 0) - seg)[which]
    if s["valid"] is None:
        return torch.ones((s["case"]["batch"], which.numel()), dtype=torch.bool, device="cuda"), which
    return place[None, :] < s["valid"][:, which], which


def _plain_rotary(s):
    c, (real, _) = s["case"], _real(s)
    hd = c["d"] // c["heads"]
    n = hd // 2
    axis = torch.repeat_interleave(torch.arange(c["axes"], device="cuda"), torch.tensor(s["sections"], device="cuda"))
    freq = torch.tensor([_BASE ** (-p / n) for p in range(n)], device="cuda", dtype=torch.float32)
    angle = (s["pos"].float()[axis] * freq[:, None, None]).permute(1, 2, 0)[:, :, None, :]      # [B, L, 1, n]
    cos, sin = torch.cos(angle), torch.sin(angle) * (-1.0 if c["back"] else 1.0)
    keep = real[:, :, None, None]

    def turn(x):
        x = x.float()
        lo, hi = (x[..., 0::2], x[..., 1::2]) if c["interleaved"] else (x[..., :n], x[..., n:])
        a, b = lo * cos - hi * sin, lo * sin + hi * cos
        y = torch.stack([a, b], dim=-1).flatten(-2) if c["interleaved"] else torch.cat([a, b], dim=-1)
        return torch.where(keep, y, 0.0).to(s["q"].dtype)

    return turn(s["q"]), turn(s["k"])


def _plain_norm(s):
    real, _ = _real(s)
    keep = real[:, :, None]
    x, dy = torch.where(keep, s["x"], 0.0), torch.where(keep, s["dy"].float(), 0.0)
    mean = x.mean(dim=2, keepdim=True)
    rstd = torch.rsqrt((x - mean).square().mean(dim=2, keepdim=True) + 1e-5)
    hat = (x - mean) * rstd
    y = torch.where(keep, hat * s["gamma"] + s["beta"], 0.0).to(s["dy"].dtype)
    g = dy * s["gamma"]
    dx = (g - g.mean(dim=2, keepdim=True) - hat * (g * hat).mean(dim=2, keepdim=True)) * rstd + s["residual"]
    zero = lambda t: torch.where(real, t[:, :, 0], 0.0)
    return {"y": y, "mean": zero(mean), "rstd": zero(rstd), "dx": torch.where(keep, dx, 0.0), "dgamma": (dy * hat).sum(dim=(0, 1)),
            "dbeta": dy.sum(dim=(0, 1))}


def _plain_attention(s):
    """The definition, dense: scores of all pairs, closed ones set to minus infinity, softmax, product; and its derivative."""
    c, (real, which) = s["case"], _real(s)
    b, h, L, ratio = c["batch"], c["heads"], real.shape[1], c["heads"] // c["kv_heads"]
    place = torch.arange(L, device="cuda").expand(b, L)
    if c["kind"] == "stream":   # one row per segment: its last real position
        first = torch.tensor([0, s["seg"][0], s["seg"][0] + s["seg"][1]], device="cuda")
        count = (s["valid"] if s["valid"] is not None else torch.tensor(s["seg"], device="cuda").expand(b, 3)).long()
        at, row_real, row_seg = (first + count - 1).clamp(min=0), count > 0, torch.arange(3, device="cuda")
    else:
        at, row_real, row_seg = place, real, which
    blocks = torch.zeros((3, 3), dtype=torch.bool, device="cuda")
    pairs = torch.tensor(_OPEN[c["phase"]], device="cuda")
    blocks[pairs[:, 0], pairs[:, 1]] = True
    is_open = blocks[row_seg][:, which][None] & row_real[:, :, None] & real[:, None, :]                 # [B, R, L]
    if s["docs"] is not None:
        is_open = is_open & (s["docs"].gather(1, at)[:, :, None] == s["docs"][:, None, :])
    if c["causal"]:
        seen = s["times"][:, None, :] <= s["times"].gather(1, at)[:, :, None]
        is_open = is_open & (seen if s["prefix"] is None else seen | (s["times"][:, None, :] < s["prefix"][:, None, None]))
    is_open = is_open[:, None]
    q = s["q"].float().transpose(1, 2)                                                                  # [B, H, R, hd]
    k, v = (t.float().transpose(1, 2).repeat_interleave(ratio, dim=1) for t in (s["k"], s["v"]))
    x = (q @ k.transpose(2, 3)) * s["scale"]
    bent = None
    if s["cap"]:
        bent = torch.tanh(x / s["cap"])
        x = s["cap"] * bent
    if s["slopes"] is not None:
        x = x - s["slopes"][None, :, None, None] * (s["times"].gather(1, at)[:, :, None] - s["times"][:, None, :]).abs()[:, None]
    x = torch.where(is_open, x, -math.inf)
    top = x.amax(dim=3, keepdim=True)
    p = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(dim=3, keepdim=True)
    p = p / torch.where(total > 0, total, 1.0)
    o = p @ v
    rows = lambda t, like: t.transpose(1, 2).to(like.dtype)
    out = rows(o, s["q"]).reshape(b, -1, c["d"])
    if c["kind"] == "stream":
        return out
    lse = torch.where(total > 0, torch.log(total) + top, -math.inf)[..., 0]
    do = torch.where(row_real[:, :, None], s["dout"].float(), 0.0).reshape(b, L, h, -1).transpose(1, 2)
    share = lambda t: t.reshape(b, c["kv_heads"], ratio, L, -1).sum(dim=2)
    dv = share(p.transpose(2, 3) @ do)
    ds = p * (do @ v.transpose(2, 3) - (do * o).sum(dim=3, keepdim=True))
    if bent is not None:
        ds = ds * (1.0 - bent * bent)
    ds = ds * s["scale"]
    return {"out": out, "lse": lse, "dq": rows(ds @ k, s["q"]), "dk": rows(share(ds.transpose(2, 3) @ q), s["k"]), "dv": rows(dv, s["v"])}


# ---------------------------------------------------------------------------------------------------------- 64 bits

def exact(case, seed):
    """The definitions in 64 bits: rotations as complex products, norms and attention sample by sample over their real positions
    only, gradients by automatic differentiation."""
    s = prepare(case, seed)
    return {"rotary": _exact_rotary, "norm": _exact_norm}.get(case["kind"], _exact_attention)(s)


def _spans(s, b):
    """(first, real positions) of each segment of sample b."""
    n = s["seg"] if s["valid"] is None else [int(m) for m in s["valid"][b]]
    first = (0, s["seg"][0], s["seg"][0] + s["seg"][1])
    return list(zip(first, n))


def _exact_rotary(s):
    c = s["case"]
    n = c["d"] // c["heads"] // 2
    of = [a for a, m in enumerate(s["sections"]) for _ in range(m)]
    angle = torch.stack([s["pos"][of[p]].double() * _BASE ** (-p / n) for p in range(n)], dim=2)
    phase = torch.polar(torch.ones_like(angle), -angle if c["back"] else angle)[:, :, None]
    got = []
    for x in (s["q"].double(), s["k"].double()):
        z = torch.complex(x[..., 0::2], x[..., 1::2]) if c["interleaved"] else torch.complex(x[..., :n], x[..., n:])
        z = z * phase
        y = torch.view_as_real(z).flatten(-2) if c["interleaved"] else torch.cat([z.real, z.imag], dim=-1)
        for b in range(c["batch"]):
            for (at, real), m in zip(_spans(s, b), s["seg"]):
                y[b, at + real:at + m] = 0
        got.append(y)
    return tuple(got)


def _exact_norm(s):
    c = s["case"]
    keep = torch.cat([b * sum(s["seg"]) + torch.arange(at, at + n) for b in range(c["batch"]) for at, n in _spans(s, b)]).cuda()
    flat = lambda t: t.reshape(-1, t.shape[-1])[keep].double()
    x, gamma, beta = flat(s["x"]).requires_grad_(), s["gamma"].double().requires_grad_(), s["beta"].double().requires_grad_()
    var, mean = torch.var_mean(x, dim=1, correction=0, keepdim=True)
    y = (x - mean) / torch.sqrt(var + 1e-5) * gamma + beta
    dx, dgamma, dbeta = torch.autograd.grad(y, (x, gamma, beta), flat(s["dy"]))

    def whole(t, *shape):
        full = torch.zeros((c["batch"] * sum(s["seg"]),) + tuple(t.shape[1:]), dtype=torch.float64, device="cuda")
        full[keep] = t.detach()
        return full.reshape(c["batch"], sum(s["seg"]), *shape)

    return {"y": whole(y, c["d"]), "mean": whole(mean), "rstd": whole((var + 1e-5) ** -0.5), "dx": whole(dx + flat(s["residual"]), c["d"]),
            "dgamma": dgamma, "dbeta": dbeta}


def _exact_attention(s):
    c = s["case"]
    h, kv, hd, stream = c["heads"], c["kv_heads"], c["d"] // c["heads"], c["kind"] == "stream"
    q, k, v = (s[x].double().requires_grad_() for x in ("q", "k", "v"))
    out = torch.zeros((c["batch"], q.shape[1], h, hd), dtype=torch.float64, device="cuda")
    lse = torch.full((c["batch"], h, q.shape[1]), -math.inf, dtype=torch.float64, device="cuda")
    grads = [torch.zeros_like(t) for t in (q, k, v)]
    for b in range(c["batch"]):
        spans = _spans(s, b)
        for a in range(3):
            at, n = spans[a]
            keys = [torch.arange(spans[r][0], spans[r][0] + spans[r][1], device="cuda") for x, r in _OPEN[c["phase"]] if x == a]
            keys = torch.cat(keys) if keys else torch.zeros(0, dtype=torch.long, device="cuda")
            if n == 0 or keys.numel() == 0:
                continue
            row = slice(a, a + 1) if stream else slice(at, at + n)
            place = torch.arange(at + n - 1, at + n, device="cuda") if stream else torch.arange(at, at + n, device="cuda")
            qb, kb, vb = q[b, row], k[b, keys], v[b, keys]
            x = torch.einsum("igrc,jgc->grij", qb.reshape(-1, kv, h // kv, hd), kb).reshape(h, -1, keys.numel()) / math.sqrt(hd)
            if c["cap"]:
                x = torch.tanh(x / c["cap"]) * c["cap"]
            if s["slopes"] is not None:
                t = s["times"][b].double()
                x = x - s["slopes"].double()[:, None, None] * (t[place][:, None] - t[keys][None, :]).abs()
            shut = torch.zeros((place.numel(), keys.numel()), dtype=torch.bool, device="cuda")
            if s["docs"] is not None:
                shut |= s["docs"][b][place][:, None] != s["docs"][b][keys][None, :]
            if c["causal"]:
                late = s["times"][b][keys][None, :] > s["times"][b][place][:, None]
                shut |= late if s["prefix"] is None else late & (s["times"][b][keys] >= s["prefix"][b])[None, :]
            some = ~shut.all(dim=1)
            x, shut = x[:, some].masked_fill(shut[some], -math.inf), shut[some]
            if x.shape[1] == 0:
                continue
            total = torch.logsumexp(x, dim=2)
            o = torch.einsum("grij,jgc->igrc", torch.exp(x - total[:, :, None]).reshape(kv, h // kv, -1, keys.numel()), vb).reshape(-1, h, hd)
            rows = torch.arange(q.shape[1], device="cuda")[row][some]
            out[b, rows], lse[b][:, rows] = o.detach(), total.detach()
            if not stream:
                for full, part, g in zip(grads, ((b, row), (b, keys), (b, keys)), torch.autograd.grad(o, (qb, kb, vb), s["dout"][b, rows].double().reshape(-1, h, hd))):
                    full[part] += g
    out = out.reshape(c["batch"], -1, c["d"])
    return out if stream else {"out": out, "lse": lse, "dq": grads[0], "dk": grads[1], "dv": grads[2]}


# ---------------------------------------------------------------------------------------------------------- what it takes

def _pairs(case):
    """(open (query, key) pairs per head, keys that some query of a sample sees), over real positions."""
    seg, b = np.asarray(_seg(case)), case["batch"]
    n = _lengths(case, 0)
    n = np.tile(seg, (b, 1)) if n is None else n
    if not case["docs"] and not case["causal"] and case["kind"] == "train":
        return int(sum((n[:, s].astype(np.int64) * n[:, r]).sum() for s, r in _OPEN[case["phase"]])), int(n.sum())
    first, t = np.concatenate([[0], np.cumsum(seg)[:2]]), _times(case)
    docs = _documents(case, 0) if case["docs"] else None
    prefix = _prefix(case, 0) if case["prefix"] else None
    pairs, seen = 0, 0
    for i in range(b):
        got = np.zeros(int(seg.sum()), dtype=bool)
        for s, r in _OPEN[case["phase"]]:
            rows, keys = np.arange(first[s], first[s] + n[i, s]), np.arange(first[r], first[r] + n[i, r])
            rows = rows[-1:] if case["kind"] == "stream" else rows
            o = np.ones((len(rows), len(keys)), dtype=bool)
            if docs is not None:
                o &= docs[i][rows][:, None] == docs[i][keys][None, :]
            if case["causal"]:
                late = t[keys][None, :] > t[rows][:, None]
                o &= ~(late if prefix is None else late & (t[keys] >= prefix[i])[None, :])
            pairs += int(o.sum())
            got[keys] |= o.any(axis=0)
        seen += int(got.sum())
    return pairs, seen


def work(case):
    """Real positions read once, whole outputs (padding included, it is written as zero) written once; multiplications and
    additions of the open pairs."""
    n = _lengths(case, 0)
    rows = case["batch"] * sum(_seg(case))
    real = rows if n is None else int(n.sum())
    d, es = case["d"], 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "rotary":
        return {"bytes": 2.0 * d * es * (real + rows) + 4.0 * case["axes"] * real, "flops": 6.0 * real * d}
    if case["kind"] == "norm":   # forward: x in, y out; backward: x, dy and the residual's gradient in, dx out
        return {"bytes": d * ((4.0 + 4.0 + es + 4.0) * real + (es + 4.0) * rows) + 16.0 * rows, "flops": 20.0 * real * d}
    pairs, seen = _pairs(case)
    hd, dk = d // case["heads"], d // case["heads"] * case["kv_heads"]
    if case["kind"] == "stream":
        return {"bytes": 2.0 * seen * dk * es + 6.0 * case["batch"] * d * es, "flops": 4.0 * d * pairs}
    # forward: q, k, v in, out and lse out; backward: q, k, v, out, its gradient and lse in, three gradients out
    return {"bytes": es * (real * (4.0 * d + 4.0 * dk) + rows * (2.0 * d + 2.0 * dk)) + 8.0 * rows * case["heads"], "flops": 14.0 * case["heads"] * hd * pairs}
