"""What the speed of the framework's streaming operators is judged by: norms of queries and keys for each head with the position rotation
in the same pass, a cache that holds the past of a stream in 8 bits with a scale for each block of 32 positions and key head, the tables
that say where its blocks lie, and interlaced-mask attention of a step's rows against it.  Shapes follow the workloads of this repository
(MOSI / MOSEI, CH-SIMS, MIntRec, a scaled stress shape) and streams that have run for longer; `draw` spreads over the ranges between them.

Kinds of case (the `kind` of a case):
  qk       q and k of a fused projection, normalised for each head and rotated
  train    the same with its backward pass: results, gradients of q and k and of both weights
  plan     blocks for what a step adds and for streams that begin anew: slots of the step's rows, lengths, tables
  fill     a step's keys and values appended to a cache, and the whole cache read back as rows
  attend   a step's rows against the cache

A cache is a dict of tensors, the same for both forms.  Block j of segment s of stream b is page tables[b, s, j]; a page holds, for each key
head, 32 positions of `hd` features in 8 bits, keys and values apart, in the order that matrix instructions take them (`_decode` below
says which byte is what), and a scale each.  The last, open block of a segment lies in open_keys[b, s, j % 2] as rows of the model's type.

`own` = False computes every operator in plain 32-bit torch operations, True through the framework's calls.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

BLOCK = 32
_OPEN = {"fwd": ((0, 1), (1, 2), (2, 0)), "bwd": ((0, 2), (1, 0), (2, 1)), "intra": ((0, 0), (1, 1), (2, 2)),
         "all": tuple((s, r) for s in range(3) for r in range(3))}
_BASE, _EPS = 10000.0, 1e-6
_LEAST = 2.0 ** -80   # of a scale


def _case(kind, batch, seg, **more):
    """seg: rows a step brings per segment; held: positions of a segment there may be at most."""
    c = {"kind": kind, "batch": batch, "seg0": seg[0], "seg1": seg[1], "seg2": seg[2], "dtype": "bf16", "heads": 8, "kv_heads": 8, "hd": 64, "padding": "none"}
    if kind in ("qk", "train"):
        c |= {"axes": 3, "interleaved": False, "far": 0}
    else:
        c |= {"held0": 0, "held1": 0, "held2": 0}
    if kind == "plan":
        c |= {"ended": False}
    if kind in ("fill", "attend"):
        c |= {"held_as": "int8"}
    if kind == "attend":
        c |= {"phase": "fwd", "cap": 0.0, "slopes": False, "causal": False}
    return c | more


def _held(n0, n1, n2):
    return {"held0": n0, "held1": n1, "held2": n2}


def listed():
    mosei, scaled = (50, 500, 500), (128, 1024, 1024)
    named = {
        # a new position per modality of 32 streams that have run for long: nothing but latency
        "qk_stream_step": _case("qk", 32, (1, 1, 1), far=100000),
        # queries and keys of the scaled model, two query heads to a key head, straight out of the fused projection
        "qk_scaled": _case("qk", 64, scaled, kv_heads=4, padding="quarter"),
        # a training step of a MOSEI batch through narrow heads in single precision
        "qk_mosei_train_f32": _case("train", 64, mosei, dtype="f32", hd=8, padding="half"),
        # a training step of the scaled model: the largest activations there are
        "qk_scaled_train": _case("train", 128, scaled, padding="quarter"),
        # one position per modality for 32 streams: where do they go?
        "plan_step": _case("plan", 32, (1, 1, 1), **_held(128, 1024, 1024)),
        # prompts of many requests at once, an eighth of them in the place of streams that have ended
        "plan_many": _case("plan", 1024, (16, 100, 100), padding="half", ended=True, **_held(64, 400, 400)),
        # what a MOSEI batch of streams brings in a second, appended to what is there
        "fill_mosei_step": _case("fill", 64, (5, 30, 15), hd=8, padding="half", **_held(45, 470, 480)),
        # whole prompts of the scaled model into an empty cache, in the finer 8 bits for outliers, and back as rows
        "fill_scaled_e4m3": _case("fill", 32, scaled, padding="half", held_as="e4m3"),
        # one stream, one position per modality: launches and latency, in single precision
        "attend_one_f32": _case("attend", 1, (1, 1, 1), dtype="f32", hd=16, **_held(40, 490, 230)),
        # the newest position of each modality of 32 streams against everything they have seen, with every rule on scores
        "attend_stream_step": _case("attend", 32, (1, 1, 1), phase="all", cap=50.0, causal=True, slopes=True, **_held(128, 1024, 1024)),
        # streams that have run for long, four query heads to a key head: the cache's bytes count and nothing else
        "attend_long_e4m3": _case("attend", 64, (1, 1, 1), kv_heads=2, phase="all", held_as="e4m3", **_held(512, 10000, 10000)),
        # a few seconds' positions at once, causal in time, as a stream that lagged behind catches up
        "attend_chunk": _case("attend", 16, (4, 25, 30), kv_heads=4, phase="fwd", causal=True, padding="half", **_held(200, 2000, 2000)),
    }
    return [dict(c, name=n) for n, c in named.items()]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the same ranges: batches of 1 to 128 (plans: to 2048), steps of 1 position per segment to whole segments of 1024, pasts
    of nothing to 16000 positions, heads of 8 to 64 features, 1 to 8 query heads to a key head, every rule alone and together."""
    kind = rng.choice(("qk", "train", "plan", "fill", "attend", "attend", "attend"))
    hd = rng.choice((8, 16, 32, 64))
    kv, group = rng.choice((1, 2, 3, 4, 8)), rng.choice((1, 1, 2, 4, 8))
    more = {"dtype": "f32" if rng.random() < 0.25 else "bf16", "hd": hd, "kv_heads": kv, "heads": kv * group if kv * group <= 16 else kv}
    if kind in ("qk", "train"):
        seg = [1, 1, 1] if rng.random() < 0.25 else [_log_int(rng, 1, 128), _log_int(rng, 8, 1024), _log_int(rng, 8, 1024)]
        more |= {"axes": rng.choice((1, 2, 3, 3)), "interleaved": rng.random() < 0.3, "padding": rng.choice(("none", "half", "quarter")),
                 "far": rng.choice((0, 1000, 100000) if more["dtype"] == "bf16" else (0, 0, 1000))}
        case = _case(kind, _log_int(rng, 1, 128), seg, **more)
    elif kind == "plan":
        seg = [1, 1, 1] if rng.random() < 0.4 else [_log_int(rng, 1, 128), _log_int(rng, 1, 500), _log_int(rng, 1, 500)]
        case = _case(kind, _log_int(rng, 1, 2048), seg, padding=rng.choice(("none", "half")), ended=rng.random() < 0.5,
                     **_held(_log_int(rng, 1, 500), _log_int(rng, 1, 2000), _log_int(rng, 1, 2000)))
    elif kind == "fill":
        more |= {"held_as": rng.choice(("int8", "e4m3")), "padding": rng.choice(("none", "half"))}
        if rng.random() < 0.5:   # prompts
            case = _case(kind, _log_int(rng, 1, 64), [_log_int(rng, 1, 128), _log_int(rng, 8, 1024), _log_int(rng, 8, 1024)], **more)
        else:
            case = _case(kind, _log_int(rng, 1, 64), [rng.randint(0, 16), rng.randint(1, 32), rng.randint(0, 32)], **more,
                         **_held(_log_int(rng, 1, 128), _log_int(rng, 1, 1024), _log_int(rng, 1, 1024)))
    else:
        long = rng.random() < 0.3
        seg = [1, 1, 1] if rng.random() < 0.7 else [rng.randint(0, 6), rng.randint(1, 32), rng.randint(0, 32)]
        more |= {"held_as": rng.choice(("int8", "e4m3")), "padding": rng.choice(("none", "none", "half")), "phase": rng.choice(("fwd", "bwd", "intra", "all", "all")),
                 "cap": rng.choice((0.0, 0.0, 30.0, 50.0)), "slopes": rng.random() < 0.4, "causal": rng.random() < 0.4}
        case = _case(kind, _log_int(rng, 1, 16 if long else 128), seg, **more,
                     **_held(_log_int(rng, 8, 512), _log_int(rng, 32, 16000 if long else 2000), _log_int(rng, 32, 16000 if long else 2000)))
    while case["batch"] > 1 and _cost(case) > _most(kind):
        case["batch"] = max(1, case["batch"] * 3 // 4)
    return case


def _cost(case):
    """About what a pass costs in either form, in seconds."""
    L, es, b = sum(_seg(case)), 4 if case["dtype"] == "f32" else 2, case["batch"]
    heads = case["heads"] + case["kv_heads"]
    if case["kind"] in ("qk", "train"):
        return (2.0 if case["kind"] == "qk" else 6.0) * b * L * heads * case["hd"] * es / 5e12
    if case["kind"] == "plan":
        return (4.0 * b * L + 12.0 * b * _blocks(case)) / 1e12
    past = 3.0 * BLOCK * b * _blocks(case)
    if case["kind"] == "fill":
        return (past + b * L) * case["kv_heads"] * case["hd"] * (2 + 2 * es) / 5e12
    return past * case["kv_heads"] * case["hd"] * 8 / 5e12 + past * case["heads"] * L * (20 + case["hd"]) / 5e12


def _most(kind):
    return max(_cost(c) for c in listed() if c["kind"] == kind)


def _seg(case):
    return (case["seg0"], case["seg1"], case["seg2"])


def _past(case):
    return (case["held0"], case["held1"], case["held2"])


def _blocks(case):
    """Blocks of a segment's row in the tables."""
    return max((h + n + BLOCK - 1) // BLOCK for h, n in zip(_past(case), _seg(case)))


def _type(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _valid(case, seed):
    """Real rows [B, 3] of a step: all, between half and all of them, or half in every fourth sample."""
    rng, seg, b = np.random.default_rng(int(seed) + 17), np.asarray(_seg(case)), case["batch"]
    n = np.tile(seg, (b, 1))
    if case["padding"] == "half":
        n = np.stack([rng.integers((m + 1) // 2, m + 1, size=b) for m in seg], axis=1)
    elif case["padding"] == "quarter":
        n[np.arange(b) % 4 == 3] = np.maximum(1, seg // 2)
    return n.astype(np.int32)


def _lengths(case, seed):
    """Positions [B, 3] that the cache holds before a step: between half of the past there may be and all of it."""
    rng, b = np.random.default_rng(int(seed) + 19), case["batch"]
    return np.stack([rng.integers((m + 1) // 2, m + 1, size=b) for m in _past(case)], axis=1).astype(np.int32)


def _sections(case):
    """How many of a head's frequencies belong to each axis: half of them to time, the rest to height and width."""
    n = case["hd"] // 2
    return {1: (n,), 2: (n - n // 2, n // 2), 3: (n - 2 * (n // 4), n // 4, n // 4)}[case["axes"]]


# ---------------------------------------------------------------------------------------------------------- inputs

def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    randn = lambda *shape: torch.randn(shape, device="cuda", generator=gen)
    b, h, kv, hd, seg, t = case["batch"], case["heads"], case["kv_heads"], case["hd"], _seg(case), _type(case)
    L = sum(seg)
    valid = _valid(case, seed)
    s = {"case": case, "seg": seg, "valid": None if case["padding"] == "none" else torch.from_numpy(valid).cuda()}
    if case["kind"] in ("qk", "train"):
        qkv = (randn(b, L, h + 2 * kv, hd) * (0.5 + 2.0 * torch.rand((h + 2 * kv, 1), device="cuda", generator=gen))).to(t)   # heads of unlike size
        s["q"], s["k"] = qkv[:, :, :h], qkv[:, :, h:h + kv]
        s["q_gamma"], s["k_gamma"] = 1 + 0.2 * randn(hd), 1 + 0.2 * randn(hd)
        # text and audio move along all axes together; video frames are grids of 5 x 5 patches
        i = np.concatenate([np.arange(m) for m in seg])
        video = np.arange(L) >= seg[0] + seg[1]
        pos = np.stack([np.where(video, i // 25, i), np.where(video, i // 5 % 5, i), np.where(video, i % 5, i)])[:case["axes"]]
        start = np.random.default_rng(int(seed)).integers(0, case["far"] + 1, size=(1, b, 1))
        s["pos"] = torch.from_numpy((pos[:, None, :] + start).astype(np.int32)).cuda()
        s["sections"] = _sections(case)
        if case["kind"] == "train":
            s["dq"], s["dk"] = randn(b, L, h, hd).to(t), randn(b, L, kv, hd).to(t)
        return s
    held = _lengths(case, seed)
    if case["kind"] == "attend":   # the step's rows are in the cache already
        s["cache"] = _cache(case, held + valid, gen, seed, times=case["slopes"] or case["causal"])
        s["q"] = randn(b, L, h, hd).to(t)
        s["slopes"] = torch.tensor([2.0 ** (-4.0 * (i + 1) / h) for i in range(h)], device="cuda") if case["slopes"] else None
        if s["cache"]["times"] is not None:
            place = np.concatenate([np.arange(m) for m in seg])
            which = np.repeat(np.arange(3), seg)
            s["times"] = torch.from_numpy(_moment(case, which, held[:, which] + place)).cuda()
        return s
    s["held"] = torch.from_numpy(held).cuda()
    s["cache"] = _cache(case, held, gen, seed)
    if case["kind"] == "plan":
        gone = np.random.default_rng(int(seed) + 23).random(b) < 0.125
        s["ended"] = torch.from_numpy(gone.astype(np.int32)).cuda() if case["ended"] else None
    else:
        s["k"] = randn(b, L, kv, hd) * torch.exp(0.5 * randn(kv, hd))    # some features of the keys are large
        s["k"], s["v"] = s["k"].to(t), randn(b, L, kv, hd).to(t)
        s["whole"] = tuple(p + n for p, n in zip(_past(case), seg))
    return s


def _moment(case, which, place):
    """Moment of a position: every modality is sampled evenly."""
    period = 10.0 / np.maximum(1, np.asarray(_past(case)))
    return (place * period[which]).astype(np.float32)


def _cache(case, n, gen, seed, times=False):
    """A cache that holds n [B, 3] positions, its pages scattered over the pool, the rest of them free."""
    b, kv, hd, m = case["batch"], case["kv_heads"], case["hd"], _blocks(case)
    used = (n + BLOCK - 1) // BLOCK
    pages = 3 * b * m + 7
    order = torch.from_numpy(np.random.default_rng(int(seed) + 11).permutation(pages).astype(np.int32)).cuda()
    here = torch.arange(m, device="cuda")[None, None, :] < torch.from_numpy(used).cuda()[:, :, None]
    tables = torch.full((b, 3, m), -1, dtype=torch.int32, device="cuda")
    taken = int(used.sum())
    tables[here] = order[:taken]
    free = torch.cat([order[taken:], torch.zeros(taken, dtype=torch.int32, device="cuda")])
    c = {"tables": tables, "lengths": torch.from_numpy(n.astype(np.int32)).cuda(), "free": free,
         "n_free": torch.tensor([pages - taken], dtype=torch.int32, device="cuda"), "times": None}
    if case["kind"] == "plan":
        return c
    draw_8 = {"int8": lambda: (40.0 * torch.randn((pages, kv, BLOCK * hd), device="cuda", generator=gen)).round().clamp(-127, 127).to(torch.int8),
              "e4m3": lambda: (140.0 * torch.randn((pages, kv, BLOCK * hd), device="cuda", generator=gen)).clamp(-448, 448).to(torch.float8_e4m3fn)}[case["held_as"]]
    of_one = 1 / 40.0 if case["held_as"] == "int8" else 1 / 140.0
    c["keys"], c["values"] = draw_8(), draw_8()
    for name in ("key_scale", "value_scale"):
        c[name] = of_one * (0.7 + 0.6 * torch.rand((pages, kv), device="cuda", generator=gen))
    for name in ("open_keys", "open_values"):
        c[name] = torch.randn((b, 3, 2, kv, BLOCK, hd), device="cuda", generator=gen).to(_type(case))
    if times:
        when = torch.from_numpy(_moment(case, np.arange(3)[:, None], np.arange(m * BLOCK)[None, :])).cuda()      # [3, m * 32]
        c["times"] = torch.zeros((pages, BLOCK), device="cuda")
        c["times"][tables[here].long()] = when.reshape(1, 3, m, BLOCK).expand(b, 3, m, BLOCK)[here]
    return c


# ---------------------------------------------------------------------------------------------------------- one pass

def run(s):
    kind = s["case"]["kind"]
    if own:
        return {"qk": _own_qk, "train": _own_qk, "plan": _own_plan, "fill": _own_fill, "attend": _own_attend}[kind](s)
    return {"qk": _plain_qk, "train": _plain_qk, "plan": _plain_plan, "fill": _plain_fill, "attend": _plain_attend}[kind](s)


def _own_qk(s):
    import paper_2505_01068_b200 as g
    where = (s["q_gamma"], s["k_gamma"], s["pos"], s["sections"], s["seg"], s["valid"], _BASE, s["case"]["interleaved"], _EPS)
    q, k = g.head_norm_rotary_fwd(s["q"], s["k"], *where)
    if s["case"]["kind"] == "qk":
        return q, k
    dq, dk, dq_gamma, dk_gamma = g.head_norm_rotary_bwd(s["dq"], s["dk"], s["q"], s["k"], *where)
    return {"q": q, "k": k, "dq": dq, "dk": dk, "dq_gamma": dq_gamma, "dk_gamma": dk_gamma}


def _own_cache(s):
    import paper_2505_01068_b200 as g
    return g.StreamCache(**s["cache"])


def _own_plan(s):
    import paper_2505_01068_b200 as g
    cache = g.StreamTables(**{n: s["cache"][n] for n in ("tables", "lengths", "free", "n_free")})
    slots = g.cache_plan(cache, s["seg"], s["valid"], ended=s["ended"], held=s["held"])
    return {"slots": slots, "lengths": cache.lengths, "tables": cache.tables, "n_free": cache.n_free}


def _own_fill(s):
    import paper_2505_01068_b200 as g
    cache = _own_cache(s)
    slots = g.cache_plan(cache, s["seg"], s["valid"], held=s["held"])
    g.cache_append(cache, s["k"], s["v"], slots, s["seg"])
    k, v = g.cache_read(cache, s["whole"])
    return {"slots": slots, "lengths": cache.lengths, "k": k, "v": v}


def _own_attend(s):
    import paper_2505_01068_b200 as g
    c = s["case"]
    phase = {"fwd": g.PHASE_INTER_FWD, "bwd": g.PHASE_INTER_BWD, "intra": g.PHASE_INTRA, "all": g.PHASE_CUSTOM}[c["phase"]]
    out, lse = g.im_cached_attention_fwd(s["q"], _own_cache(s), s["seg"], s["valid"], phase=phase, custom_mask=0x1FF if c["phase"] == "all" else 0, softcap=c["cap"],
                                         slopes=s["slopes"], times=s.get("times"), causal=c["causal"], want_lse=True)
    return {"out": out, "lse": lse}


def _rows(s):
    """The segment [L] of each of a step's rows, its place in it [L], and truth values [B, L] of the rows that are not padding."""
    seg = torch.tensor(s["seg"], device="cuda")
    which = torch.repeat_interleave(torch.arange(3, device="cuda"), seg)
    place = torch.arange(which.numel(), device="cuda") - (torch.cumsum(seg, 0) - seg)[which]
    n = seg.expand(s["case"]["batch"], 3) if s["valid"] is None else s["valid"]
    return which, place, place[None, :] < n[:, which]


def _plain_qk(s):
    c = s["case"]
    n, keep = c["hd"] // 2, _rows(s)[2][:, :, None, None]
    axis = torch.repeat_interleave(torch.arange(c["axes"], device="cuda"), torch.tensor(s["sections"], device="cuda"))
    freq = torch.exp(torch.arange(n, device="cuda", dtype=torch.float64) * (-math.log(_BASE) / n))
    angle = (s["pos"].double()[axis] * freq[:, None, None]).permute(1, 2, 0)[:, :, None, :]      # [B, L, 1, n]; far positions need 64 bits
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()

    def turn(x, sin):
        lo, hi = (x[..., 0::2], x[..., 1::2]) if c["interleaved"] else (x[..., :n], x[..., n:])
        a, b = lo * cos - hi * sin, lo * sin + hi * cos
        return torch.stack([a, b], dim=-1).flatten(-2) if c["interleaved"] else torch.cat([a, b], dim=-1)

    def both(x, gamma, dy):
        t, x = x.dtype, torch.where(keep, x.float(), 0.0)
        r = torch.rsqrt(x.square().mean(dim=3, keepdim=True) + _EPS)
        h = x * r
        y = torch.where(keep, turn(h * gamma, sin), 0.0).to(t)
        if dy is None:
            return y, None, None
        u = turn(torch.where(keep, dy.float(), 0.0), -sin)
        g = u * gamma
        dx = r * (g - h * (g * h).mean(dim=3, keepdim=True))
        return y, dx.to(t), (u * h).sum(dim=(0, 1, 2), dtype=torch.float64).float()

    q, dq, dq_gamma = both(s["q"], s["q_gamma"], s.get("dq"))
    k, dk, dk_gamma = both(s["k"], s["k_gamma"], s.get("dk"))
    return (q, k) if dq is None else {"q": q, "k": k, "dq": dq, "dk": dk, "dq_gamma": dq_gamma, "dk_gamma": dk_gamma}


def _plain_tables(s, ended=None):
    """(tables, lengths, n_free, slots): pages of ended streams go back to the list, the last of them lowest, so that taking from its end gives
    them out in order again; blocks that open take theirs in the order of streams, segments and positions."""
    c, (which, place, real) = s["cache"], _rows(s)
    b, _, m = c["tables"].shape
    tables, held, free, n_free = c["tables"], s["held"].long(), c["free"].long(), c["n_free"].long()
    if ended is not None:
        gone = (ended != 0)[:, None, None]
        back = (gone & (tables >= 0)).flatten()
        count = back.sum()
        at = n_free + count - torch.cumsum(back.long(), 0)      # the first goes on top
        free = torch.zeros(free.numel() + 1, dtype=torch.long, device="cuda").index_copy(0, torch.arange(free.numel(), device="cuda"), free)
        free = free.scatter(0, torch.where(back, at, free.numel() - 1), tables.flatten().long())
        n_free, tables, held = n_free + count, torch.where(gone, -1, tables), torch.where(gone[:, :, 0], 0, held)
    new = held + torch.zeros((b, 3), dtype=torch.long, device="cuda").index_add(1, which, real.long())
    j = torch.arange(m, device="cuda")
    need = ((j < ((new + BLOCK - 1) // BLOCK)[:, :, None]) & (tables < 0)).flatten()
    rank = torch.cumsum(need.long(), 0) - 1
    page = free[(n_free - 1 - rank).clamp(min=0)]
    tables = torch.where(need, page, tables.flatten().long()).reshape(b, 3, m)
    at = held[:, which] + place
    slots = tables.gather(2, (at // BLOCK).clamp(max=m - 1).reshape(b, 1, -1).expand(b, 3, -1))
    slots = slots.gather(1, which.reshape(1, 1, -1).expand(b, 1, -1))[:, 0] * BLOCK + at % BLOCK
    return tables.int(), new.int(), (n_free - need.sum()).int(), torch.where(real, slots, -1).int()


def _plain_plan(s):
    tables, lengths, n_free, slots = _plain_tables(s, s["ended"])
    return {"slots": slots, "lengths": lengths, "tables": tables, "n_free": n_free}


def _decode(x, scale, hd, values):
    """Pages [.., kv, 32 * hd] in 8 bits as float [.., 32, kv, hd].  Keys: position 16 m + 8 h + g, feature 16 s + 8 c + 2 t + e lies at [s][g][t][m][c][h][e];
    values with position and feature exchanged.  Heads of 8 features have no s and c (keys), no m and h (values)."""
    x, lead = x.float() * scale[..., None], x.dim() - 1
    x = x.reshape(x.shape[:-1] + ((hd // 16, 8, 4, 2, 2, 2, 2) if hd > 8 else (8, 4, 2, 2, 2)))
    if hd > 8:     # axes behind the head: outer (s or m), g, t, inner (m or s), c, h, e
        order = (3, 4, 2, 6, "kv", 0, 5, 1) if values else (3, 5, 1, "kv", 0, 4, 2, 6)
    else:          # g, t, inner, h or c, e
        order = (2, 3, 1, 4, "kv", 0) if values else (2, 3, 0, "kv", 1, 4)
    x = x.permute(*range(lead - 1), *(lead - 1 if o == "kv" else lead + o for o in order))
    return x.reshape(x.shape[:lead - 1] + (BLOCK, scale.shape[-1], hd))


def _plain_fill(s):
    """All positions as rows in 32 bits: what was held, then the step's; blocks that it fills go through 8 bits."""
    c, cache, (which, place, real) = s["case"], s["cache"], _rows(s)
    b, kv, hd, m = c["batch"], c["kv_heads"], c["hd"], _blocks(c)
    tables, lengths, _, slots = _plain_tables(s)
    held = s["held"].long()
    block = torch.arange(m, device="cuda")
    full, was_full = (block < (lengths.long() // BLOCK)[:, :, None]), (block < (held // BLOCK)[:, :, None])
    most, step = (127.0, None) if c["held_as"] == "int8" else (448.0, torch.float8_e4m3fn)
    rows_of = torch.arange(b, device="cuda")[:, None].expand(b, which.numel())[real]
    at = (held[:, which] + place)[real]
    got = []
    for name, scale, opened, x in (("keys", "key_scale", "open_keys", s["k"]), ("values", "value_scale", "open_values", s["v"])):
        old = _decode(cache[name], cache[scale], hd, name == "values")[tables.clamp(min=0).long()]             # [B, 3, m, 32, kv, hd]
        rows = cache[opened].float().gather(2, ((held // BLOCK) % 2)[:, :, None, None, None, None].expand(b, 3, 1, kv, BLOCK, hd))[:, :, 0].transpose(2, 3)
        old = torch.where((block == (held // BLOCK)[:, :, None])[..., None, None, None], rows[:, :, None], old)
        old = old.reshape(b, 3, m * BLOCK, kv, hd).index_put((rows_of, which.expand(b, -1)[real], at), x.float()[real]).reshape(b, 3, m, BLOCK, kv, hd)
        new = (full & ~was_full)[..., None, None, None]
        top = torch.where(new, old, 0.0).abs().amax(dim=(3, 5), keepdim=True)
        unit = torch.clamp(torch.div(top, torch.full_like(top, most)), min=_LEAST)
        q = (old.double() / unit.double()).clamp(-most, most)
        if step is None:
            q = torch.round(q)
        else:   # the nearest of 3 bits behind the first, ties to even, 2^-9 at least: in 64 bits, so that nothing is rounded twice
            grain = torch.exp2(torch.floor(torch.log2(q.abs().clamp(min=2.0 ** -6))) - 3)
            q = (torch.round(q / grain) * grain).clamp(-most, most)
        held_rows = torch.where(new, q.float() * unit, old).reshape(b, 3, m * BLOCK, kv, hd)
        there = (torch.arange(m * BLOCK, device="cuda") < lengths.long()[:, :, None])[..., None, None]
        held_rows = torch.where(there, held_rows, 0.0)
        got.append(torch.cat([held_rows[:, 0, :s["whole"][0]], held_rows[:, 1, :s["whole"][1]], held_rows[:, 2, :s["whole"][2]]], dim=1).to(_type(c)))
    return {"slots": slots, "lengths": lengths, "k": got[0], "v": got[1]}


def _plain_attend(s):
    """The definition, dense: the cache as rows, scores of all pairs, closed ones set to minus infinity, softmax, product."""
    c, cache, (which, place, real) = s["case"], s["cache"], _rows(s)
    b, h, kv, hd, m, L = c["batch"], c["heads"], c["kv_heads"], c["hd"], _blocks(c), which.numel()
    n = cache["lengths"].long()
    tables = cache["tables"].clamp(min=0).long()
    is_open_block = torch.arange(m, device="cuda") == (n // BLOCK)[:, :, None]
    buffer = ((n // BLOCK) % 2)[:, :, None, None, None, None].expand(b, 3, 1, kv, BLOCK, hd)

    def rows(name, scale, opened):
        x = _decode(cache[name], cache[scale], hd, name == "values")[tables]
        last = cache[opened].gather(2, buffer)[:, :, 0].transpose(2, 3).float()
        x = torch.where(is_open_block[..., None, None, None], last[:, :, None], x)
        return x.reshape(b, -1, kv, hd)

    k, v = rows("keys", "key_scale", "open_keys"), rows("values", "value_scale", "open_values")
    spot = torch.arange(m * BLOCK, device="cuda")
    there = (spot < n[:, :, None]).reshape(b, -1)                                                 # [B, 3 m 32]
    blocks = torch.zeros((3, 3), dtype=torch.bool, device="cuda")
    pairs = torch.tensor(_OPEN[c["phase"]], device="cuda")
    blocks[pairs[:, 0], pairs[:, 1]] = True
    is_open = blocks[which].repeat_interleave(m * BLOCK, dim=1)[None] & there[:, None, :] & real[:, :, None]
    when = None
    if cache["times"] is not None:
        when = torch.where(there, cache["times"][tables].reshape(b, -1), 0.0)
    if c["causal"]:
        is_open = is_open & (when[:, None, :] <= s["times"][:, :, None])
    q = s["q"].float().reshape(b, L, kv, h // kv, hd)
    x = torch.einsum("bigrc,bjgc->bgrij", q, k) * hd ** -0.5
    if c["cap"]:
        x = c["cap"] * torch.tanh(x / c["cap"])
    if s["slopes"] is not None:
        x = x - s["slopes"].reshape(1, kv, h // kv, 1, 1) * (s["times"][:, :, None] - when[:, None, :]).abs()[:, None, None]
    x = torch.where(is_open[:, None, None], x, -math.inf)
    top = x.amax(dim=4, keepdim=True)
    p = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(dim=4, keepdim=True)
    out = torch.einsum("bgrij,bjgc->bigrc", p / torch.where(total > 0, total, 1.0), v).to(s["q"].dtype).reshape(b, L, h * hd)
    lse = torch.where(total > 0, torch.log(total) + top, -math.inf)[..., 0].reshape(b, h, L)
    return {"out": out, "lse": lse}


# ---------------------------------------------------------------------------------------------------------- 64 bits

def exact(case, seed):
    """The definitions in 64 bits: rotations as complex products and gradients by automatic differentiation, bytes of the cache by the
    address of each, quantisation as a search among the values that 8 bits have, attention stream by stream over what is there."""
    if case["kind"] == "plan":
        return None
    s = prepare(case, seed)
    return {"qk": _exact_qk, "train": _exact_qk, "fill": _exact_fill, "attend": _exact_attend}[case["kind"]](s)


def _spans(s, b):
    """(first row, real rows) of each segment of sample b of a step."""
    n = s["seg"] if s["valid"] is None else [int(m) for m in s["valid"][b]]
    first = (0, s["seg"][0], s["seg"][0] + s["seg"][1])
    return list(zip(first, n))


def _exact_qk(s):
    c = s["case"]
    n, train = c["hd"] // 2, c["kind"] == "train"
    of = [a for a, m in enumerate(s["sections"]) for _ in range(m)]
    angle = torch.stack([s["pos"][of[p]].double() * _BASE ** (-p / n) for p in range(n)], dim=2)
    phase = torch.polar(torch.ones_like(angle), angle)[:, :, None]
    keep = torch.zeros((c["batch"], sum(s["seg"]), 1, 1), dtype=torch.float64, device="cuda")
    for b in range(c["batch"]):
        for at, m in _spans(s, b):
            keep[b, at:at + m] = 1
    got = {}
    for name in ("q", "k"):
        x, gamma = s[name].double().requires_grad_(train), s[name + "_gamma"].double().requires_grad_(train)
        y = x / torch.sqrt((x * x).sum(dim=3, keepdim=True) / c["hd"] + _EPS) * gamma
        z = torch.complex(y[..., 0::2], y[..., 1::2]) if c["interleaved"] else torch.complex(y[..., :n], y[..., n:])
        z = z * phase
        y = (torch.view_as_real(z).flatten(-2) if c["interleaved"] else torch.cat([z.real, z.imag], dim=-1)) * keep
        got[name] = y.detach()
        if train:
            got["d" + name], got["d" + name + "_gamma"] = torch.autograd.grad(y, (x, gamma), s["d" + name].double())
        del x, y, z
    return got if train else (got["q"], got["k"])


def _addresses(hd, values):
    """[32, hd]: where the byte of (position, feature) lies in a page of one head."""
    at = np.zeros((BLOCK, hd), dtype=np.int64)
    for position in range(BLOCK):
        for feature in range(hd):
            row, col = (feature, position) if values else (position, feature)     # of a 16 x 16 operand
            lane = 4 * (row % 8) + col % 8 // 2
            if hd > 8:
                outer, inner = (row // 16, col // 16) if values else (col // 16, row // 16)
                at[position, feature] = 512 * outer + 16 * lane + 8 * inner + 4 * (col % 16 // 8) + 2 * (row % 16 // 8) + col % 2
            elif values:
                at[position, feature] = 8 * lane + 4 * (col // 16) + 2 * (col % 16 // 8) + col % 2
            else:
                at[position, feature] = 8 * lane + 4 * (row // 16) + 2 * (row % 16 // 8) + col % 2
    return torch.from_numpy(at).cuda()


def _exact_rows(cache, b, s, n, hd, values, at):
    """Positions [n, kv, hd] of one segment in 64 bits."""
    name, scale, opened = ("values", "value_scale", "open_values") if values else ("keys", "key_scale", "open_keys")
    full = n // BLOCK
    page = cache["tables"][b, s, :full].long()
    x = cache[name][page].double()[:, :, at] * cache[scale][page].double()[:, :, None, None]       # [full, kv, 32, hd]
    last = cache[opened][b, s, full % 2, :, :n % BLOCK].double()
    return torch.cat([x.transpose(1, 2).reshape(-1, x.shape[1], hd), last.transpose(0, 1)])


def _exact_fill(s):
    c, cache = s["case"], s["cache"]
    kv, hd = c["kv_heads"], c["hd"]
    if c["held_as"] == "int8":
        values, most = torch.arange(-127, 128, dtype=torch.float64, device="cuda"), 127.0
    else:
        every = torch.arange(256, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn).double()
        values, most = torch.unique(every[torch.isfinite(every)]), 448.0
    even = {"int8": values.long() % 2 == 0}.get(c["held_as"])
    if even is None:   # of the last bit of the byte
        even = values.float().to(torch.float8_e4m3fn).view(torch.uint8) % 2 == 0
    middle = (values[1:] + values[:-1]) / 2

    def nearest(x):
        i = torch.searchsorted(middle, x.contiguous())                    # middle[i - 1] < x <= middle[i]
        tie = (i < middle.numel()) & (x == middle[i.clamp(max=middle.numel() - 1)]) & ~even[i.clamp(max=middle.numel() - 1)]
        return values[i + tie.long()]

    got = []
    for name, new in (("keys", s["k"]), ("values", s["v"])):
        at = _addresses(hd, name == "values")
        whole = torch.zeros((c["batch"], sum(s["whole"]), kv, hd), dtype=torch.float64, device="cuda")
        first = np.concatenate([[0], np.cumsum(s["whole"])])
        held = s["held"].cpu().numpy()
        for b in range(c["batch"]):
            for q, (row, n) in enumerate(_spans(s, b)):
                old = int(held[b, q])
                x = torch.cat([_exact_rows(cache, b, q, old, hd, name == "values", at), new[b, row:row + n].double()])
                lo, hi = old // BLOCK, (old + n) // BLOCK
                if hi > lo:
                    part = x[lo * BLOCK:hi * BLOCK].reshape(hi - lo, BLOCK, kv, hd)
                    unit = (part.abs().amax(dim=(1, 3), keepdim=True) / most).float().double().clamp(min=_LEAST)
                    x[lo * BLOCK:hi * BLOCK] = (nearest((part / unit).clamp(-most, most)) * unit).reshape(-1, kv, hd)
                whole[b, first[q]:first[q] + old + n] = x
        got.append(whole)
    return {"k": got[0], "v": got[1]}


def _exact_attend(s):
    c, cache = s["case"], s["cache"]
    h, kv, hd = c["heads"], c["kv_heads"], c["hd"]
    n = cache["lengths"].cpu().numpy()
    if int(n.sum()) * h * sum(s["seg"]) > 1 << 30:
        return None
    at = [_addresses(hd, False), _addresses(hd, True)]
    out = torch.zeros((c["batch"], sum(s["seg"]), h, hd), dtype=torch.float64, device="cuda")
    lse = torch.full((c["batch"], h, sum(s["seg"])), -math.inf, dtype=torch.float64, device="cuda")
    for b in range(c["batch"]):
        keys = [_exact_rows(cache, b, r, int(n[b, r]), hd, False, at[0]) for r in range(3)]
        vals = [_exact_rows(cache, b, r, int(n[b, r]), hd, True, at[1]) for r in range(3)]
        when = [cache["times"][cache["tables"][b, r].clamp(min=0).long()].flatten()[:int(n[b, r])].double() for r in range(3)] if cache["times"] is not None else None
        for a, (row, m) in enumerate(_spans(s, b)):
            over = [r for x, r in _OPEN[c["phase"]] if x == a]
            if m == 0 or sum(int(n[b, r]) for r in over) == 0:
                continue
            k, v = torch.cat([keys[r] for r in over]), torch.cat([vals[r] for r in over])
            q = s["q"][b, row:row + m].double().reshape(m, kv, h // kv, hd)
            x = torch.einsum("igrc,jgc->grij", q, k).reshape(h, m, -1) / math.sqrt(hd)
            if c["cap"]:
                x = torch.tanh(x / c["cap"]) * c["cap"]
            if when is not None:
                mine, theirs = s["times"][b, row:row + m].double()[:, None], torch.cat([when[r] for r in over])[None, :]
                if s["slopes"] is not None:
                    x = x - s["slopes"].double()[:, None, None] * (mine - theirs).abs()
                if c["causal"]:
                    x = x.masked_fill((theirs > mine)[None], -math.inf)
            total = torch.logsumexp(x, dim=2)
            p = torch.where(torch.isinf(total)[:, :, None], 0.0, torch.exp(x - torch.where(torch.isinf(total), 0.0, total)[:, :, None]))
            out[b, row:row + m] = torch.einsum("grij,jgc->igrc", p.reshape(kv, h // kv, m, -1), v).reshape(m, h, hd)
            lse[b, :, row:row + m] = total
    return {"out": out.reshape(c["batch"], -1, h * hd), "lse": lse}


# ---------------------------------------------------------------------------------------------------------- what it takes

def work(case):
    """Real positions read once, whole results (padding included, it is written as zero) written once; multiplications and additions."""
    b, h, kv, hd, seg = case["batch"], case["heads"], case["kv_heads"], case["hd"], _seg(case)
    rows, es, valid = b * sum(seg), 4 if case["dtype"] == "f32" else 2, _valid(case, 0).astype(np.int64)
    real = int(valid.sum())
    if case["kind"] in ("qk", "train"):
        d = (h + kv) * hd
        if case["kind"] == "qk":
            return {"bytes": d * es * (real + rows) + 4.0 * case["axes"] * real, "flops": 10.0 * real * d}
        return {"bytes": d * es * (3.0 * real + 2.0 * rows) + 8.0 * case["axes"] * real, "flops": 30.0 * real * d}
    held = _lengths(case, 0).astype(np.int64)
    opened = int(((held + valid + BLOCK - 1) // BLOCK - (held + BLOCK - 1) // BLOCK).sum())
    if case["kind"] == "plan":   # lengths and counts in, lengths and slots out, a page from the list and an entry for each block that opens
        return {"bytes": 4.0 * (9 * b + rows + 2 * opened), "flops": 0.0}
    n = held + valid
    if case["kind"] == "fill":   # the step's rows in, 8 bits of the blocks that fill up out, everything in and out as rows
        whole = b * sum(p + m for p, m in zip(_past(case), seg))
        full = BLOCK * int((n // BLOCK).sum())
        filled = BLOCK * int((n // BLOCK - held // BLOCK).sum())
        return {"bytes": 2.0 * kv * hd * (es * real + filled + full + es * (int(n.sum()) - full) + es * whole), "flops": 6.0 * kv * hd * (filled + full)}
    read = {r for s, r in _OPEN[case["phase"]] if seg[s] > 0}
    pairs = sum(int((valid[:, s] * n[:, r]).sum()) for s, r in _OPEN[case["phase"]])
    keys = sum(int(n[:, r].sum()) for r in read)
    moments = 4.0 * keys if case["slopes"] or case["causal"] else 0.0
    return {"bytes": 2.0 * keys * kv * (hd + 4.0 / BLOCK) + moments + es * h * hd * (real + rows) + 4.0 * rows * h, "flops": 4.0 * h * hd * pairs}
