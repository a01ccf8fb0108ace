"""Runs an Interlaced-Mask encoder layer over streams of text, audio and video whose past is held in 8 bits: every step brings each stream a few new
positions of each modality -- more of one, fewer of another -- and now and then a stream ends and another begins in its place.  The step is captured into a
CUDA graph once and replayed.

    python examples/stream_encoder.py [--batch 8] [--steps 60] [--held-as int8|e4m3]
"""
from __future__ import annotations

import argparse
import sys
from pathlib import Path

import torch

sys.path.insert(0, str(Path(__file__).resolve().parent.parent))

import paper_2505_01068_b200 as g                                      # noqa: E402
from paper_2505_01068_b200.training import ImEncoderLayer             # noqa: E402

STEP, D, HEADS, KV_HEADS, SECTIONS, MOST = (1, 5, 3), 128, 4, 2, (8, 4, 4), (80, 400, 240)


def further(worst, y, z):
    """The larger of `worst` and the largest difference of two results; NaN once there was one."""
    return torch.cat([worst.reshape(1), (y - z).abs().flatten()]).max()


@torch.no_grad()
def run(batch, steps, held_as):
    """(largest difference of a step's rows from attention over 16-bit rows of the same past, positions held, bytes of the cache, of 16-bit rows)."""
    torch.manual_seed(0)
    layer = ImEncoderLayer(D, HEADS, MOST, kv_heads=KV_HEADS, sections=SECTIONS, qk_norm=True)
    cache = layer.open_cache(batch, MOST, held_as, times=True)
    rule = dict(phase=g.PHASE_CUSTOM, custom_mask=0x1FF, softcap=30.0, causal=True, slopes=torch.tensor([0.5 ** (i + 1) for i in range(HEADS)], device="cuda"))
    rows, segment = sum(STEP), torch.cat([torch.full((n,), s) for s, n in enumerate(STEP)]).cuda()
    place = torch.cat([torch.arange(n) for n in STEP]).cuda()
    rate = torch.tensor([10.0 / n for n in MOST], device="cuda")
    # what a step is given: buffers that the captured step reads
    x = torch.zeros((batch, rows, D), device="cuda")
    valid, ended = torch.zeros((batch, 3), dtype=torch.int32, device="cuda"), torch.zeros(batch, dtype=torch.int32, device="cuda")
    positions, times = torch.zeros((3, batch, rows), dtype=torch.int32, device="cuda"), torch.zeros((batch, rows), device="cuda")
    layer.step(cache, x, STEP, valid, positions, times, ended, **rule)   # once, before the capture
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = layer.step(cache, x, STEP, valid, positions, times, ended, **rule)
    held = torch.zeros((batch, 3), dtype=torch.int32, device="cuda")
    worst = torch.zeros((), device="cuda")
    for i in range(steps):
        x.normal_()
        ended.copy_((torch.rand(batch, device="cuda") < 0.02).int())
        valid.copy_(torch.stack([torch.randint(0, n + 1, (batch,), device="cuda") for n in STEP], dim=1).int())
        held.mul_(1 - ended[:, None])
        at = held[:, segment] + place
        positions.copy_(torch.stack([at, torch.where(segment == 2, at // 5 % 5, at), torch.where(segment == 2, at % 5, at)]).int())
        times.copy_(at * rate[segment])
        graph.replay()
        held.add_(valid)
        assert torch.equal(held, cache.lengths)
        if i % 20 == 19:   # the same rows by attention over the past as 16-bit rows
            k, v = g.cache_read(cache, MOST)
            when = torch.cat([torch.arange(n, device="cuda") * (10.0 / n) for n in MOST]).expand(batch, -1).contiguous()
            q, _, _ = layer.project(x, valid, positions, STEP)
            # a stream's newest rows are the last of its segment: each of them in the place where q_len looks for it
            newest = torch.zeros_like(q)
            back = (torch.tensor(STEP, device="cuda") - valid)[:, segment]
            b = torch.arange(batch, device="cuda")[:, None].expand(batch, rows)
            real = place < valid[:, segment]
            to = torch.arange(rows, device="cuda") + back
            newest[b[real], to[real]] = q[real]
            att = g.im_scored_attention_fwd(newest, k, v, MOST, held, q_len=STEP, times=when, **rule)
            z = layer.finish(x[real][None], att[b[real], to[real]][None], None, (int(real.sum()), 0, 0))
            worst = further(worst, y[real], z[0])
    used = int((cache.tables >= 0).sum())
    per = KV_HEADS * (g.CACHE_BLOCK * (D // HEADS) + 4) * 2
    return float(worst), int(held.sum()), used * per, int(held.sum()) * 2 * KV_HEADS * (D // HEADS) * 2


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--batch", type=int, default=8)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--held-as", choices=("int8", "e4m3"), default="int8")
    a = ap.parse_args(argv)
    got = run(a.batch, a.steps, a.held_as)
    print(f"{got[1]} positions held in {got[2]} bytes of pages (16-bit rows: {got[3]}); largest difference from attention over 16-bit rows: {got[0]:.2e}")
    return got


if __name__ == "__main__":
    main()
