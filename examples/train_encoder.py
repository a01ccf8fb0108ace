"""Trains two Interlaced-Mask encoder layers -- a forward ring and a backward ring over text, audio and video -- on synthetic batches with
capped scores, a bias by distance in time and three-axis rotary positions, then runs the first layer over a stream: one new position per
modality at a time against the keys seen so far.

    python examples/train_encoder.py [--steps 30] [--batch 16] [--dtype bf16|f32]
"""
from __future__ import annotations

import argparse
import sys
from pathlib import Path

import torch

sys.path.insert(0, str(Path(__file__).resolve().parent.parent))

import paper_2505_01068_b200 as g                                      # noqa: E402
from paper_2505_01068_b200.training import ImEncoderLayer             # noqa: E402

SEG, D, HEADS, SECTIONS = (50, 125, 100), 64, 8, (2, 1, 1)


def clock(batch):
    """Moments [B, L] in seconds, every modality sampled over the same ten seconds, and positions [3, B, L]: time for all, and for video
    the row and column of a 5 x 5 grid of patches."""
    step = torch.cat([torch.full((n,), 10.0 / n) for n in SEG])
    place = torch.cat([torch.arange(n) for n in SEG])
    video = torch.arange(sum(SEG)) >= SEG[0] + SEG[1]
    pos = torch.stack([torch.where(video, place // 25, place), torch.where(video, place // 5 % 5, place), torch.where(video, place % 5, place)])
    return (place * step).float().expand(batch, -1).contiguous().cuda(), pos.int()[:, None].expand(3, batch, -1).contiguous().cuda()


def train(steps, batch, dtype):
    """Losses of the first and the last steps (means of five)."""
    torch.manual_seed(0)
    layers = torch.nn.ModuleList(ImEncoderLayer(D, HEADS, SEG, sections=SECTIONS, dtype=dtype) for _ in range(2))
    head = torch.nn.Linear(D, 1).cuda()
    opt = torch.optim.Adam([*layers.parameters(), *head.parameters()], lr=3e-3)
    times, pos = clock(batch)
    slopes = torch.tensor([2.0 ** -(i + 1) for i in range(HEADS)], device="cuda")
    rule = {"softcap": 30.0, "slopes": slopes, "times": times}
    seg = torch.tensor(SEG, device="cuda")
    losses = []
    for _ in range(steps):
        x = torch.randn((batch, sum(SEG), D), device="cuda")
        valid = torch.stack([torch.randint((n + 1) // 2, n + 1, (batch,)) for n in SEG], dim=1).int().cuda()
        real = torch.cat([torch.arange(n, device="cuda") for n in SEG])[None] < torch.repeat_interleave(valid, seg, dim=1)
        # something one layer can learn: the mean over the audio of one feature, asked for at every real text step
        audio = slice(SEG[0], SEG[0] + SEG[1])
        want = (x[:, audio, 0] * real[:, audio]).sum(dim=1) / valid[:, 1] * 5.0
        y = layers[1](layers[0](x, valid, pos, phase=g.PHASE_INTER_FWD, **rule), valid, pos, phase=g.PHASE_INTER_BWD, **rule)
        text = real[:, :SEG[0]]
        loss = (((head(y[:, :SEG[0]])[..., 0] - want[:, None]) ** 2) * text).sum() / text.sum()
        opt.zero_grad()
        loss.backward()
        opt.step()
        losses.append(float(loss.detach()))
    return sum(losses[:5]) / 5, sum(losses[-5:]) / 5


@torch.no_grad()
def stream(batch, dtype):
    """The layer over a stream: largest difference between the rows computed one position at a time and the whole pass."""
    torch.manual_seed(1)
    layer = ImEncoderLayer(D, HEADS, SEG, sections=SECTIONS, dtype=dtype)
    times, pos = clock(batch)
    x = torch.randn((batch, sum(SEG), D), device="cuda")
    full = dict(phase=g.PHASE_CUSTOM, custom_mask=0x1FF, softcap=30.0, times=times, causal=True)
    q, k, v = layer.project(x, None, pos)
    whole = layer.finish(x, g.im_scored_attention_fwd(q, k, v, SEG, **full), None)
    first = (0, SEG[0], SEG[0] + SEG[1])
    worst = 0.0
    for n in ((1, 1, 1), (7, 18, 14), (30, 77, 61), SEG):   # how much of each modality the stream has seen
        valid = torch.tensor([n] * batch, dtype=torch.int32, device="cuda")
        at = [first[s] + n[s] - 1 for s in range(3)]
        att = g.im_scored_attention_fwd(q[:, at].contiguous(), k, v, SEG, valid, q_len=(1, 1, 1), **full)
        y = layer.finish(x[:, at].contiguous(), att, seg_len=(1, 1, 1))
        # the whole pass sees the same keys only where all that is not later has arrived: the modality that lags behind
        s = min(range(3), key=lambda i: float(times[0, at[i]]))
        worst = max(worst, float((y[:, s] - whole[:, at[s]]).abs().max()))
    return worst


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--batch", type=int, default=16)
    ap.add_argument("--dtype", choices=("bf16", "f32"), default="bf16")
    a = ap.parse_args(argv)
    dtype = torch.bfloat16 if a.dtype == "bf16" else torch.float32
    first, last = train(a.steps, a.batch, dtype)
    off = stream(a.batch, dtype)
    print(f"loss {first:.4f} -> {last:.4f}; stream against whole pass: {off:.2e}")
    return first, last, off


if __name__ == "__main__":
    main()
