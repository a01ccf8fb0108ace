"""Streams' caches and attention over them as plain lists of rows, in 64 bits, for the tests of the streaming calls."""
import functools
import math

import numpy as np
import torch

BLOCK = 32
OPEN = {0: ((0, 1), (1, 2), (2, 0)), 1: ((0, 2), (1, 0), (2, 1)), 2: ((0, 0), (1, 1), (2, 2))}


def open_blocks(phase, mask=0):
    return OPEN[phase] if phase in OPEN else tuple((s, r) for s in range(3) for r in range(3) if mask >> (3 * s + r) & 1)


def _grid(held_as):
    """Values that 8 bits have, and which of them end in a 0 bit."""
    if held_as == "int8":
        v = torch.arange(-127, 128, dtype=torch.float64)
        return v, v.long() % 2 == 0
    byte = torch.arange(256, dtype=torch.uint8)
    v = byte.view(torch.float8_e4m3fn).double()
    keep = torch.isfinite(v) & (byte != 0x80)
    v, order = v[keep].sort()
    return v, (byte[keep] % 2 == 0)[order]


def quantised(x, held_as):
    """A block [32, heads, hd] (float64): (8-bit values, scale [heads]) by search among the values there are."""
    values, even = _grid(held_as)
    most = 127.0 if held_as == "int8" else 448.0
    top = x.abs().amax(dim=(0, 2))
    bad = ~torch.isfinite(x).all(dim=2).all(dim=0)
    scale = (top.float() / torch.tensor(most)).double().clamp(min=2.0 ** -80)
    scale = torch.where(bad, torch.ones_like(scale), scale)
    y = torch.where(bad[None, :, None], torch.zeros_like(x), x / scale[None, :, None]).clamp(-most, most)
    middle = (values[1:] + values[:-1]) / 2
    i = torch.searchsorted(middle, y.contiguous())
    at = i.clamp(max=len(middle) - 1)
    i = i + ((i < len(middle)) & (y == middle[at]) & ~even[at]).long()
    return values[i], torch.where(bad, torch.full_like(scale, math.nan), scale)


@functools.lru_cache(maxsize=None)
def addresses(hd, values):
    """[32, hd]: byte of (position, feature) in a page of one head, as gsit_stream.h has them."""
    at = torch.zeros((BLOCK, hd), dtype=torch.long)
    for position in range(BLOCK):
        for feature in range(hd):
            row, col = (feature, position) if values else (position, feature)
            lane, pair = 4 * (row % 8) + col % 8 // 2, col % 2
            if hd == 8:
                at[position, feature] = 8 * lane + (4 * (col // 16) + 2 * (col // 8 % 2) if values else 4 * (row // 16) + 2 * (row // 8 % 2)) + pair
            else:
                outer, inner = (row // 16, col // 16) if values else (col // 16, row // 16)
                at[position, feature] = 512 * outer + 16 * lane + 8 * inner + 4 * (col // 8 % 2) + 2 * (row // 8 % 2) + pair
    return at


def bytes_of(cache, b, s, name):
    """Positions [n, heads, hd] of a segment in 64 bits, from the bytes and scales where they lie."""
    hd, n = cache.open_keys.shape[-1], int(cache.lengths[b, s])
    full = n // BLOCK
    x8, scale, opened = (cache.keys, cache.key_scale, cache.open_keys) if name == "k" else (cache.values, cache.value_scale, cache.open_values)
    page = cache.tables[b, s, :full].long()
    x = x8.view(torch.uint8)[page].view(x8.dtype).double()[:, :, addresses(hd, name == "v").to(x8.device)] * scale[page].double()[:, :, None, None]
    return torch.cat([x.transpose(1, 2).flatten(0, 1), opened[b, s, full % 2, :, :n % BLOCK].double().transpose(0, 1)])


class Streams:
    """What a cache holds: rows of every segment of every stream, on the CPU."""

    def __init__(self, batch, held_as):
        self.held_as = held_as
        self.rows = [[{"k": [], "v": [], "t": []} for _ in range(3)] for _ in range(batch)]

    def step(self, seg, valid, k, v, times=None, ended=None):
        first = np.concatenate([[0], np.cumsum(seg)])
        for b, stream in enumerate(self.rows):
            for s in range(3):
                if ended is not None and ended[b]:
                    stream[s] = {"k": [], "v": [], "t": []}
                for i in range(int(valid[b][s])):
                    stream[s]["k"].append(k[b, first[s] + i].cpu())
                    stream[s]["v"].append(v[b, first[s] + i].cpu())
                    stream[s]["t"].append(float(times[b, first[s] + i]) if times is not None else float(len(stream[s]["t"])))

    def length(self, b, s):
        return len(self.rows[b][s]["k"])

    def held(self, b, s, name, exactly=True):
        """Positions [n, heads, hd] as the cache holds them: in 64 bits, or as the type's rows that it gives back."""
        rows = self.rows[b][s][name]
        if not rows:
            return None
        x = torch.stack(rows)
        full = len(rows) // BLOCK
        parts = []
        for j in range(full):
            q, scale = quantised(x[BLOCK * j:BLOCK * (j + 1)].double(), self.held_as)
            parts.append(q * scale[None, :, None] if exactly else (q.float() * scale.float()[None, :, None]).to(x.dtype))
        last = x[BLOCK * full:]
        if exactly and len(last):
            bad = ~torch.isfinite(last.double()).all(dim=2).all(dim=0)
            last = torch.where(bad[None, :, None], torch.full_like(last, math.nan), last)   # what attention takes of a block with NaN or Inf
        parts.append(last.double() if exactly else last)
        return torch.cat(parts)

    def attention(self, q, seg, valid, pairs, scale, softcap=0.0, slopes=None, times=None, causal=False):
        """(out [B, L, H, hd], lse [B, H, L], the weighted mean of |v| [B, L, H, 1], the largest |score| [B, H, L]) in 64 bits."""
        Bn, L, H, hd = q.shape
        out, size = torch.zeros((Bn, L, H, hd), dtype=torch.float64), torch.zeros((Bn, L, H, hd), dtype=torch.float64)
        lse, most = torch.full((Bn, H, L), -math.inf, dtype=torch.float64), torch.zeros((Bn, H, L), dtype=torch.float64)
        first = np.concatenate([[0], np.cumsum(seg)])
        for b in range(Bn):
            for s in range(3):
                n = int(valid[b][s])
                over = [r for a, r in pairs if a == s and self.length(b, r) > 0]
                if n == 0 or not over:
                    continue
                k, v = (torch.cat([self.held(b, r, name) for r in over]) for name in ("k", "v"))
                group = H // k.shape[1]
                k, v = k.repeat_interleave(group, dim=1), v.repeat_interleave(group, dim=1)
                at = slice(first[s], first[s] + n)
                x = torch.einsum("ihc,jhc->hij", q[b, at].cpu().double(), k) * scale
                if softcap:
                    x = torch.tanh(x / softcap) * softcap
                theirs = torch.tensor([t for r in over for t in self.rows[b][r]["t"]], dtype=torch.float64)
                mine = (times[b, at].cpu().double() if times is not None else torch.arange(self.length(b, s) - n, self.length(b, s)).double())[:, None]
                if slopes is not None:
                    x = x - slopes.cpu().double()[:, None, None] * (mine - theirs[None]).abs()
                shut = (theirs[None] > mine) if causal else torch.zeros((n, len(theirs)), dtype=torch.bool)
                for i in range(n):
                    j = ~shut[i]
                    if not j.any():
                        continue
                    y = x[:, i, j]
                    total = torch.logsumexp(y, dim=1)
                    p = torch.exp(y - total[:, None])
                    out[b, first[s] + i] = torch.einsum("hj,jhc->hc", p, v[j])
                    size[b, first[s] + i] = torch.einsum("hj,jhc->hc", p, v[j].abs()).amax(dim=1, keepdim=True)
                    lse[b, :, first[s] + i] = total
                    most[b, :, first[s] + i] = y.abs().amax(dim=1)
        return out, lse, size, most
