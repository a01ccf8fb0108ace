"""Training of Interlaced-Mask encoder layers: the operators of gsit_ops.h as differentiable functions of torch, and an encoder layer
made of them.

The functions sequence library calls only: what they save for the backward pass is what those calls ask for (statistics of a norm,
result and log-sum-exp of an attention), and every gradient is one library call.  The linear layers are plain torch products in the
type of their weights, as the rest of a training program's are."""
from __future__ import annotations

import torch
from torch.autograd.function import once_differentiable

from . import binding as B
from . import streaming as S


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, gamma, beta, seg_len, valid_len, eps, out_dtype):
        y, mean, rstd = B.layer_norm_fwd(x, gamma, beta, seg_len, valid_len, eps, out_dtype, want_stats=True)
        ctx.save_for_backward(x, gamma, mean, rstd, valid_len)
        ctx.seg_len = seg_len
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        x, gamma, mean, rstd, valid_len = ctx.saved_tensors
        got = B.layer_norm_bwd(dy.contiguous(), x, mean, rstd, gamma, ctx.seg_len, valid_len, want_params=gamma is not None)
        dx, dgamma, dbeta = got if gamma is not None else (got, None, None)
        return dx, dgamma, dbeta, None, None, None, None


class _Rotary(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, positions, sections, seg_len, valid_len, base, interleaved):
        ctx.save_for_backward(positions, valid_len)
        ctx.args = (sections, seg_len, base, interleaved)
        return B.rotary_fwd(q, k, positions, sections, seg_len, valid_len, base, interleaved)

    @staticmethod
    @once_differentiable
    def backward(ctx, dq, dk=None):
        positions, valid_len = ctx.saved_tensors
        sections, seg_len, base, interleaved = ctx.args
        got = B.rotary_bwd(dq.contiguous(), None if dk is None else dk.contiguous(), positions, sections, seg_len, valid_len, base, interleaved)
        dq, dk = (got, None) if dk is None else got
        return dq, dk, None, None, None, None, None, None


class _HeadNormRotary(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, q_gamma, k_gamma, positions, sections, seg_len, valid_len, base, interleaved, eps):
        ctx.save_for_backward(q, k, q_gamma, k_gamma, positions, valid_len)
        ctx.args = (sections, seg_len, base, interleaved, eps)
        return B.head_norm_rotary_fwd(q, k, q_gamma, k_gamma, positions, sections, seg_len, valid_len, base, interleaved, eps)

    @staticmethod
    @once_differentiable
    def backward(ctx, dq, dk=None):
        q, k, q_gamma, k_gamma, positions, valid_len = ctx.saved_tensors
        sections, seg_len, base, interleaved, eps = ctx.args
        wants = ctx.needs_input_grad[2:4]
        got = B.head_norm_rotary_bwd(dq.contiguous(), None if dk is None else dk.contiguous(), q, k, q_gamma, k_gamma, positions, sections, seg_len, valid_len, base,
                                     interleaved, eps, want_params=any(wants))
        got = got if isinstance(got, tuple) else (got,)
        rows = 1 if k is None else 2
        of = got[:rows] + (None,) * (2 - rows) + got[rows:] + (None,) * 2   # gradients of q, k and the weights that there are
        return *of[:2], *(d if want else None for d, want in zip(of[2:4], wants)), None, None, None, None, None, None, None


class _ScoredAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, seg_len, valid_len, rule):
        out, lse = B.im_scored_attention_fwd(q, k, v, seg_len, valid_len, want_lse=True, **rule)
        # the rule's tensors are saved as the others are: what is written to them before the backward pass raises there
        tensors = {n: t for n, t in rule.items() if isinstance(t, torch.Tensor)}
        ctx.save_for_backward(q, k, v, out, lse, valid_len, *tensors.values())
        ctx.args = (seg_len, {n: t for n, t in rule.items() if n not in tensors}, tuple(tensors))
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        q, k, v, out, lse, valid_len, *tensors = ctx.saved_tensors
        seg_len, rule, names = ctx.args
        return B.im_scored_attention_bwd(dout.contiguous(), q, k, v, out, lse, seg_len, valid_len, **rule, **dict(zip(names, tensors))) + (None, None, None)


def layer_norm(x, gamma, beta, seg_len=None, valid_len=None, eps=1e-5, out_dtype=None):
    """Differentiable layer_norm_fwd (gamma and beta: both tensors, or both None)."""
    if (gamma is None) != (beta is None):
        raise ValueError("gamma and beta: both or none")
    return _LayerNorm.apply(x, gamma, beta, seg_len, valid_len, eps, out_dtype)


def rotary(q, k, positions, sections, seg_len, valid_len=None, base=10000.0, interleaved=False):
    """Differentiable rotary_fwd (k None: q' alone)."""
    return _Rotary.apply(q, k, positions, sections, seg_len, valid_len, base, interleaved)


def head_norm_rotary(q, k, q_gamma=None, k_gamma=None, positions=None, sections=None, seg_len=None, valid_len=None, base=10000.0, interleaved=False, eps=1e-6):
    """Differentiable head_norm_rotary_fwd (k None: q' alone): gradients of q, k and both weights."""
    return _HeadNormRotary.apply(q, k, q_gamma, k_gamma, positions, sections, seg_len, valid_len, base, interleaved, eps)


def im_scored_attention(q, k, v, seg_len, valid_len=None, **rule):
    """Differentiable im_scored_attention_fwd; rule: phase, custom_mask, scale, softcap, slopes, times, documents, causal, prefix (slopes,
    times and prefix are constants: tensors that ask for a gradient are refused, and so is q_len, which has no backward pass)."""
    wants = [n for n, t in rule.items() if isinstance(t, torch.Tensor) and t.requires_grad]
    if wants or rule.get("q_len") is not None:
        raise ValueError(f"no gradient for {', '.join(wants)}" if wants else "q_len: the newest positions alone have no backward pass")
    rule.pop("q_len", None)
    return _ScoredAttention.apply(q, k, v, seg_len, valid_len, rule)


class ImEncoderLayer(torch.nn.Module):
    """A trainable Interlaced-Mask encoder layer, pre-norm with residuals (Eq. 1 with a = MLP o MHSA_2), float residual stream and weights
    of `dtype`:
        h = LN1(x);  q, k, v = h W_qkv^T;  q, k rotated by `positions`;  y1 = x + attention(q, k, v) W_o^T;
        y = y1 + relu(LN2(y1) W_1^T) W_2^T
    sections: pairs of a head that each axis of positions rotates (None: no positions).  qk_norm: heads of q and k are normalised, with weights of
    their own, before they are rotated.  Padded rows of the result are +0, and nothing
    that stands in padded rows of the input reaches the result or a gradient."""

    def __init__(self, d_model, heads, seg_len, d_ff=None, kv_heads=None, sections=None, base=10000.0, dtype=torch.bfloat16, device="cuda", qk_norm=False):
        super().__init__()
        kv_heads = heads if kv_heads is None else kv_heads
        self.heads, self.kv_heads, self.hd, self.seg_len, self.sections, self.base, self.dtype = heads, kv_heads, d_model // heads, tuple(seg_len), sections, base, dtype
        d_ff = 4 * d_model if d_ff is None else d_ff
        shapes = {"w_qkv": ((heads + 2 * kv_heads) * self.hd, d_model), "w_o": (d_model, d_model), "w_1": (d_ff, d_model), "w_2": (d_model, d_ff)}
        for name, (rows, cols) in shapes.items():
            w = torch.empty((rows, cols), device=device)
            torch.nn.init.xavier_uniform_(w)
            setattr(self, name, torch.nn.Parameter(w))   # kept in float, rounded to dtype for the products
        for name in ("ln1", "ln2"):
            setattr(self, name + "_g", torch.nn.Parameter(torch.ones(d_model, device=device)))
            setattr(self, name + "_b", torch.nn.Parameter(torch.zeros(d_model, device=device)))
        self.qk_norm = qk_norm
        if qk_norm:
            self.q_g = torch.nn.Parameter(torch.ones(self.hd, device=device))
            self.k_g = torch.nn.Parameter(torch.ones(self.hd, device=device))
        # of every row its place in its segment, and that segment: on the device once, so that a captured step has nothing to copy
        self.register_buffer("place", torch.cat([torch.arange(n, device=device) for n in self.seg_len]), persistent=False)
        self.register_buffer("segment", torch.cat([torch.full((n,), s, device=device) for s, n in enumerate(self.seg_len)]), persistent=False)

    def project(self, x, valid_len=None, positions=None, seg_len=None):
        """(q, k, v) [B, L, H, hd] of the layer: norm, shared projection, norms of the heads where there are any, rotation."""
        seg_len = self.seg_len if seg_len is None else seg_len
        h = layer_norm(x, self.ln1_g, self.ln1_b, seg_len, valid_len, out_dtype=self.dtype)
        qkv = (h @ self.w_qkv.to(self.dtype).t()).unflatten(-1, (self.heads + 2 * self.kv_heads, self.hd))
        q, k, v = qkv.split((self.heads, self.kv_heads, self.kv_heads), dim=2)
        if self.qk_norm:
            q, k = head_norm_rotary(q, k, self.q_g, self.k_g, positions if self.sections is not None else None, self.sections, seg_len, valid_len, self.base)
        elif self.sections is not None:
            q, k = rotary(q, k, positions, self.sections, seg_len, valid_len, self.base)
        return q, k, v

    def finish(self, x, att, valid_len=None, seg_len=None):
        """What follows the attention: out-projection, residual, MLP."""
        y1 = x + (att @ self.w_o.to(self.dtype).t()).float()
        h = layer_norm(y1, self.ln2_g, self.ln2_b, self.seg_len if seg_len is None else seg_len, valid_len, out_dtype=self.dtype)
        return y1 + (torch.relu(h @ self.w_1.to(self.dtype).t()) @ self.w_2.to(self.dtype).t()).float()

    def forward(self, x, valid_len=None, positions=None, **rule):
        q, k, v = self.project(x, valid_len, positions)
        y = self.finish(x, im_scored_attention(q, k, v, self.seg_len, valid_len, **rule), valid_len)
        if valid_len is None:
            return y
        real = self.place < valid_len[:, self.segment]
        return torch.where(real[:, :, None], y, 0.0)

    def open_cache(self, batch, max_len, held_as="int8", pages=None, times=False):
        """An empty cache for step(): `batch` streams of at most max_len (three numbers) positions a segment, held as "int8" or "e4m3" (see stream_cache)."""
        return S.stream_cache(batch, max_len, self.kv_heads, self.hd, self.dtype, held_as, pages, times, self.place.device)

    @torch.no_grad()
    def step(self, cache, x, seg_len, valid_len=None, positions=None, times=None, ended=None, held=None, **rule):
        """The layer for the newest positions of streams: x float32 [B, L, d] holds seg_len rows of each segment, the first valid_len of them real, which join
        the cache and then attend to all that it holds.  positions int32 [axes, B, L] and times float32 [B, L] are those of these rows; ended int32 [B]:
        streams that begin anew; held int32 [B, 3]: the cache's lengths before a step that is taken again (of 32 rows a segment at most, or one that started from
        nothing); rule: phase, custom_mask, scale, softcap, slopes, causal.  Returns y [B, L, d], padded rows +0, and so are
        those of segments that found no pages or no room in their tables (DEVFLAG_FULL in last_device_status).  Arguments that are refused leave the cache as it was.
        Made for a few rows a segment: a prompt of many is faster by project(), cache_plan, cache_append, im_scored_attention_fwd on its rows, and finish()."""
        q, k, v = self.project(x, valid_len, positions, seg_len)
        att, slots = S.cache_step(cache, q, k, v, seg_len, valid_len, ended, held, times=times, **rule)
        y = self.finish(x, att, valid_len, seg_len)
        return torch.where((slots >= 0)[:, :, None], y, 0.0)
