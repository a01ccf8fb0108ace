"""Rotary positions, LayerNorm and scored attention behind a kernel that lets its successor start at once and writes the call's inputs late:
nothing may be read before it has ended, by any of the kernels that serve these calls, the second and third of a backward pass included."""
import numpy as np
import pytest
import torch

from test_gpu_stream_order import Late, SEG

pytestmark = pytest.mark.gpu
L = sum(SEG)


@pytest.fixture(scope="module")
def g():
    import paper_2505_01068_b200 as lib
    lib.load()
    return lib


def _lengths(B, seed):
    rng = np.random.default_rng(seed)
    return torch.from_numpy(np.stack([rng.integers(1, n + 1, size=B) for n in SEG], axis=1).astype(np.int32)).cuda()


def _randn(shape, dtype, seed):
    return torch.randn(shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).to(dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B", [2, 60])
def test_rotary(g, dtype, B):
    x, pos = _randn((B, L, 4, 16), dtype, 0), torch.arange(B * L, device="cuda", dtype=torch.int32).view(1, B, L) % 97
    late = Late(g, [x, pos, _lengths(B, B)])
    xl, pl, vl = late.views
    late.check(lambda: [g.rotary_fwd(xl, xl, pl, (8,), SEG, vl)[0], g.rotary_bwd(xl, xl, pl, (8,), SEG, vl)[1]])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,d", [(2, 32), (60, 512)])
def test_layer_norm(g, dtype, B, d):
    x, dy, gamma, beta = _randn((B, L, d), dtype, 1), _randn((B, L, d), dtype, 2), _randn((d,), torch.float32, 3), _randn((d,), torch.float32, 4)
    late = Late(g, [x, dy, gamma, beta, _lengths(B, B)])
    xl, dl, gl, bl, vl = late.views

    def call():
        y, mean, rstd = g.layer_norm_fwd(xl, gl, bl, SEG, vl, want_stats=True)
        return [y, *g.layer_norm_bwd(dl, xl, mean, rstd, gl, SEG, vl)]
    late.check(call)


@pytest.mark.parametrize("dtype,hd,seg_rule", [(torch.bfloat16, 8, True), (torch.bfloat16, 32, False), (torch.bfloat16, 64, True), (torch.bfloat16, 64, False),
                                               (torch.float32, 16, True), (torch.float32, 96, False)])
def test_scored_attention(g, dtype, hd, seg_rule):
    B, H, HK = 6, 4, 2
    q, k, v, dout = _randn((B, L, H, hd), dtype, 1), _randn((B, L, HK, hd), dtype, 2), _randn((B, L, HK, hd), dtype, 3), _randn((B, L, H * hd), dtype, 4)
    times = torch.arange(L, device="cuda", dtype=torch.float32).repeat(B, 1)
    docs = torch.arange(L, device="cuda", dtype=torch.int32).div(40, rounding_mode="floor").int().repeat(B, 1)
    late = Late(g, [q, k, v, dout, torch.tensor([0.5, 0.25, 0.125, 0.0625], device="cuda"), times, docs, torch.full((B,), 5.0, device="cuda"), _lengths(B, 9)])
    ql, kl, vl, dl, slopes, times, docs, prefix, valid = late.views
    rule = dict(phase=g.PHASE_CUSTOM, custom_mask=0x1ff, softcap=20.0)
    if seg_rule:
        rule |= dict(slopes=slopes, times=times, documents=docs, causal=True, prefix=prefix)

    def call():
        out, lse = g.im_scored_attention_fwd(ql, kl, vl, SEG, valid, want_lse=True, **rule)
        return [out, lse, *g.im_scored_attention_bwd(dl, ql, kl, vl, out, lse, SEG, valid, **rule)]
    late.check(call)


@pytest.mark.parametrize("dtype,hd", [(torch.bfloat16, 8), (torch.bfloat16, 64), (torch.float32, 24)])
def test_newest_positions(g, dtype, hd):
    B, H, HK = 6, 4, 2
    q, k, v = _randn((B, 3, H, hd), dtype, 1), _randn((B, L, HK, hd), dtype, 2), _randn((B, L, HK, hd), dtype, 3)
    late = Late(g, [q, k, v, _lengths(B, 9)])
    ql, kl, vl, valid = late.views
    late.check(lambda: g.im_scored_attention_fwd(ql, kl, vl, SEG, valid, g.PHASE_CUSTOM, 0x1ff, softcap=20.0, causal=True, q_len=(1, 1, 1), want_lse=True))
