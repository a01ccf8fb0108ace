"""The encoder layer made of the training operators: its gradients against the same layer in 64 bits, and the example that trains one."""
import importlib.util
import math
from pathlib import Path

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def g():
    import paper_2505_01068_b200 as lib
    lib.load()
    return lib


def _plain(layer, x, real, pos, seg, allowed, cap, slopes, times, causal):
    """The layer in float64 on whole rows, closed pairs at minus infinity."""
    w = {n: p.double() for n, p in layer.named_parameters()}
    norm = lambda t, n: torch.nn.functional.layer_norm(t, t.shape[-1:], w[n + "_g"], w[n + "_b"], 1e-5)
    B, L, d = x.shape
    H, K, hd = layer.heads, layer.kv_heads, layer.hd
    qkv = (norm(x, "ln1") @ w["w_qkv"].t()).unflatten(-1, (H + 2 * K, hd))
    q, k, v = qkv.split((H, K, K), dim=2)
    n = hd // 2
    axis = [a for a, m in enumerate(layer.sections) for _ in range(m)]
    angle = torch.stack([pos[axis[p]].double() * 10000.0 ** (-p / n) for p in range(n)], dim=2)[:, :, None]
    turn = lambda t: torch.cat([t[..., :n] * angle.cos() - t[..., n:] * angle.sin(), t[..., :n] * angle.sin() + t[..., n:] * angle.cos()], dim=-1)
    q, k, v = turn(q).transpose(1, 2), turn(k).transpose(1, 2).repeat_interleave(H // K, dim=1), v.transpose(1, 2).repeat_interleave(H // K, dim=1)
    s = q @ k.transpose(2, 3) / math.sqrt(hd)
    s = cap * torch.tanh(s / cap) - slopes.double()[:, None, None] * (times[:, :, None] - times[:, None]).abs()[:, None].double()
    which = torch.repeat_interleave(torch.arange(3), torch.tensor(seg)).cuda()
    ok = torch.tensor(allowed, device="cuda")[which][:, which][None] & real[:, None] & real[:, :, None]
    if causal:
        ok = ok & (times[:, None] <= times[:, :, None])
    some = ok.any(-1)
    p = torch.softmax(torch.where(ok | ~some[:, :, None], s.transpose(0, 1), -math.inf).transpose(0, 1), dim=-1) * some[:, None, :, None]
    y1 = x + (p @ v).transpose(1, 2).reshape(B, L, d) @ w["w_o"].t()
    y = y1 + torch.relu(norm(y1, "ln2") @ w["w_1"].t()) @ w["w_2"].t()
    return torch.where(real[:, :, None], y, 0.0)


@pytest.mark.parametrize("dtype,causal", [("f32", False), ("f32", True), ("bf16", False)])
def test_layer_and_its_gradients(g, dtype, causal):
    """float: within 2e-5 of the norm of each gradient (sums of some thousand products in float); bf16: seven products of rounded operands
    and rounded intermediate results, 2^-9 each, on the way to a gradient: 3e-2."""
    from paper_2505_01068_b200.training import ImEncoderLayer
    torch.manual_seed(3)
    seg, B, d, H, K = (9, 70, 33), 3, 32, 4, 2
    layer = ImEncoderLayer(d, H, seg, d_ff=64, kv_heads=K, sections=(2, 1, 1), dtype=torch.float32 if dtype == "f32" else torch.bfloat16)
    for n, p in layer.named_parameters():
        if n.startswith("ln"):
            p.data += 0.1 * torch.randn_like(p)
        elif dtype == "bf16":
            p.data.copy_(p.data.bfloat16().float())
    valid = torch.tensor([[9, 70, 33], [4, 41, 0], [0, 5, 20]], dtype=torch.int32, device="cuda")
    real = torch.cat([torch.arange(n) for n in seg]).cuda()[None] < torch.repeat_interleave(valid, torch.tensor(seg).cuda(), dim=1)
    x = torch.randn((B, sum(seg), d), device="cuda")
    times = torch.cat([torch.arange(n) * (10.0 / n) for n in seg]).cuda().expand(B, -1).contiguous()
    pos = torch.randint(0, 60, (3, B, sum(seg)), device="cuda", dtype=torch.int32)
    slopes = torch.tensor([0.5, 0.25, 0.125, 0.0625], device="cuda")
    w = torch.randn_like(x) * real[:, :, None]
    allowed = [[False, True, False], [False, False, True], [True, False, False]]

    names = [n for n, _ in layer.named_parameters()]
    xin = torch.where(real[:, :, None], x, float("nan")).requires_grad_()
    y = layer(xin, valid, pos, phase=g.PHASE_INTER_FWD, softcap=10.0, slopes=slopes, times=times, causal=causal)
    got = torch.autograd.grad((y * w).sum(), [xin, *layer.parameters()])
    xr = (x * real[:, :, None]).double().requires_grad_()
    ref = _plain(layer, xr, real, pos, seg, allowed, 10.0, slopes, times, causal)
    want = torch.autograd.grad((ref * w.double()).sum(), [xr, *layer.parameters()])
    tol = 2e-5 if dtype == "f32" else 3e-2
    close = lambda a, b: float((a.detach().double() - b.detach().double()).norm()) <= tol * float(b.detach().double().norm())
    assert close(y, ref) and not torch.signbit(y[~real]).any() and not y[~real].any()
    for n, a, b in zip(["x"] + names, got, want):
        a = torch.where(real[:, :, None], a, 0.0) if n == "x" else a
        assert bool(torch.isfinite(a).all()) and close(a, b), n


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_example_learns_and_streams(g, dtype):
    """The loss falls by more than half in 60 steps; a stream's rows are those of the whole pass to the rounding of two attention kernels
    (bf16: weights and results rounded at 2^-9, values of order one behind two products)."""
    spec = importlib.util.spec_from_file_location("train_encoder", Path(__file__).resolve().parent.parent / "examples" / "train_encoder.py")
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    first, last, off = m.main(["--dtype", dtype, "--steps", "60"])
    assert last < 0.5 * first
    assert off <= (1e-1 if dtype == "bf16" else 1e-4)
    assert g.last_device_status() == (0, 0)


def test_what_has_no_gradient_is_refused_and_what_has_one_gets_it(g):
    from paper_2505_01068_b200 import training as t
    q, k, v = (torch.randn((2, 30, 4, 8), device="cuda", requires_grad=True) for _ in range(3))
    slopes = torch.rand(4, device="cuda", requires_grad=True)
    for rule in (dict(slopes=slopes), dict(q_len=(1, 1, 1))):
        with pytest.raises(ValueError):
            t.im_scored_attention(q, k, v, (8, 12, 10), **rule)
    with pytest.raises(ValueError):
        t.layer_norm(q.flatten(2), torch.ones(32, device="cuda"), None)
    out = t.im_scored_attention(q, k, v, (8, 12, 10), slopes=slopes.detach(), q_len=None)
    grads = torch.autograd.grad(out.square().sum(), (q, k, v), create_graph=True)
    with pytest.raises(RuntimeError):   # once differentiable
        grads[0].sum().backward()
    pos = torch.arange(30, device="cuda", dtype=torch.int32)[None]
    w = torch.randn_like(q)
    alone, = torch.autograd.grad((t.rotary(q, None, pos, (4,), (8, 12, 10)) * w).sum(), q)
    both = torch.autograd.grad(sum((x * w).sum() for x in t.rotary(q, k, pos, (4,), (8, 12, 10))), (q, k))
    assert torch.equal(alone, both[0]) and torch.equal(both[0], both[1])
    plain, = torch.autograd.grad(t.layer_norm(q.flatten(2), None, None).square().sum() + (q * w).sum(), q)
    assert bool(torch.isfinite(plain).all())
