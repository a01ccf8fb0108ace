"""The differentiable operators as a training program uses them: tensors that are written to between the passes, steps that are captured."""
import pytest
import torch

pytestmark = pytest.mark.gpu

SEG = (8, 40, 30)


@pytest.fixture(scope="module")
def g():
    import paper_2505_01068_b200 as lib
    lib.load()
    return lib


def _rule(name):
    rule = dict(slopes=torch.tensor([0.5, 0.25, 0.125, 0.0625], device="cuda"), times=torch.rand((2, 78), device="cuda"),
                documents=torch.randint(0, 3, (2, 78), device="cuda", dtype=torch.int32), causal=True, prefix=torch.rand(2, device="cuda"), softcap=10.0)
    return rule if name is None else {n: v for n, v in rule.items() if n == name or (name == "prefix" and n == "causal")}


@pytest.mark.parametrize("name", ["slopes", "times", "documents", "prefix"])
def test_a_rule_that_is_written_to_before_the_backward_pass_raises(g, name):
    """As any tensor that autograd saved: the gradients would be those of another rule."""
    from paper_2505_01068_b200 import training as t
    torch.manual_seed(0)
    q, k, v = (torch.randn((2, 78, 4, 16), device="cuda", requires_grad=True) for _ in range(3))
    rule = _rule(name)
    out = t.im_scored_attention(q, k, v, SEG, **rule)
    rule[name].add_(1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        out.sum().backward()


def test_saved_tensor_hooks_see_the_rule(g):
    from paper_2505_01068_b200 import training as t
    torch.manual_seed(1)
    q, k, v = (torch.randn((2, 78, 4, 16), device="cuda", requires_grad=True) for _ in range(3))
    rule, seen = _rule(None), []

    def pack(x):
        seen.append(x.data_ptr())
        return x.cpu()
    want = torch.autograd.grad(t.im_scored_attention(q, k, v, SEG, **rule).square().sum(), (q, k, v))
    with torch.autograd.graph.saved_tensors_hooks(pack, lambda x: x.cuda()):
        out = t.im_scored_attention(q, k, v, SEG, **rule)
    assert {rule[n].data_ptr() for n in ("slopes", "times", "documents", "prefix")} <= set(seen)
    assert all(torch.equal(a, b) for a, b in zip(want, torch.autograd.grad(out.square().sum(), (q, k, v))))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_a_layers_step_is_captured(g, dtype):
    """Forward and backward pass in a CUDA graph, with lengths that change from replay to replay: the bits of plain calls."""
    from paper_2505_01068_b200.training import ImEncoderLayer
    torch.manual_seed(2)
    layer = ImEncoderLayer(32, 4, SEG, sections=(2, 1, 1), dtype=dtype)
    assert not any("place" in n or "segment" in n for n in layer.state_dict())
    x, w = (torch.randn((3, 78, 32), device="cuda") for _ in range(2))
    pos = torch.randint(0, 50, (3, 3, 78), device="cuda", dtype=torch.int32)
    lengths = [torch.tensor(n, dtype=torch.int32, device="cuda") for n in ([[8, 40, 30], [3, 20, 0], [0, 1, 30]], [[1, 2, 3], [8, 40, 30], [5, 0, 29]])]
    valid = lengths[0].clone()
    x.requires_grad_()

    def step():
        y = layer(x, valid, pos, phase=g.PHASE_INTER_FWD, softcap=10.0)
        return [y.detach()] + list(torch.autograd.grad((y * w).sum(), [x, *layer.parameters()]))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(3):
            step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for n in (1, 0, 1):
        valid.copy_(lengths[n])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, step())), n
    assert g.last_device_status() == (0, 0)
