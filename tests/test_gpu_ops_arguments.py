"""Workspaces that a caller hands to the training operators: host memory and gaps are refused, what is large enough is used."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def g():
    import paper_2505_01068_b200 as lib
    lib.load()
    return lib


def _bytes(n, device="cuda"):
    return torch.empty(n, dtype=torch.uint8, device=device)


def test_layer_norm(g):
    x = torch.randn((2, 30, 32), device="cuda")
    _, mean, rstd = g.layer_norm_fwd(x, want_stats=True)
    want = g.layer_norm_bwd(x, x, mean, rstd)
    for bad in (_bytes(1 << 20, "cpu"), _bytes(1 << 21)[::2]):
        with pytest.raises(AssertionError, match="workspace"):
            g.layer_norm_bwd(x, x, mean, rstd, workspace=bad)
    assert all(torch.equal(a, b) for a, b in zip(want, g.layer_norm_bwd(x, x, mean, rstd, workspace=_bytes(1 << 20))))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_scored_attention(g, dtype):
    q, k, v = (torch.randn((2, 30, 4, 16), device="cuda").to(dtype) for _ in range(3))
    seg = (8, 12, 10)
    out, lse = g.im_scored_attention_fwd(q, k, v, seg, want_lse=True)
    want = g.im_scored_attention_bwd(out, q, k, v, out, lse, seg)
    for bad in (_bytes(1 << 20, "cpu"), _bytes(1 << 21)[::2]):
        with pytest.raises(AssertionError, match="workspace"):
            g.im_scored_attention_bwd(out, q, k, v, out, lse, seg, workspace=bad)
    assert all(torch.equal(a, b) for a, b in zip(want, g.im_scored_attention_bwd(out, q, k, v, out, lse, seg, workspace=_bytes(1 << 20))))
