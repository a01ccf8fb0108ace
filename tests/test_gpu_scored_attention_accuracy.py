"""How many bits the gradients of bf16 attention keep: next to a result's own rounding, one rounding of a product's operand and no more,
also where rows see a handful of keys."""
import pytest
import torch

from test_gpu_scored_attention import Problem

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def g():
    import paper_2505_01068_b200 as lib
    lib.load()
    return lib


# dtype, batch, segments, heads, key heads, head_dim, phase, rule.  Heads of 64 on either side of the line between the kernels.
CASES = [(6, (50, 300, 300), 8, 8, 8, "fwd", dict(cap=30.0, slopes=True, times="seconds")), (6, (39, 55, 300), 4, 4, 8, "intra", dict(causal=True, docs=-8)),
         (6, (39, 55, 300), 8, 4, 16, "intra", dict(causal=True, docs=-8, cap=20.0)), (6, (39, 55, 400), 4, 2, 32, "intra", dict(causal=True, docs=-20)),
         (4, (50, 300, 300), 4, 4, 32, "all", dict()), (4, (130, 300, 257), 2, 2, 64, "intra", dict(causal=True, docs=-20)),
         (4, (130, 300, 257), 2, 1, 64, "fwd", dict(cap=30.0)), (8, (70, 41, 60), 2, 2, 64, "intra", dict(causal=True, docs=-12)),
         (8, (30, 20, 25), 4, 4, 16, "fwd", dict(slopes=True))]


@pytest.mark.parametrize("case", CASES, ids=str)
def test_gradients_keep_their_bits(g, case):
    """Norms of errors against 64 bits, in units of the error that rounding the exact result to bf16 makes (which is measured).  One operand of
    the last product is rounded to bf16, too: for independent terms that error is as large again, so sqrt(2) together; terms that cancel
    in a sum make it somewhat larger, 1.6 at the most.  A row's delta from a result that was rounded would add a third one, 1.6 to 2 where rows
    see few keys."""
    B, seg, H, HK, hd, phase, rule = case
    p = Problem("bf16", B, seg, H, HK, hd, phase, padded=False, seed=hd, **rule)
    out, lse = p.forward(g)
    want = p.exact()
    for what, got, ref in zip(("out", "dq", "dk", "dv"), (out,) + p.backward(g, out, lse), (want[0],) + want[2:]):
        own = float((ref.bfloat16().double() - ref).norm())
        err = float((got.double() - ref).norm())
        print(what, round(err / own, 3))
        assert err <= 1.6 * own, (what, err / own)
