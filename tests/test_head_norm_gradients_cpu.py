"""Which gradients the differentiable head norm asks for, with the library's calls replaced by torch on the CPU."""
import pytest
import torch

import paper_2505_01068_b200 as g
from paper_2505_01068_b200 import training


@pytest.fixture
def asked(monkeypatch):
    """want_params of every backward call; gradients that tell their places apart."""
    calls = []

    def fwd(q, k, *rest):
        return q * 1.0 if k is None else (q * 1.0, k * 1.0)

    def bwd(dq, dk, q, k, *rest, want_params=True):
        calls.append(want_params)
        rows = (dq * 2,) if k is None else (dq * 2, dk * 3)
        weights = (torch.full((4,), 5.0), torch.full((4,), 7.0))[:len(rows)] if want_params else ()
        return rows + weights if len(rows + weights) > 1 else rows[0]

    monkeypatch.setattr(g.binding, "head_norm_rotary_fwd", fwd)
    monkeypatch.setattr(g.binding, "head_norm_rotary_bwd", bwd)
    return calls


@pytest.mark.parametrize("alone", [False, True])
@pytest.mark.parametrize("q_weight, k_weight", [(None, None), (False, False), (True, None), (None, True), (True, False), (True, True)])
def test_gradients_that_nobody_wants_are_not_asked_for(asked, q_weight, k_weight, alone):
    """None: no weight; False: one that asks for no gradient."""
    q, k = (torch.ones((1, 2, 1, 4), requires_grad=True) for _ in range(2))
    k = None if alone else k
    weight = lambda w: None if w is None else torch.ones(4, requires_grad=w)
    qg, kg = weight(q_weight), None if alone else weight(k_weight)
    out = training.head_norm_rotary(q, k, qg, kg)
    (out if alone else out[0] + out[1]).sum().backward()
    assert asked == [bool(q_weight) or bool(k_weight and not alone)]
    assert torch.equal(q.grad, torch.full_like(q, 2.0)) and (alone or torch.equal(k.grad, torch.full_like(k, 3.0)))
    assert qg is None or (qg.grad is None) != q_weight and (not q_weight or torch.equal(qg.grad, torch.full((4,), 5.0)))
    assert kg is None or (kg.grad is None) != k_weight and (not k_weight or torch.equal(kg.grad, torch.full((4,), 7.0)))
