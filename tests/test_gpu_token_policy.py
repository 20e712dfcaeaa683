"""The example that runs the operators over a vocabulary together: its gradients against torch's own of the same objective in 64
bits, and that it learns."""
import os
import sys

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_gradients_of_one_step():
    """fp32 products and sums of a few hundred terms: off by less than 1e-5 of the gradient's norm."""
    import torch
    import token_policy as T
    p = T.TokenPolicy(rules=50, length=4, dim=32, hidden=64, seed=1)
    history, taken = T.histories(np.random.Generator(np.random.PCG64(3)), 200, 50, 4)
    w = [v.double().clone().requires_grad_() for v in p.views(p.weights)]
    table = p.table.double().clone().requires_grad_()
    place = torch.arange(4, device="cuda") * 50
    at = (history.long() + place).clamp(min=0)
    rows = table[at] * (history >= 0)[..., None] * 32 ** 0.5
    lp = torch.log_softmax(torch.relu(rows.sum(1) @ w[0]) @ w[1], 1)
    J = -(lp.gather(1, taken.long()[:, None]).mean() + 0.001 * -(lp.exp() * lp).sum(1).mean())
    J.backward()
    before = p.table.clone()
    got, _ = p.step(history, taken)
    torch.cuda.synchronize()
    assert abs(float(got) - J.item()) < 1e-5 * abs(J.item())
    for g, v in zip(p.views(p.grads), w):
        assert float((g.double() - v.grad).norm()) < 1e-5 * float(v.grad.norm())
    assert float((p.dtable.double() - table.grad).norm()) < 1e-5 * float(table.grad.norm())
    assert torch.equal(p.table, before.sub(p.dtable, alpha=0.5))


def test_it_learns():
    import token_policy as T
    record = T.main(steps=80, verbose=False)
    assert record[-1][0] < 0.2 * record[0][0] and record[-1][1] > 0.95
