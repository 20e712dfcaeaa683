"""The orthogonalised update does not depend on the gradient's size: by powers of two, to the bit, up to the largest that fp32 has."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,cols", [(40, 60), (400, 60), (70, 90), (300, 1100)])
def test_gradients_of_any_size(rows, cols):
    import torch
    import paper_2304_14698_amd as xrl
    model = dict(n_op_types=4, n_node_dense=0, d_edge=4, d_global=0, hidden=64, rounds=0)
    enc = xrl.Encoder(model, np.zeros(xrl.weight_count(model), np.float32))
    g = torch.Generator(device="cuda").manual_seed(rows)
    base = torch.randn(rows * cols, generator=g, device="cuda").clamp_(-3.9, 3.9)
    W = []
    for power in (40, 60, 100, 120, 126):        # (from 2^40 on the 1e-7 that is added to |U| is nothing beside it)
        w, m = torch.zeros_like(base), torch.zeros_like(base)
        enc.muon_step(w, base * 2.0 ** power, m, [(0, rows, cols)], lr=1.0, beta=0.0, nesterov=False, rms=1.0)
        W.append(w)
    torch.cuda.synchronize()
    assert W[0].abs().max() > 0 and torch.isfinite(W[0]).all()
    for w in W[1:]:
        assert torch.equal(w, W[0])
    enc.close()
