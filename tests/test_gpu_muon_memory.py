"""The workspace of an update of many large matrices is that of a few: they are not all worked on at once."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def test_workspace_of_many_large_matrices():
    import torch
    import paper_2304_14698_amd as xrl
    model = dict(n_op_types=4, n_node_dense=0, d_edge=4, d_global=0, hidden=64, rounds=0)
    enc = xrl.Encoder(model, np.zeros(xrl.weight_count(model), np.float32))
    shapes = [(4096, 6144)] * 20 + [(100, 70), (64, 300)]
    mats, at = [], 0
    for r, c in shapes:
        mats.append((at, r, c))
        at += r * c
    g = torch.Generator(device="cuda").manual_seed(1)
    G = torch.randn(at, generator=g, device="cuda")
    W, M = torch.zeros_like(G), torch.zeros_like(G)
    w, m = torch.zeros_like(G), torch.zeros_like(G)
    torch.cuda.synchronize()
    free = torch.cuda.mem_get_info()[0]
    enc.muon_step(W, G, M, mats, lr=0.02, steps=2)
    torch.cuda.synchronize()
    assert free - torch.cuda.mem_get_info()[0] < 3 << 30         # 8.6 GB for all twenty
    for one in mats[:20]:
        enc.muon_step(w, G, m, [one], lr=0.02, steps=2)
    enc.muon_step(w, G, m, mats[20:], lr=0.02, steps=2)
    torch.cuda.synchronize()
    large = slice(0, mats[20][0])
    assert torch.equal(M, m) and torch.equal(W[large], w[large])   # the same tiles, each with its whole sum
    assert float((W - w).abs().max()) <= 1e-5 * float(w.abs().max())
    enc.close()
