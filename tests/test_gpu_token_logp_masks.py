"""Masks of torch's own truth values are those of bytes."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def test_masks_of_truth_values():
    import torch
    import paper_2304_14698_amd as xrl
    model = dict(n_op_types=4, n_node_dense=0, d_edge=4, d_global=0, hidden=64, rounds=0)
    enc = xrl.Encoder(model, np.zeros(xrl.weight_count(model), np.float32))
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(6, 90, generator=g, device="cuda")
    wide = torch.rand(6, 100, generator=g, device="cuda") < 0.5
    ids, one = torch.arange(6, dtype=torch.int32, device="cuda"), torch.ones(6, device="cuda")
    ptr = torch.tensor([0, 100, 100, 230, 500, 539, 540], dtype=torch.int32, device="cuda")
    for logits, mask, kw in ((x, wide[:, :90], {}), (x, wide[0, :90], {}), (x.flatten(), wide[:, :90].flatten(), dict(row_ptr=ptr))):
        f, d = [], []
        for m in (mask, mask.to(torch.uint8)):
            f.append(enc.token_logp(logits, ids, mask=m, top_k=3, **kw))
            d.append(enc.token_logp_backward(logits, ids, f[-1], one, one, mask=m, **kw))
        torch.cuda.synchronize()
        assert all(torch.equal(f[0][k], f[1][k]) for k in f[0]) and torch.equal(*d)
    for bad in (x, wide[:, :90].to(torch.int8)):
        with pytest.raises(ValueError):
            enc.token_logp(x, ids, mask=bad)
    enc.close()
