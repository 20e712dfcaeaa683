"""Log-probabilities below fp32's lowest value: the given entry's is that value, as -inf says that it may not be chosen; an alternative's is -inf, as its
index says whether it is there."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cols", [5, 3000, 20000])
def test_alternatives_below_the_lowest_value(cols):
    import torch
    import paper_2304_14698_amd as xrl
    model = dict(n_op_types=4, n_node_dense=0, d_edge=4, d_global=0, hidden=64, rounds=0)
    enc = xrl.Encoder(model, np.zeros(xrl.weight_count(model), np.float32))
    low = torch.finfo(torch.float32).min
    x = torch.full((2, cols), -math.inf, device="cuda")
    x[:, 0], x[:, cols - 1] = -low, low                          # two entries that may be chosen, 6.8e38 apart
    ids = torch.tensor([cols - 1, 1], dtype=torch.int32, device="cuda")
    f = enc.token_logp(x, ids, top_k=3)
    torch.cuda.synchronize()
    assert f["logp"].tolist() == [low, -math.inf]
    assert f["top_ids"].tolist() == [[0, cols - 1, -1]] * 2
    assert f["top_logp"].tolist() == [[0.0, -math.inf, -math.inf]] * 2
    enc.close()
