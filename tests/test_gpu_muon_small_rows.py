"""The orthogonalised update where rows differ in size: an update turns every row alike, so a row of small size (a unit that is rarely active) has to be
as right as a large one.

Tolerances. Each factor of a product keeps 22 bits, where a product in fp32 keeps 24, and the sums are fp32 in both: a row is off by at most about
four times what the same steps in fp32 products are off by, and by twice that as both errors are the worst of many rows, each of them once by chance.
Rows from 1e-7 of the largest on lie at 2^-31 of the matrix's norm here, where two halves leave 2^-48 / 2^-31 = 2^-17 of an entry: within it."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
A, B, C = 3.4445, -4.7750, 2.0315


@pytest.fixture(scope="module")
def enc():
    import torch
    assert torch.cuda.is_available(), "these tests need the GPU"
    import paper_2304_14698_amd as xrl
    model = dict(n_op_types=4, n_node_dense=0, d_edge=4, d_global=0, hidden=64, rounds=0)
    e = xrl.Encoder(model, np.zeros(xrl.weight_count(model), np.float32))
    yield e
    e.close()


def orthogonalised(U, steps=5):
    """U m x n with m <= n, in its own type."""
    f = U.dtype.type
    X = U * f(1.0 / (math.sqrt((U.astype(np.float64) ** 2).sum()) + 1e-7))
    for _ in range(steps):
        K = X @ X.T
        X = f(A) * X + (f(B) * K + f(C) * (K @ K)) @ X
    return X


@pytest.mark.parametrize("fall", [3, 5, 6, 7])
@pytest.mark.parametrize("m,n", [(256, 512), (64, 256), (64, 512), (200, 333), (128, 4000), (1100, 1300)])
@pytest.mark.parametrize("turned", [False, True])
def test_rows_of_small_size(enc, m, n, fall, turned):
    import torch
    rng = np.random.Generator(np.random.PCG64(m + n + fall))
    U = (rng.standard_normal((m, n)) * np.logspace(0, -fall, m)[rng.permutation(m)][:, None]).astype(np.float32)
    G = torch.from_numpy(np.ascontiguousarray(U.T if turned else U).ravel()).cuda()
    W, M = torch.zeros_like(G), torch.zeros_like(G)
    rows, cols = (n, m) if turned else (m, n)
    enc.muon_step(W, G, M, [(0, rows, cols)], lr=1.0, beta=0.0, nesterov=False, rms=1.0)
    torch.cuda.synchronize()
    got = -W.cpu().numpy().reshape(rows, cols).astype(np.float64) / math.sqrt(n)
    got = got.T if turned else got
    want, plain = orthogonalised(U.astype(np.float64)), orthogonalised(U).astype(np.float64)
    off = lambda x: np.linalg.norm(x - want, axis=1) / np.linalg.norm(want, axis=1)  # noqa: E731
    assert off(got).max() <= 8 * off(plain).max(), (off(got).max(), off(plain).max())
