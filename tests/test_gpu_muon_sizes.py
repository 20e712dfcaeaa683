"""The orthogonalised update in every way that sizes choose: one block a matrix of eight or of sixteen waves, tiles of 64 x 64 with sums whole and cut, tiles of
128 x 128, and the sizes at which these change.

Tolerance. Each factor of a product keeps 22 bits where fp32 products keep 24, and both add up in fp32: the update is at most four times as far from 64 bits as
the same steps in fp32 products are, and by the weights' rounding besides (3 of them, of 2^-24)."""
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


def orthogonalised(u, steps):
    import torch
    x = u / (torch.linalg.vector_norm(u.double()) + 1e-7).to(u.dtype)
    x = x.T.contiguous() if u.shape[0] > u.shape[1] else x
    for _ in range(steps):
        k = x @ x.T.contiguous()
        x = A * x + (B * k + C * (k @ k)) @ x
    return x.T if u.shape[0] > u.shape[1] else x


def waves(rows, cols, seed):
    """A matrix whose singular values are all one, dense: cosines, which are orthogonal, with signs."""
    import torch
    n, m = max(rows, cols), min(rows, cols)
    i, j = torch.arange(m, device="cuda", dtype=torch.float64)[:, None], torch.arange(n, device="cuda", dtype=torch.float64)
    q = math.sqrt(2.0 / n) * torch.cos(math.pi / n * i * (j + 0.5))
    q[0] *= math.sqrt(0.5)
    q = q * (torch.rand(n, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda") < 0.5).mul(2).sub(1)
    return q.T.contiguous() if rows > cols else q


def spread(rows, cols, seed):
    """A gradient's spectrum: it falls off, over noise."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda", dtype=torch.float64)  # noqa: E731
    r = max(1, min(rows, cols) // 4)
    return (randn(rows, r) * torch.arange(1, r + 1, device="cuda") ** -0.5) @ randn(r, cols) / math.sqrt(r) + 0.1 * randn(rows, cols)


def check(enc, shapes, make, steps=5):
    import torch
    mats, at, parts = [], 0, []
    for k, (r, c) in enumerate(shapes):
        mats.append((at, r, c))
        parts.append((1e-3 * make(r, c, 7 * k + r + c)).float().flatten())
        at += r * c
    G = torch.cat(parts)
    W, M = torch.zeros_like(G), torch.zeros_like(G)
    enc.muon_step(W, G, M, mats, lr=1.0, beta=0.0, nesterov=False, steps=steps, rms=1.0)
    torch.cuda.synchronize()
    assert torch.equal(M, G)
    for o, r, c in mats:
        u = G[o:o + r * c].view(r, c)
        want = -math.sqrt(max(r, c)) * orthogonalised(u.double(), steps)
        plain = -math.sqrt(max(r, c)) * orthogonalised(u, steps).double()
        off = float((W[o:o + r * c].view(r, c).double() - want).norm() / want.norm())
        limit = 4 * float((plain - want).norm() / want.norm()) + 3 * 2.0 ** -24
        assert off <= limit, (r, c, off, limit)


@pytest.mark.parametrize("steps", [1, 5])
@pytest.mark.parametrize("make", [waves, spread])
@pytest.mark.parametrize("shapes", [[(64, 256)], [(256, 64)], [(64, 257)], [(257, 64)], [(64, 512)], [(512, 64)], [(33, 257)], [(300, 5)], [(257, 2)], [(2, 512)],
                                    [(65, 512)], [(64, 513)], [(513, 64)], [(512, 65)], [(40, 500), (480, 17), (64, 64), (3, 260), (511, 63)],
                                    [(64, 480)] * 33])
def test_one_block_a_matrix(enc, shapes, make, steps):
    check(enc, shapes, make, steps)


@pytest.mark.parametrize("make", [waves, spread])
@pytest.mark.parametrize("shapes", [[(89, 2859)], [(2859, 89)], [(2, 2342)], [(128, 6000)], [(300, 300), (1100, 700)], [(2960, 2990)], [(2990, 2960)], [(2049, 2100)],
                                    [(2000, 4100), (70, 3001)], [(128, 4096), (4096, 2050)]])
def test_tiles_of_both_sizes_and_cut_sums(enc, shapes, make):
    check(enc, shapes, make)


@pytest.mark.parametrize("rows,cols", [(64, 512), (400, 33), (64, 256)])
def test_bad_gradients_stay_in_their_matrix(enc, rows, cols):
    """As one block a matrix: NaN and infinity reach all of theirs and nothing of the next."""
    import torch
    n = rows * cols
    g = torch.Generator(device="cuda").manual_seed(n)
    G = torch.randn(4 * n, generator=g, device="cuda")
    G[n:2 * n] = 0
    good = G.clone()
    G[17], G[3 * n - 5] = math.nan, math.inf
    mats = [(k * n, rows, cols) for k in range(4)]
    out = []
    for v in (G, good):
        W, M = torch.ones_like(G), torch.zeros_like(G)
        enc.muon_step(W, v, M, mats, lr=0.1, rms=0.2)
        out.append(W)
    torch.cuda.synchronize()
    bad, fine = out
    assert torch.isnan(bad[:n]).all() and torch.isnan(bad[2 * n:3 * n]).all()
    assert (bad[n:2 * n] == 1).all()
    assert torch.equal(bad[3 * n:], fine[3 * n:]) and torch.isfinite(fine).all()


@pytest.mark.parametrize("rows,cols", [(1, 512), (257, 1), (1, 300), (1, 1), (400, 1), (1, 2342)])
def test_a_single_row(enc, rows, cols):
    """U / |U| and its one singular value through the quintic: six roundings a step, carried on by its slope, at most 3.4445 a step where the value is small and
    below 2 from one on."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(rows + cols)
    G = torch.randn(rows * cols, generator=g, device="cuda")
    W, M = torch.zeros_like(G), torch.zeros_like(G)
    enc.muon_step(W, G, M, [(0, rows, cols)], lr=1.0, beta=0.0, nesterov=False, rms=1.0)
    torch.cuda.synchronize()
    want = -math.sqrt(max(rows, cols)) * orthogonalised(G.double().view(rows, cols), 5).flatten()
    assert float((W.double() - want).norm() / want.norm()) <= 5 * 6 * 2.0 ** -22 * 2 ** 5
