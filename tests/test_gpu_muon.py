"""The orthogonalised update of a flat vector's matrices against the formulas in 64 bits.

Tolerances. Each of a step's three products is off by about 2^-22 of its norm (both factors keep 22 bits, the sums are fp32), and what one
step leaves is carried on by the steps behind it: relative to X by at most |q'(s) s / q(s)| at the singular values s there are, q the quintic, or
1 where that is less (a disturbance across two singular values grows like X itself). Where all singular values are equal that is a number;
where they are spread, what lies at small ones grows by up to 3.4445 a step while the largest do not."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
A, B, C = 3.4445, -4.7750, 2.0315
EPS = 3 * 2.0 ** -22


@pytest.fixture(scope="module")
def enc():
    import torch
    assert torch.cuda.is_available(), "these tests need the GPU"
    import paper_2304_14698_amd as xrl
    model = dict(n_op_types=4, n_node_dense=0, d_edge=4, d_global=0, hidden=64, rounds=0)
    e = xrl.Encoder(model, np.zeros(xrl.weight_count(model), np.float32))
    yield e
    e.close()


def orthogonalised(U, steps):
    X = U / (math.sqrt((U * U).sum()) + 1e-7)
    turn = X.shape[0] > X.shape[1]
    X = X.T if turn else X
    for _ in range(steps):
        K = X @ X.T
        X = A * X + (B * K + C * K @ K) @ X
    return X.T if turn else X


def step64(W, G, M, matrices, lr, beta, nesterov, wd, steps, rms):
    W, G, M = (v.astype(np.float64) for v in (W, G, M))
    f = lambda v: float(np.float32(v))  # noqa: E731
    lr, beta, wd, rms = f(lr), f(beta), f(wd), f(rms)
    for at, r, c in matrices:
        s = slice(at, at + r * c)
        if r * c == 0:
            continue
        M[s] = beta * M[s] + G[s]
        U = (G[s] + beta * M[s] if nesterov else M[s]).reshape(r, c)
        W[s] = (1 - lr * wd) * W[s] - lr * rms * math.sqrt(max(r, c)) * orthogonalised(U, steps).ravel()
    return W, M


def run(enc, W, G, M, matrices, **kw):
    import torch
    t = [torch.from_numpy(v.copy()).cuda() for v in (W, G, M)]
    enc.muon_step(*t, matrices, **kw)
    torch.cuda.synchronize()
    assert np.array_equal(t[1].cpu().numpy(), G, equal_nan=True)
    return t[0].cpu().numpy(), t[2].cpu().numpy()


def equal_growth(sigma, steps):
    """Sum over the steps of the growth behind each, all singular values at sigma."""
    carried = []
    for _ in range(steps):
        q, dq = A * sigma + B * sigma ** 3 + C * sigma ** 5, A + 3 * B * sigma ** 2 + 5 * C * sigma ** 4
        carried = [c * max(1.0, abs(dq * sigma / q)) for c in carried] + [1.0]
        sigma = q
    return sum(carried)


@pytest.mark.parametrize("rows,cols", [(64, 64), (128, 128), (100, 300), (300, 100), (1, 50), (50, 1), (1, 1), (257, 129), (640, 192)])
@pytest.mark.parametrize("steps", [1, 5])
def test_equal_singular_values(enc, rows, cols, steps):
    rng = np.random.Generator(np.random.PCG64(rows + cols))
    q, _ = np.linalg.qr(rng.standard_normal((max(rows, cols), min(rows, cols))))
    G = np.ascontiguousarray(q.T if rows < cols else q).astype(np.float32).ravel() * np.float32(1e-3)
    W, M = np.zeros_like(G), np.zeros_like(G)
    w, m = run(enc, W, G, M, [(0, rows, cols)], lr=1.0, beta=0.0, nesterov=False, steps=steps, rms=1.0)
    assert np.array_equal(m, G)
    want, _ = step64(W, G, M, [(0, rows, cols)], 1.0, 0.0, False, 0.0, steps, 1.0)
    off = np.linalg.norm(w - want) / np.linalg.norm(want)
    tol = (EPS + 2.0 ** -23) * equal_growth(1 / math.sqrt(min(rows, cols)), steps)
    assert off <= tol, (off, tol)


def spread(rng, rows, cols):
    """A gradient's spectrum: it falls off, over noise."""
    r = max(1, min(rows, cols) // 4)
    fall = np.arange(1, r + 1) ** -0.5
    g = (rng.standard_normal((rows, r)) * fall) @ rng.standard_normal((r, cols)) / math.sqrt(r) + 0.1 * rng.standard_normal((rows, cols))
    return 1e-3 * g


@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("shapes", [[(5, 7)], [(64, 64), (1, 9), (130, 65)], [(44, 64), (64, 64), (136, 64), (64, 256), (256, 64), (64, 1)],
                                    [(513, 256), (256, 1025)], [(3, 700)] * 70, [(700, 700), (0, 5), (33, 31)]])
def test_many_matrices_of_one_vector(enc, shapes, nesterov):
    """Gaps between the matrices (biases) keep their bits; more matrices than one launch's list holds; the order does not matter."""
    rng = np.random.Generator(np.random.PCG64(len(shapes) + shapes[0][0]))
    at, mats, G = 3, [], [np.ones(3)]
    for r, c in shapes:
        mats.append((at, r, c))
        G += [spread(rng, r, c).ravel(), np.ones(5)] if r * c else [np.ones(5)]
        at += r * c + 5
    G = np.concatenate(G).astype(np.float32)
    W = rng.standard_normal(G.size).astype(np.float32)
    M = (rng.standard_normal(G.size) * 1e-3).astype(np.float32)
    kw = dict(lr=0.02, beta=0.95, nesterov=nesterov, weight_decay=0.1, steps=5, rms=0.2)
    w, m = run(enc, W, G, M, mats[::-1], **kw)
    w2, m2 = run(enc, W, G, M, np.array(mats), **kw)
    assert np.array_equal(w, w2) and np.array_equal(m, m2)
    want, mwant = step64(W, G, M, mats, 0.02, 0.95, nesterov, 0.1, 5, 0.2)
    inside = np.zeros(G.size, bool)
    for at, r, c in mats:
        s = slice(at, at + r * c)
        inside[s] = True
        if r * c == 0:
            continue
        # momentum: two roundings; the update: see above; the weights: three roundings
        assert (np.abs(m[s] - mwant[s]) <= 2.0 ** -23 * (np.abs(G[s]) + np.abs(M[s]))).all()
        update = want[s] - (1 - 0.02 * 0.1) * W[s]
        off = np.linalg.norm(w[s] - want[s])
        assert off <= EPS * A ** 5 * np.linalg.norm(update) + 3 * 2.0 ** -24 * np.linalg.norm(W[s]), (r, c, off / np.linalg.norm(update))
    assert np.array_equal(w[~inside], W[~inside]) and np.array_equal(m[~inside], M[~inside])


def test_update_has_the_stated_size_and_is_near_orthogonal(enc):
    """Singular values of X after five steps lie in [0.65, 1.25] where they began above 1 / 100 of the norm."""
    rng = np.random.Generator(np.random.PCG64(3))
    r, c = 96, 320
    G = rng.standard_normal(r * c).astype(np.float32)
    w, _ = run(enc, np.zeros_like(G), G, np.zeros_like(G), [(0, r, c)], lr=1.0, beta=0.0, nesterov=False, rms=1 / math.sqrt(c))
    s = np.linalg.svd(-w.reshape(r, c).astype(np.float64), compute_uv=False)
    assert s.min() > 0.65 and s.max() < 1.25


def test_zero_tiny_huge_and_bad_gradients(enc):
    rng = np.random.Generator(np.random.PCG64(6))
    r, c = 70, 90
    n = r * c
    base = rng.standard_normal(n).astype(np.float32)
    G = np.concatenate([np.zeros(n), base * 1e-6, base * 1e-22, base * 1e25, base, base, base]).astype(np.float32)
    G[4 * n + 17], G[5 * n + 5] = np.nan, np.inf
    W = rng.standard_normal(G.size).astype(np.float32)
    M = np.zeros_like(W)
    mats = [(k * n, r, c) for k in range(7)]
    kw = dict(lr=0.1, beta=0.9, nesterov=True, weight_decay=0.0, steps=5, rms=0.2)
    w, m = run(enc, W, G, M, mats, **kw)
    assert np.array_equal(w[:n], W[:n])                          # no gradient, no update
    for k in (1, 2, 3, 6):                                        # (|U| is summed in 64 bits: 1e25 squared is no infinity)
        s = slice(k * n, k * n + n)
        want, _ = step64(W[s], G[s], M[s], [(0, r, c)], 0.1, 0.9, True, 0.0, 5, 0.2)
        assert np.linalg.norm(w[s] - want) <= EPS * A ** 5 * np.linalg.norm(want - W[s]) + 3 * 2.0 ** -24 * np.linalg.norm(W[s]), k
    assert np.isnan(w[4 * n:6 * n]).all()                         # that matrix, no other


def test_on_an_agents_gradients(enc):
    """The library's own flat layout: all matrices of a model step, biases keep their bits."""
    import torch
    import paper_2304_14698_amd as xrl
    import synth
    model, state = synth.make_config(1)
    rng = np.random.Generator(np.random.PCG64(7))
    w0 = synth.init_weights(rng, xrl.weight_layout(model), bias_range=0.1)
    e = xrl.Encoder(model, w0)
    batch = e.pack(state)
    emb = e.encode(batch, save_for_backward=True)
    e.policy_value(batch, emb)
    ones = lambda n: torch.ones(n, device="cuda")  # noqa: E731
    dw = torch.zeros(e.n_weights, device="cuda")
    e.encode_backward(batch, e.policy_value_backward(batch, emb, ones(batch.G), ones(batch.S), ones(batch.S), dw), dw)
    mats = xrl.weight_matrices(model)
    assert len(mats) == sum(len(s) == 2 for _, s in xrl.weight_layout(model))
    W, M = torch.from_numpy(w0.astype(np.float32)).cuda(), torch.zeros(e.n_weights, device="cuda")
    e.muon_step(W, dw, M, mats, lr=0.02)
    torch.cuda.synchronize()
    g = dw.cpu().numpy()
    want, _ = step64(w0.astype(np.float32), g, np.zeros_like(g), mats.tolist(), 0.02, 0.95, True, 0.0, 5, 0.2)
    got, moved = W.cpu().numpy(), np.zeros(e.n_weights, bool)
    for at, r, c in mats.tolist():
        s = slice(at, at + r * c)
        moved[s] = True
        u = want[s] - w0[s]
        assert np.linalg.norm(got[s] - want[s]) <= EPS * A ** 5 * np.linalg.norm(u) + 3 * 2.0 ** -24 * np.linalg.norm(w0[s])
    assert np.array_equal(got[~moved], w0.astype(np.float32)[~moved])
    batch.free()
    e.close()


def test_nothing_to_do_and_refusals(enc):
    import torch
    import paper_2304_14698_amd as xrl
    v = [torch.ones(100, device="cuda") for _ in range(3)]
    enc.muon_step(*v, [], lr=0.1)
    enc.muon_step(*v, [(100, 0, 7), (0, 5, 0)], lr=0.1)
    for mats, code in (([(0, 10, 11)], "SHAPE"), ([(-1, 2, 2)], "SHAPE"), ([(0, -2, 2)], "SHAPE"), ([(0, 5, 5), (24, 2, 2)], "SHAPE"),
                       ([(50, 5, 5), (30, 5, 5)], "SHAPE"), ([(0, 1, 40000)], "UNSUPPORTED"), ([(2 ** 62, 5, 5)], "SHAPE")):
        with pytest.raises(xrl.XrlError) as ei:
            enc.muon_step(*v, mats, lr=0.1)
        assert ei.value.code == xrl.ERR[code], mats
    for kw in (dict(lr=-1.0), dict(lr=float("nan")), dict(lr=0.1, steps=0), dict(lr=0.1, steps=17), dict(lr=0.1, beta=-0.5),
               dict(lr=0.1, weight_decay=float("inf")), dict(lr=0.1, rms=-1.0)):
        with pytest.raises(xrl.XrlError) as ei:
            enc.muon_step(*v, [(0, 5, 5)], **kw)
        assert ei.value.code == xrl.ERR["VALUE"], kw
    with pytest.raises(ValueError):
        enc.muon_step(v[0], v[1][:50], v[2], [(0, 5, 5)], lr=0.1)
    with pytest.raises(ValueError):
        enc.muon_step(v[0].double(), v[1], v[2], [(0, 5, 5)], lr=0.1)
    torch.cuda.synchronize()
    assert all((x == 1).all() for x in v)
