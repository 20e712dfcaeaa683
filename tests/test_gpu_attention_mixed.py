"""Attention over many short sequences, where a tile holds rows of several: empty sequences among them, other numbers of keys than of queries, rows of no sequence, and what is
not finite beside a sequence's own rows. Oracle and tolerances: attention_checks.py."""
import math

import numpy as np
import pytest

from test_gpu_attention_packed import check, enc, ptr, tensors  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("type", ["fp32", "bf16"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("empty", [0, 3, 70, 200])
@pytest.mark.parametrize("dim", [32, 40, 128])
def test_empty_sequences_among_short_ones(enc, type, causal, empty, dim):  # noqa: F811
    r = np.random.default_rng(empty + dim)
    nq, nk = [], []
    for _ in range(12 if empty < 10 else 3):
        nq += [int(r.integers(1, 30))] + [0] * empty
        nk += [int(r.integers(0, 30))] + list(r.integers(0, 2, empty))
    q, k, v, d = tensors(empty, sum(nq), sum(nk), 4, 2, dim, type)
    check(enc, q, k, v, d, ptr(nq), ptr(nk), causal)
    check(enc, q, k, v, d, ptr(nq), ptr([min(n, int(m)) for n, m in zip(nq, nk)]), causal)   # fewer keys than there are rows of them


@pytest.mark.parametrize("type", ["fp32", "bf16"])
@pytest.mark.parametrize("front,back", [(0, 40), (37, 0), (64, 33)])
def test_rows_in_front_and_behind(enc, type, front, back):  # noqa: F811
    """Rows of no sequence hold NaN: they reach nothing, and their results are left as they were."""
    import torch
    lengths = [5, 1, 0, 31, 9, 2]
    n = front + sum(lengths) + back
    q, k, v, d = tensors(3, n, n, 2, 1, 32, type)
    for x in (q, k, v, d):
        x[:front] = math.nan
        x[n - back:] = math.nan
    new = lambda x: torch.full_like(x, 7.0)  # noqa: E731
    out = dict(out=new(q), lse=torch.full((n, 2), 7.0, device="cuda"))
    p = ptr(lengths, front)
    got = check(enc, q, k, v, d, p, None, True, out=out, grads=[new(q), new(k), new(v)])
    for name, x in got.items():
        assert (x[:front] == 7.0).all() and (x[n - back:] == 7.0).all(), name


@pytest.mark.parametrize("type", ["fp32", "bf16"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("what", [math.nan, math.inf, -math.inf])
def test_neighbours_that_are_not_finite(enc, type, causal, what):  # noqa: F811
    """A whole sequence of NaN or infinities between others: their results have the same bits as without it."""
    import torch
    nq, nk = [3, 7, 2, 11, 9], [5, 7, 4, 2, 20]
    (qp, tq), (kp, tk) = ptr(nq), ptr(nk)
    clean = tensors(8, sum(nq), sum(nk), 4, 2, 32, type)
    bad = [x.clone() for x in clean]
    for x, p in zip(bad, (qp, kp, kp, qp)):
        x[p[2]:p[3]] = what
    res = []
    for t in (clean, bad):
        f = enc.attention(*t[:3], tq, k_ptr=tk, causal=causal)
        res.append([f["out"], f["lse"], *enc.attention_backward(*t[:3], tq, f, t[3], k_ptr=tk, causal=causal)])
    torch.cuda.synchronize()
    for a, b, p in zip(*res, (qp, qp, qp, kp, kp)):
        assert torch.equal(a[:p[2]], b[:p[2]]) and torch.equal(a[p[3]:], b[p[3]:])


@pytest.mark.parametrize("type", ["fp32", "bf16"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("far", ["keys", "queries"])
def test_long_sequences_without_the_other_side(enc, type, causal, far):  # noqa: F811
    """Keys that no query has, or queries without keys, lie between the rows of a tile, whole tiles of them."""
    few, many = [3, 0, 2] * 8, [4, 300, 6] * 8
    nq, nk = (few, many) if far == "keys" else (many, few)
    q, k, v, d = tensors(9, sum(nq), sum(nk), 4, 2, 32, type)
    check(enc, q, k, v, d, ptr(nq), ptr(nk), causal)
