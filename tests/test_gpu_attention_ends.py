"""Packed attention where ends of sequences fall or lie outside the tensors: everything that is written lies inside, rows of no sequence are left, and sequences that no wrong end belongs to
and no other one overlaps are as they would be. And more than 64 long sequences, whose tiles are found in another way than few. Oracle and tolerances: attention_checks.py."""
import math

import numpy as np
import pytest

from attention_checks import close, packed
from test_gpu_attention_packed import TYPES, check, enc, ptr, tensors  # noqa: F401

pytestmark = pytest.mark.gpu
GUARD = 300


def inside(x, fill):
    """The same rows in the middle of a larger tensor of `fill`: that one, and its part."""
    import torch
    big = torch.full((len(x) + 2 * GUARD, *x.shape[1:]), fill, dtype=x.dtype, device="cuda")
    big[GUARD:GUARD + len(x)] = x
    return big, big[GUARD:GUARD + len(x)]


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("n,ends,good", [(100, [0, 30, 50, 40, 500], 1), (100, [0, 30, 33, 2000000000, -2000000000], 4), (2000, [0, 700, 900, 800, 5000], 1),
                                         (2000, [0, 130, 900, 2 ** 31 - 1, -5], 4), (100, [-3, 10, 500, 600], 3), (100, [70, 60, 50], 2), (100, [0, 0, 0], 2), (2000, [1900, 2100, -2 ** 31, 2 ** 31 - 1], 0),
                                         (20000, [0] + [i * 200 + 9 for i in range(80)] + [12000, 30000], 60)])
def test_wrong_ends(enc, type, causal, n, ends, good):  # noqa: F811
    import torch
    given = tensors(n, n, n, 2, 1, 32, type)
    q, k, v, d = (inside(x, math.nan)[1] for x in given)
    p = torch.tensor(ends, dtype=torch.int32, device="cuda")
    rows = torch.full((n, 2), 7.0, device="cuda")
    results = dict(out=inside(torch.full_like(q, 7.0), 7.0), lse=inside(rows, 7.0))
    results |= {name: inside(torch.full_like(x, 7.0), 7.0) for name, x in (("dq", q), ("dk", k), ("dv", v))}
    f = {name: results[name][1] for name in ("out", "lse")}
    enc.attention(q, k, v, p, causal=causal, out=f)
    enc.attention_backward(q, k, v, p, f, d, causal=causal, out=[results[name][1] for name in ("dq", "dk", "dv")])
    torch.cuda.synchronize()
    at = np.clip(ends, 0, n)
    of_none = torch.ones(n, dtype=torch.bool, device="cuda")
    for a, b in zip(at[:-1], at[1:]):
        of_none[a:b] = False
    for name, (big, x) in results.items():
        assert (big[:GUARD] == 7.0).all() and (big[GUARD + n:] == 7.0).all() and (x[of_none] == 7.0).all(), name
    spans = [(int(a), int(max(a, b))) for a, b in zip(at[:good], at[1:good + 1])]
    for a, b in spans:
        if a < b:
            want = packed(*(x[a:b] for x in given[:3]), [0, b - a], [0, b - a], causal, 32 ** -0.5, 2.0 ** -8 if type == "bf16" else 0.0, given[3][a:b])
            for name, w in want.items():
                close(results[name][1][a:b], w, (name, a))


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dim", [32, 128])
@pytest.mark.parametrize("other", [False, True])
def test_many_long_sequences(enc, type, causal, dim, other):  # noqa: F811
    """70 sequences, 150 rows on average: some shorter than a tile, some empty, one of many tiles; and other numbers of keys."""
    rng = np.random.Generator(np.random.PCG64(dim))
    nq = rng.integers(0, 260, 70)
    nq[[3, 40, 69]] = 0, 1500, 0
    nk = rng.integers(0, 300, 70) if other else nq
    assert nq.sum() > 128 * 70 or nk.sum() > 128 * 70
    check(enc, *tensors(dim, int(nq.sum()), int(nk.sum()), 2, 1, dim, type), ptr(nq), ptr(nk) if other else None, causal)
