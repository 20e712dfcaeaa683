"""What attention in bf16 is off by over whole tensors: the roundings that it says it makes, and nothing besides.

The model is the formulas in 64 bits with those roundings alone: p as a factor of v and dout, ds as a factor of q, and each result once. ds as a factor of k is two bf16 numbers,
2^-17 of it or less, and D = sum_j p_ij (dout_i . v_j) is free of out's rounding, but for dq of rows that see more than 512 keys: there D comes from the out that
was given, off by delta_i = dout_i . (out given - out), which is -scale delta_i sum_j p_ij k_j of dq. A kernel with these roundings makes nearly the same ones, of fp32 values (sums off by up to
(m + dim) 2^-24 or 1e-4 of their terms' sizes, some 2 % of the roundings' 1.7e-3 if they all had one sign, far less as they have not): 5 % more than the model are allowed. Leaving out ds's second part
would be 1.5 times the model of dq, D from the rounded out 1.1 to 2 times that of dq and 1.17 times that of dk.

The forward pass rounds e^(s - reference), the reference a maximum of the keys so far; the model rounds e^(s - lse). A weight w = 2^n f, 1 <= f < 2, is rounded with a mean square of (2^(n - 7))^2 / 12, or 2^-14 / (12 f^2) of w^2,
and over many rows a shift of all s spreads f in the same way, but for rows whose reference is their own largest score: that weight is 1, without an error, so the kernel has less than the model there. (Relative to
each row's largest score every row would have such a weight, which the kernel's have not: with references from the first 32 or 64 keys, in rows of 100, some are above 1.)"""
import math

import pytest

from test_gpu_attention_packed import enc, ptr, tensors  # noqa: F401

pytestmark = pytest.mark.gpu


def rounded(x):
    import torch
    return x.to(torch.bfloat16).double()


def model(q, k, v, dout, out, causal, scale):
    """One sequence and one head in 64 bits, `out` what the backward call is given: the results, and what the roundings leave of them before their own."""
    import torch
    n, m = q.shape[0], k.shape[0]
    s = scale * (q @ k.T)
    if causal:
        s = s.masked_fill(torch.ones(n, m, dtype=torch.bool, device=q.device).triu(1 + m - n), -math.inf)
    top = s.amax(1, keepdim=True)
    p = (s - top).exp()
    p = p / p.sum(1, keepdim=True)
    o = p @ v
    dp = dout @ v.T
    ds = p * (dp - (p * dp).sum(1, keepdim=True))
    delta = (dout * (out - o)).sum(1) if m > 512 else torch.zeros(n, dtype=s.dtype, device=s.device)
    exact = dict(out=o, dq=scale * ds @ k, dk=scale * ds.T @ q, dv=p.T @ dout)
    off = dict(out=rounded(p) @ v, dq=scale * (ds - delta[:, None] * p) @ k, dk=scale * rounded(ds).T @ q, dv=rounded(p).T @ dout)
    return exact, off


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dim", [32, 64, 128])
@pytest.mark.parametrize("lengths", [[1 + i % 24 for i in range(240)], [300, 512, 411, 500], [100] * 20, [1500, 2000]])
def test_whole_tensors(enc, causal, dim, lengths):  # noqa: F811
    import torch
    p, t = ptr(lengths)
    n, heads, kv = p[-1], 4, 2
    q, k, v, d = tensors(dim + len(lengths), n, n, heads, kv, dim, "bf16")
    f = enc.attention(q, k, v, t, causal=causal)
    got = dict(zip(("dq", "dk", "dv"), enc.attention_backward(q, k, v, t, f, d, causal=causal)), out=f["out"])
    torch.cuda.synchronize()
    like = dict(out=q, dq=q, dk=k, dv=k)
    exact, off = ({name: torch.zeros(x.shape, dtype=torch.float64, device="cuda") for name, x in like.items()} for _ in range(2))
    q, k, v, d, out = (x.double() for x in (q, k, v, d, f["out"]))
    for a, b in zip(p[:-1], p[1:]):
        for h in range(heads):
            g = h * kv // heads
            for to, one in zip((exact, off), model(q[a:b, h], k[a:b, g], v[a:b, g], d[a:b, h], out[a:b, h], causal, dim ** -0.5)):
                for name, x in one.items():
                    to[name][a:b, g if name in ("dk", "dv") else h] += x
    errors = {name: (float((got[name].double() - x).norm() / x.norm()), float((rounded(off[name]) - x).norm() / x.norm())) for name, x in exact.items()}
    print(errors)
    for name, (err, least) in errors.items():
        assert err <= 1.05 * least, (name, errors)
