"""Attention by its formulas in 64 bits, with bounds of what fp32 sums (and, in bf16, roundings of the factors) may be off by.

u = 2^-24, a score's sum of `dim` products is off by at most (dim + 4) u of the sum of the products' sizes; an exponential by that, by the roundings of its argument
(4 u of the sizes of the score and of the row's largest) and by 8 u; a sum of n of them by (n + 16) u of the sum of sizes. In bf16 the probabilities and their
gradients are rounded as factors of the second product, and results when they are stored: half a step, 2^-8, each. An exponential below the least
normal number, 2^-126, counts as 0: a probability is off by that besides (with scores some 87 apart, where a row's sum of 2 e-37 is then 0)."""
import math

U = 2.0 ** -24
LEAST = 2.0 ** -126


def seen(n, m, causal, device):
    import torch
    i, j = torch.arange(n, device=device)[:, None], torch.arange(m, device=device)[None]
    return j <= i + (m - n) if causal else torch.ones(n, m, dtype=torch.bool, device=device)


def one_head(q, k, v, causal, scale, half, dout=None, out_bound=None, terms=1):
    """q [n, dim], k, v [m, dim] in float64 (the inputs' own values): results and bounds as dict name -> (value, bound). out_bound: of the out that the
    backward call was given. half: half a step of the type that factors and results are rounded to (0: fp32)."""
    import torch
    n, m, dim = q.shape[0], k.shape[0], q.shape[1]
    ok = seen(n, m, causal, q.device)
    s = scale * (q @ k.T)
    size = scale * (q.abs() @ k.abs().T)
    s = s.masked_fill(~ok, -math.inf)
    any_ = ok.any(1)
    top = torch.where(any_, s.amax(1) if m else torch.zeros(n, dtype=s.dtype, device=s.device), 0.0)
    lse = torch.where(any_, torch.logsumexp(s, 1) if m else top, -math.inf)
    p = torch.where(ok, (s - lse.nan_to_num(neginf=0.0)[:, None]).exp(), 0.0)
    s0 = torch.where(ok, s, 0.0)
    rel = torch.where(ok, (dim + 4) * U * size + 4 * U * (s0.abs() + top.abs()[:, None]) + 8 * U, 0.0)
    worst = rel.amax(1) if m else torch.zeros_like(top)
    total = worst + (m + 16) * U
    res = dict(lse=(lse, torch.where(any_, total + 8 * U * (lse.abs().nan_to_num(posinf=0.0) + top.abs()), 0.0)))
    out = p @ v
    least = torch.where(ok, LEAST, 0.0)
    b = (p @ v.abs()) * (2 * total + half)[:, None] + least.to(v.dtype) @ v.abs() if m else torch.zeros_like(out)
    store = half if half else 2 * U
    res["out"] = (out, b + store * (out.abs() + b))
    if dout is None:
        return res
    r = rel + total[:, None] + 8 * U * (lse.abs().nan_to_num(posinf=0.0) + top.abs())[:, None]
    add = lambda k: (k + 16) * U  # noqa: E731
    dv, size_dv = p.T @ dout, p.T @ dout.abs()
    bdv = (p * (r + half) + least).T @ dout.abs() + add(n * terms) * size_dv
    dp, D = dout @ v.T, (dout * out).sum(1)
    bdp = (dim + 4) * U * (dout.abs() @ v.abs().T)
    bD = (dim + 4) * U * (dout.abs() * out.abs()).sum(1) + (dout.abs() * out_bound).sum(1)
    ds = p * (dp - D[:, None])
    bds = p * (r * (dp - D[:, None]).abs() + bdp + bD[:, None] + 2 * U * (dp.abs() + D.abs()[:, None])) + least * (dp - D[:, None]).abs()
    bds = bds + half * (ds.abs() + bds)
    res["dq"] = (scale * ds @ k, scale * (bds @ k.abs() + add(m) * ds.abs() @ k.abs()))
    res["dk"] = (scale * ds.T @ q, scale * (bds.T @ q.abs() + add(n * terms) * ds.abs().T @ q.abs()))
    res["dv"] = (dv, bdv)
    return res


def packed(q, k, v, q_ptr, k_ptr, causal, scale, half, dout=None):
    """All sequences and heads: dict name -> (value, bound), of the packed tensors' shapes; rows of no sequence NaN. q_ptr, k_ptr: lists."""
    import torch
    q, k, v = q.double(), k.double(), v.double()
    heads, kv = q.shape[1], k.shape[1]
    group = heads // kv
    nan = lambda x: [torch.full(x.shape, math.nan, dtype=torch.float64, device=q.device) for _ in range(2)]  # noqa: E731
    res = dict(out=nan(q), lse=nan(q[..., 0]))
    if dout is not None:
        res.update(dq=nan(q), dk=nan(k), dv=nan(v))
    for a, b, c, d in zip(q_ptr[:-1], q_ptr[1:], k_ptr[:-1], k_ptr[1:]):
        for h in range(kv):
            for name in ("dk", "dv"):
                if name in res:
                    for x in res[name]:
                        x[c:d, h] = 0.0
            for e in range(h * group, (h + 1) * group):
                args = (q[a:b, e], k[c:d, h], v[c:d, h], causal, scale, half)
                one = one_head(*args)
                if dout is not None:
                    one = one_head(*args, dout[a:b, e].double(), one["out"][1], group)
                for name, (x, y) in one.items():
                    for to, part in zip(res[name], (x, y)):
                        if name in ("dk", "dv"):
                            to[c:d, h] += part
                        else:
                            to[a:b, e] = part
    store = half if half else 2 * U
    for name in ("dq", "dk", "dv"):
        if name in res:
            res[name][1] += store * (res[name][0].abs() + res[name][1])
    return res


def close(got, want, where=""):
    """Every covered entry of `got` within its bound, infinities equal."""
    import torch
    x, b = want
    covered = ~x.isnan()
    g, x, b = got.double()[covered], x[covered], b[covered]
    inf = x.isinf()
    assert torch.equal(g[inf], x[inf]), where
    off = (g - x).abs()[~inf]
    bad = ~(off <= b[~inf] + 1e-37)
    assert not bad.any(), (where, int(bad.sum()), float(off[bad].nan_to_num(nan=math.inf).max()), float((off / b[~inf].clamp(min=1e-37))[bad].nan_to_num(nan=math.inf).max()))
