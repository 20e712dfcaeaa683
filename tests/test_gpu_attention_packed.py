"""Attention over packed sequences and its gradients against the formulas in 64 bits (bounds: tests/attention_checks.py)."""
import math

import numpy as np
import pytest

from attention_checks import U, close, one_head, packed

pytestmark = pytest.mark.gpu
TYPES = ["fp32", "bf16"]


def dtype(type):
    import torch
    return dict(fp32=torch.float32, bf16=torch.bfloat16)[type]


@pytest.fixture(scope="module")
def enc():
    import torch
    assert torch.cuda.is_available(), "these tests need the GPU"
    import paper_2304_14698_amd as xrl
    model = dict(n_op_types=4, n_node_dense=0, d_edge=4, d_global=0, hidden=64, rounds=0)
    e = xrl.Encoder(model, np.zeros(xrl.weight_count(model), np.float32))
    yield e
    e.close()


def ptr(lengths, front=0):
    import torch
    p = np.concatenate([[front], front + np.cumsum(lengths)]).astype(np.int32)
    return p.tolist(), torch.from_numpy(p).cuda()


def tensors(seed, n, m, heads, kv, dim, type):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda").to(dtype(type))  # noqa: E731
    return r(n, heads, dim), r(m, kv, dim), r(m, kv, dim), r(n, heads, dim)


def check(enc, q, k, v, dout, q_ptr, k_ptr, causal, scale=None, out=None, grads=None):
    """Forward and backward against 64 bits; what they wrote."""
    import torch
    qp, tq = q_ptr
    kp, tk = k_ptr or q_ptr
    how = dict(k_ptr=None if k_ptr is None else tk, causal=causal, scale=scale)
    f = enc.attention(q, k, v, tq, out=out, **how)
    g = enc.attention_backward(q, k, v, tq, f, dout, out=grads, **how)
    again = enc.attention(q, k, v, tq, **how)
    g2 = enc.attention_backward(q, k, v, tq, f, dout, **how)
    torch.cuda.synchronize()
    half = 2.0 ** -8 if q.dtype == torch.bfloat16 else 0.0
    s = float(np.float32(q.shape[2] ** -0.5 if scale is None else scale))
    want = packed(q, k, v, qp, kp, causal, s, half, dout)
    got = dict(f, dq=g[0], dk=g[1], dv=g[2])
    for name, w in want.items():
        close(got[name], w, name)
    for a, b, w in ((f["out"], again["out"], "out"), (f["lse"], again["lse"], "lse"), (g[0], g2[0], "dq"), (g[1], g2[1], "dk"), (g[2], g2[2], "dv")):
        covered = ~want[w][0].isnan()
        assert torch.equal(a[covered], b[covered])
    return got


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dim", [1, 8, 20, 32, 33, 40, 64, 80, 96, 127, 128])
@pytest.mark.parametrize("heads,kv", [(1, 1), (6, 2)])
def test_dims(enc, type, causal, dim, heads, kv):
    p = ptr([1, 0, 31, 32, 33, 70, 2, 130])
    check(enc, *tensors(dim, p[0][-1], p[0][-1], heads, kv, dim, type), p, None, causal)


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("nq,nk", [([1], [1]), ([1], [300]), ([257], [257]), ([64, 0, 5], [64, 9, 0]), ([130, 40], [20, 41]), ([128, 129], [129, 128]),
                                   ([0], [77]), ([500], [1000]), ([1] * 70, [3] * 70), ([7] * 300, [7] * 300)])
@pytest.mark.parametrize("dim", [32, 64, 128])
def test_lengths(enc, type, causal, nq, nk, dim):
    """Sequences of nothing, of one row, of rows that see no key (fewer keys than rows), tiles that end inside and at their end."""
    q_ptr, k_ptr = ptr(nq), ptr(nk)
    got = check(enc, *tensors(sum(nq), sum(nq), sum(nk), 4, 2, dim, type), q_ptr, k_ptr, causal)
    for s, (n, m) in enumerate(zip(nq, nk)):
        a = q_ptr[0][s]
        blind = min(n, max(0, n - m)) if causal else (n if m == 0 else 0)
        assert not got["out"][a:a + blind].any() and not got["dq"][a:a + blind].any() and (got["lse"][a:a + blind] == -math.inf).all()


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("seqs,total", [(1, 2000), (3, 3000), (40, 2500), (1000, 4000)])
def test_many_and_long(enc, type, seqs, total):
    rng = np.random.Generator(np.random.PCG64(seqs))
    cut = np.sort(rng.integers(0, total + 1, seqs - 1))
    p = ptr(np.diff(np.concatenate([[0], cut, [total]])))
    check(enc, *tensors(seqs, total, total, 2, 1, 64, type), p, None, True)


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("scale", [1e-3, 1.0, 5.0])
def test_scales(enc, type, scale):
    """Flat and steep softmaxes: maxima that grow along a row."""
    import torch
    p = ptr([200, 100])
    q, k, v, d = tensors(5, 300, 300, 2, 2, 64, type)
    k = (k.float() * torch.linspace(0.1, 3.0, 300, device="cuda")[:, None, None]).to(k.dtype)
    check(enc, q, k, v, d, p, None, True, scale=scale)


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("dim", [64, 40, 7])
def test_strides(enc, type, dim):
    """Parts of one product's rows, heads outside rows, odd addresses, one row of keys or of gradients for all (strides of 0), results in rows apart."""
    import torch
    p = ptr([50, 1, 90])
    n, heads, kv = 141, 4, 2
    g = torch.Generator(device="cuda").manual_seed(dim)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda").to(dtype(type))  # noqa: E731
    qkv = r(n, heads + 2 * kv, dim)
    check(enc, qkv[:, :heads], qkv[:, heads:heads + kv], qkv[:, heads + kv:], r(n, heads, dim), p, None, True)
    major = lambda h: r(h, n, dim).transpose(0, 1)  # noqa: E731
    check(enc, major(heads), major(kv), major(kv), major(heads), p, None, True)
    odd = lambda h: r(n * h * dim + 1)[1:].view(n, h, dim)  # noqa: E731
    check(enc, odd(heads), odd(kv), odd(kv), odd(heads), p, None, False)
    one = r(1, 1, dim)
    check(enc, r(n, heads, dim), one.expand(n, kv, dim), r(n, 1, dim).expand(n, kv, dim), one.expand(n, heads, dim), p, None, True)
    wide = [torch.full((n, 2 * h, dim + 3), 7.0, device="cuda", dtype=dtype(type)) for h in (heads, heads, kv, kv)]
    views = [w[:, ::2, 1:dim + 1] for w in wide]
    check(enc, r(n, heads, dim), r(n, kv, dim), r(n, kv, dim), r(n, heads, dim), p, None, True,
          out=dict(out=views[0], lse=torch.empty(n, heads, device="cuda")), grads=views[1:])
    for w in wide:
        assert (w[:, 1::2] == 7).all() and (w[..., 0] == 7).all() and (w[..., dim + 1:] == 7).all()


@pytest.mark.parametrize("type", TYPES)
def test_rows_of_no_sequence_are_left(enc, type):
    import torch
    p = ptr([40, 3, 60], front=5)
    n = 120
    q, k, v, d = tensors(1, n, n, 2, 2, 32, type)
    for x in (q, k, v, d):
        x[:5] = math.nan
        x[108:] = math.nan
    full = lambda: torch.full_like(q, 7.0)  # noqa: E731
    out, lse, grads = full(), torch.full((n, 2), 7.0, device="cuda"), [full() for _ in range(3)]
    check(enc, q, k, v, d, p, None, True, out=dict(out=out, lse=lse), grads=grads)
    for x in [out, lse] + grads:
        assert (x[:5] == 7).all() and (x[108:] == 7).all()


@pytest.mark.parametrize("ends", [[0, 50, 20, 60], [-3, 10, 500, 600], [70, 60, 50], [0, 0, 0], [2000000000, -2000000000, 5]])
def test_ends_outside_and_falling(enc, ends):
    """Every read and write stays inside the tensors; sequences in front of the first wrong end are as they would be."""
    import torch
    q, k, v, d = tensors(2, 100, 100, 2, 1, 32, "bf16")
    p = torch.tensor(ends, dtype=torch.int32, device="cuda")
    f = dict(out=torch.zeros_like(q), lse=torch.zeros(100, 2, device="cuda"))
    enc.attention(q, k, v, p, out=f)
    enc.attention_backward(q, k, v, p, f, d, out=[torch.zeros_like(x) for x in (q, k, v)])
    torch.cuda.synchronize()
    if ends[0] == 0 and ends[1] == 50:
        want = packed(q[20:50], k[20:50], v[20:50], [0, 30], [0, 30], True, 32 ** -0.5, 2.0 ** -8)
        assert f["out"][:20].isfinite().all() and want["out"][0].isfinite().all()


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("dim", [32, 64, 128])
@pytest.mark.parametrize("n,at", [(300, 170), (64, 63), (40, 0), (130, 129)])
@pytest.mark.parametrize("what", [math.nan, math.inf])
def test_what_a_row_does_not_see_reaches_nothing(enc, type, dim, n, at, what):
    """A NaN or infinity in row `at` of each tensor: results of rows that do not see it are as without it, the others are not finite."""
    import torch
    p = ptr([20, n, 20])
    a = 20 + at
    clean = tensors(n, n + 40, n + 40, 2, 1, dim, type)
    f0 = enc.attention(*clean[:3], p[1])
    g0 = enc.attention_backward(*clean[:3], p[1], f0, clean[3])
    for x in range(4):
        t = [y.clone() for y in clean]
        t[x][a, :, 3] = what
        f = enc.attention(*t[:3], p[1])
        dq, dk, dv = enc.attention_backward(*t[:3], p[1], f, t[3])
        torch.cuda.synchronize()
        late, early = slice(a, 20 + n), slice(20, a + 1)
        others = torch.ones(n + 40, dtype=torch.bool, device="cuda")
        sees = others.clone()
        if x in (1, 2):
            others[late] = False                             # rows that see the key
        elif x == 0:
            others[a] = False
        assert torch.equal(f["out"][others], f0["out"][others]), x
        if x == 2 or (x < 2 and math.isnan(what)):           # (an infinity in q or k may make a score -inf: a key that does not count)
            assert not f["out"][~others].isfinite().all()
        assert torch.equal(dq[others if x < 3 else torch.arange(n + 40, device="cuda") != a], g0[0][others if x < 3 else torch.arange(n + 40, device="cuda") != a]), x
        sees[early if x in (0, 3) else slice(20, 20 + n)] = False   # keys that a row which is not finite sees
        if x in (1, 2):
            # rows from `at` on are not finite, and reach all keys of the sequence that they see
            sees[:] = True
            sees[20:20 + n] = False
        assert torch.equal(dk[sees], g0[1][sees]) and torch.equal(dv[sees], g0[2][sees]), x


@pytest.mark.parametrize("type", TYPES)
def test_against_differences(enc, type):
    """The gradient along random directions against differences of the forward pass in 64 bits at the kernel's own inputs."""
    import torch
    p = ptr([9, 30])
    q, k, v, d = tensors(3, 39, 39, 2, 1, 32, type)
    f = enc.attention(q, k, v, p[1])
    grads = enc.attention_backward(q, k, v, p[1], f, d)
    torch.cuda.synchronize()

    def J(q, k, v):
        return float((packed(q, k, v, p[0], p[0], True, 32 ** -0.5, 0.0)["out"][0] * d.double()).sum())
    g = torch.Generator(device="cuda").manual_seed(0)
    half = 2.0 ** -8 if type == "bf16" else 0.0
    bounds = packed(q, k, v, p[0], p[0], True, 32 ** -0.5, half, d)
    for x, name in enumerate(("dq", "dk", "dv")):
        t = [y.double() for y in (q, k, v)]
        way = torch.randn(t[x].shape, generator=g, device="cuda", dtype=torch.float64)
        step = 1e-4
        up, down = list(t), list(t)
        up[x], down[x] = t[x] + step * way, t[x] - step * way
        diff = (J(*up) - J(*down)) / (2 * step)
        along = float((grads[x].double() * way).sum())
        assert abs(along - diff) <= float((bounds[name][1] * way.abs()).sum()) + 1e-5 * (1 + abs(diff)), name


def test_refusals(enc):
    import torch
    import paper_2304_14698_amd as xrl
    q, k, v, d = tensors(0, 10, 10, 4, 2, 32, "bf16")
    p = torch.tensor([0, 10], dtype=torch.int32, device="cuda")
    f = enc.attention(q, k, v, p)

    def refused(code, *a, **kw):
        with pytest.raises(xrl.XrlError) as e:
            enc.attention(*a, **kw)
        assert e.value.code == xrl.ERR[code]
    refused("VALUE", q, k, v, p, scale=0.0)
    refused("VALUE", q, k, v, p, scale=-1.0)
    refused("VALUE", q, k, v, p, scale=math.nan)
    refused("VALUE", q, k, v, p, scale=math.inf)
    big = torch.zeros(10, 1, 129, device="cuda")
    refused("UNSUPPORTED", big, big, big, p)
    refused("SHAPE", q, k, v, p, out=dict(out=torch.empty(10, 1, 32, device="cuda", dtype=q.dtype).expand(10, 4, 32), lse=f["lse"]))
    refused("SHAPE", q, k, v, p, out=dict(out=torch.empty(1, 4, 32, device="cuda", dtype=q.dtype).expand(10, 4, 32), lse=f["lse"]))
    far = torch.as_strided(torch.zeros(1, device="cuda", dtype=q.dtype), (1, 2, 32), ((1 << 23) + 1, 0, 0))   # one row: its stride does not count
    for bad in (lambda: enc.attention(q.half(), k.half(), v.half(), p), lambda: enc.attention(q, k.float(), v, p), lambda: enc.attention(q, k[:, :, :16], v, p),
                lambda: enc.attention(q, k, v[:9], p), lambda: enc.attention(q[:, :3], k, v, p), lambda: enc.attention(q, k[:9], v[:9], p),
                lambda: enc.attention(q.cpu(), k, v, p), lambda: enc.attention(q, k, v, p.long()), lambda: enc.attention(q, k, v, p[:0]),
                lambda: enc.attention(q, k, v, p, k_ptr=torch.tensor([0, 5, 10], dtype=torch.int32, device="cuda")),
                lambda: enc.attention(q.transpose(1, 2), k, v, p), lambda: enc.attention(q, k, v, p.cpu()), lambda: enc.attention(q[0], k, v, p),
                lambda: enc.attention_backward(q, k, v, p, f, d[:, :, :16]), lambda: enc.attention_backward(q, k, v, p, f, d, out=(q, k, v[:5]))):
        with pytest.raises(ValueError):
            bad()
    assert far.shape[0] == 1
    assert enc.attention(q[:0], k[:0], v[:0], p[:1])["out"].shape == (0, 4, 32)


@pytest.mark.parametrize("dim", [64, 20])
def test_recorded_in_a_graph_and_on_another_stream(dim):
    import torch
    import paper_2304_14698_amd as xrl
    stream = torch.cuda.Stream()
    model = dict(n_op_types=4, n_node_dense=0, d_edge=4, d_global=0, hidden=64, rounds=0)
    p = ptr([100, 40, 0, 7])
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        enc = xrl.Encoder(model, np.zeros(xrl.weight_count(model), np.float32))
        q, k, v, d = tensors(3, 147, 147, 4, 2, dim, "bf16")
        f = enc.attention(q, k, v, p[1])
        g = enc.attention_backward(q, k, v, p[1], f, d)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            enc.attention(q, k, v, p[1], out=f)
            enc.attention_backward(q, k, v, p[1], f, d, out=g)
        for replay in range(4):
            q.copy_(tensors(10 + replay, 147, 147, 4, 2, dim, "bf16")[0])
            graph.replay()
            stream.synchronize()
            want = enc.attention(q, k, v, p[1])
            dw = enc.attention_backward(q, k, v, p[1], want, d)
            torch.zeros(1 << 20, device="cuda").add_(1.0).sum().item()
            for a, b in zip([f["out"], f["lse"], *g], [want["out"], want["lse"], *dw]):
                assert torch.equal(a, b), replay
        enc.close()


def test_rows_behind_two_to_the_31st(enc):
    """Elements behind 2^31 of every tensor."""
    import torch
    n, heads, dim = (1 << 31) // (4 * 128) + 300, 4, 128
    q = torch.zeros(n, heads, dim, device="cuda", dtype=torch.bfloat16)
    p = torch.tensor([0, 0, n - 200, n], dtype=torch.int32, device="cuda")
    p[1] = n - 400
    p[0] = n - 400
    g = torch.Generator(device="cuda").manual_seed(1)
    q[-400:] = torch.randn(400, heads, dim, generator=g, device="cuda").bfloat16()
    f = enc.attention(q, q, q, p)
    dq, dk, dv = enc.attention_backward(q, q, q, p, f, q)
    torch.cuda.synchronize()
    x = q[-200:]
    want = packed(x, x, x, [0, 200], [0, 200], True, 128 ** -0.5, 2.0 ** -8, x)
    for got, name in ((f["out"], "out"), (f["lse"], "lse"), (dq, "dq"), (dk, "dk"), (dv, "dv")):
        close(got[-200:], want[name], name)


def test_bounds_hold_for_roundings_alone():
    """The bounds themselves, on the CPU's formulas: float32 scores and exponentials stay inside them."""
    import torch
    g = torch.Generator().manual_seed(0)
    q, k, v = (torch.randn(40, 16, generator=g) for _ in range(3))
    want = one_head(q.double(), k.double(), v.double(), True, 0.25, 0.0)
    s = (0.25 * (q @ k.T)).masked_fill(~torch.ones(40, 40).tril().bool(), -math.inf)
    close(s.softmax(1) @ v, want["out"])
    close(s.logsumexp(1), want["lse"])
    assert U == 2.0 ** -24
