"""The norm of heads with the rotation by position, and its gradients, against the formulas in 64 bits.

u = 2^-24. A row's sum of squares has dim positive terms: r is off by R = (dim / 2 + 6) u of itself. A cosine or sine is off by 8 u and by 2^-52 of the angle, which is taken in
64 bits. The rest is a handful of roundings of the terms' sizes, and one of the result: 2^-8 of it in bf16."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
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


def turned(y, pos, freqs, interleaved, back=False):
    """(value, size of the terms, error of the angles' cosines) of y [n, h, dim] float64."""
    import torch
    half = freqs.numel()
    a = pos.double()[:, None] * freqs.double()
    c, s = a.cos()[:, None], a.sin()[:, None] * (-1 if back else 1)
    j = torch.arange(half, device=y.device)
    i1, i2 = (2 * j, 2 * j + 1) if interleaved else (j, j + half)
    z, size, err = y.clone(), y.abs(), torch.zeros_like(y)
    y1, y2 = y[..., i1], y[..., i2]
    z[..., i1], z[..., i2] = y1 * c - y2 * s, y1 * s + y2 * c
    both = y1.abs() + y2.abs()
    size[..., i1] = size[..., i2] = both
    off = both * (8 * U + 2.0 ** -52 * a.abs()[:, None])
    err[..., i1] = err[..., i2] = off
    return z, size, err


def normed(x, w, eps):
    if w is None:
        return x, 1.0, 0.0
    r = ((x * x).mean(-1, keepdim=True) + eps).rsqrt()
    return x * r * w.double(), r, (x.shape[-1] / 2 + 6) * U


def sizes_turned(b, freqs, interleaved):
    """Sums over the pairs of a bound's entries."""
    import torch
    half = freqs.numel()
    j = torch.arange(half, device=b.device)
    i1, i2 = (2 * j, 2 * j + 1) if interleaved else (j, j + half)
    out = b.clone()
    out[..., i1] = out[..., i2] = b[..., i1] + b[..., i2]
    return out


def check(enc, q, k, pos, freqs, wq, wk, eps=1e-6, interleaved=False, out=None, back=None):
    import torch
    g = torch.Generator(device="cuda").manual_seed(9)
    dz = [(torch.randn(x.shape, generator=g, device="cuda")).to(x.dtype) for x in (q, k) if x is not None] + [None]
    dw0 = [torch.randn(q.shape[2], generator=g, device="cuda") for _ in range(2)]
    how = dict(q_weight=wq, k_weight=wk, eps=eps, interleaved=interleaved)
    z = enc.head_rotary(q, k, pos, freqs, out=out, **how)
    dw = [w.clone() for w in dw0]
    dx = enc.head_rotary_backward(q, k, pos, freqs, dz[0], dz[1], dq_weight=dw[0], dk_weight=dw[1], out=back, **how)
    dw2 = [w.clone() for w in dw0]
    again = enc.head_rotary_backward(q, k, pos, freqs, dz[0], dz[1], dq_weight=dw2[0], dk_weight=dw2[1], **how)
    torch.cuda.synchronize()
    half = 2.0 ** -8 if q.dtype == torch.bfloat16 else U
    for x, w, zz, d, ddx, a, ddw, a2, first in zip((q, k), (wq, wk), z, dz, dx, again, dw, dw2, dw0):
        if x is None:
            assert zz is None and ddx is None
            continue
        if back is None:                                     # (rows at odd places are read in another way, which sums in another order)
            assert torch.equal(ddx, a) and torch.equal(ddw, a2)
        x = x.double()
        y, r, R = normed(x, w, eps)
        want, size, err = turned(y, pos, freqs, interleaved)
        bound = size * (R + 6 * U) + err
        assert ((zz.double() - want).abs() <= bound + half * (want.abs() + bound) + 1e-37).all()
        d = d.double()
        back_, size, gerr = turned(d, pos, freqs, interleaved, True)
        gerr = gerr + 2 * U * size
        if w is None:
            want, bound = back_, gerr
            assert torch.equal(ddw, first)
        else:
            ww, n = w.double(), x.shape[-1]
            gw = back_ * ww
            along = (gw * x).mean(-1, keepdim=True)
            want = r * gw - x * r ** 3 * along
            b1 = r * (gw.abs() * (R + 6 * U) + ww.abs() * gerr)
            b2 = r ** 3 * x.abs() * ((gw * x).abs().mean(-1, keepdim=True) * (3 * R + (n + 8) * U) + (gerr * (ww * x).abs()).mean(-1, keepdim=True))
            bound = b1 + b2
            terms = back_ * x * r
            sdw = first.double() + terms.sum((0, 1))
            count = x.shape[0] * x.shape[1]
            bdw = (terms.abs() * (R + 8 * U) + gerr * (x * r).abs()).sum((0, 1)) + (count + 32) * U * (terms.abs().sum((0, 1)) + first.abs())
            assert ((ddw.double() - sdw).abs() <= bdw).all()
        assert ((ddx.double() - want).abs() <= bound + half * (want.abs() + bound) + 1e-37).all()
    return z, dx


def inputs(seed, n, heads, kv, dim, type, far):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda h: (3 * torch.randn(n, h, dim, generator=g, device="cuda")).to(dtype(type))  # noqa: E731
    pos = torch.randint(0, far, (n,), generator=g, device="cuda").int()
    w = lambda: 1 + 0.2 * torch.randn(dim, generator=g, device="cuda")  # noqa: E731
    return r(heads), r(kv), pos, w(), w()


def freqs_of(rotary, **kw):
    import torch
    import paper_2304_14698_amd as xrl
    return torch.from_numpy(xrl.rotary_freqs(rotary, **kw)).cuda()


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dim,rotary", [(1, 0), (2, 2), (6, 4), (7, 6), (32, 32), (32, 16), (40, 40), (40, 8), (64, 64), (64, 22), (96, 96), (128, 128), (128, 64), (128, 126),
                                        (129, 128), (200, 160), (256, 256), (256, 0)])
@pytest.mark.parametrize("norm", [True, False])
def test_dims_and_layouts(enc, type, interleaved, dim, rotary, norm):
    q, k, pos, wq, wk = inputs(dim + rotary, 37, 5, 2, dim, type, 5000)
    check(enc, q, k, pos, freqs_of(rotary), wq if norm else None, wk if norm else None, interleaved=interleaved)


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("n,heads,kv", [(1, 1, 1), (1, 32, 8), (3, 7, 1), (2000, 8, 2), (9000, 3, 3), (5, 40, 0)])
@pytest.mark.parametrize("which", ["both", "q", "k"])
def test_counts(enc, type, n, heads, kv, which):
    """One row to more than the chip holds at once, heads of one tensor, weights of one."""
    q, k, pos, wq, wk = inputs(n, n, heads, max(kv, 1), 64, type, 1 << 20)
    check(enc, q, k if kv else None, pos, freqs_of(64), wq if which != "k" else None, wk if which != "q" else None)


def test_far_and_negative_positions(enc):
    import torch
    q, k, _, wq, wk = inputs(1, 6, 2, 2, 64, "fp32", 10)
    pos = torch.tensor([0, -1, 2 ** 31 - 1, -2 ** 31, 1 << 24, 123456789], dtype=torch.int32, device="cuda")
    check(enc, q, k, pos, freqs_of(64), wq, wk)
    z, _ = check(enc, q, k, pos, freqs_of(64), None, None)
    assert torch.equal(z[0][0], q[0])                        # position 0: as it was


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("dim", [64, 20])
def test_strides_and_in_place(enc, type, dim):
    """Parts of one product's rows, written where they lay; heads outside rows; odd addresses; one row for all; rows apart."""
    import torch
    n, heads, kv = 50, 4, 2
    g = torch.Generator(device="cuda").manual_seed(1)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda").to(dtype(type))  # noqa: E731
    pos = torch.arange(n, device="cuda", dtype=torch.int32)
    w, f = 1 + 0.1 * torch.randn(dim, generator=g, device="cuda"), freqs_of(dim // 4 * 2)
    qkv = r(n, heads + 2 * kv, dim)
    q, k = qkv[:, :heads], qkv[:, heads:heads + kv]
    z, _ = check(enc, q, k, pos, f, w, w)
    rest = qkv[:, heads + kv:].clone()
    enc.head_rotary(q, k, pos, f, q_weight=w, k_weight=w, out=(q, k))
    torch.cuda.synchronize()
    assert torch.equal(q, z[0]) and torch.equal(k, z[1]) and torch.equal(qkv[:, heads + kv:], rest)
    dq, dk = r(n, heads, dim), r(n, kv, dim)
    want = enc.head_rotary_backward(q, k, pos, f, dq, dk, q_weight=w, k_weight=w)
    enc.head_rotary_backward(q, k, pos, f, dq, dk, q_weight=w, k_weight=w, out=(dq, dk))
    torch.cuda.synchronize()
    assert torch.equal(dq, want[0]) and torch.equal(dk, want[1])
    major = lambda h: r(h, n, dim).transpose(0, 1)  # noqa: E731
    check(enc, major(heads), major(kv), pos, f, w, w, interleaved=True)
    odd = lambda h: r(n * h * dim + 1)[1:].view(n, h, dim)  # noqa: E731
    check(enc, odd(heads), odd(kv), pos, f, w, w)
    check(enc, r(1, 1, dim).expand(n, heads, dim), r(n, 1, dim).expand(n, kv, dim), pos, f, w, w)
    wide = [torch.full((n, 2 * h, dim + 3), 7.0, device="cuda", dtype=dtype(type)) for h in (heads, kv)]
    check(enc, r(n, heads, dim), r(n, kv, dim), pos, f, w, w, out=[x[:, ::2, 1:dim + 1] for x in wide], back=[x[:, 1::2, 1:dim + 1] for x in wide])
    for x in wide:
        assert (x[..., 0] == 7).all() and (x[..., dim + 1:] == 7).all()


def test_what_is_not_finite_stays_in_its_row(enc):
    import torch
    q, k, pos, wq, wk = inputs(4, 20, 3, 2, 64, "bf16", 100)
    f = freqs_of(32)
    z0 = enc.head_rotary(q, k, pos, f, q_weight=wq, k_weight=None)
    q[7, 1, 3], k[9, 0, 2], k[9, 0, 50] = math.nan, math.inf, -math.inf
    z = enc.head_rotary(q, k, pos, f, q_weight=wq, k_weight=None)
    torch.cuda.synchronize()
    ok = torch.ones(20, 3, dtype=torch.bool, device="cuda")
    ok[7, 1] = False
    assert torch.equal(z[0][ok], z0[0][ok]) and z[0][7, 1].isnan().all()
    odd = ~torch.isfinite(z[1])
    assert odd[9, 0].nonzero()[:, 0].tolist() == [2, 18, 50] and int(odd.sum()) == 3 and float(z[1][9, 0, 50]) == -math.inf


@pytest.mark.parametrize("interleaved", [False, True])
def test_against_differences(enc, interleaved):
    import torch
    q, k, pos, wq, wk = inputs(5, 4, 2, 1, 16, "fp32", 50)
    f = freqs_of(12)
    g = torch.Generator(device="cuda").manual_seed(0)
    d = torch.randn(q.shape, generator=g, device="cuda")
    dw = torch.zeros(16, device="cuda")
    dq, _ = enc.head_rotary_backward(q, k, pos, f, d, torch.zeros_like(k), q_weight=wq, k_weight=wk, dq_weight=dw, interleaved=interleaved)
    torch.cuda.synchronize()

    def J(x, w):
        return float((turned(normed(x, w, 1e-6)[0], pos, f, interleaved)[0] * d.double()).sum())
    way, wway = torch.randn(q.shape, generator=g, device="cuda").double(), torch.randn(16, generator=g, device="cuda").double()
    h = 1e-5
    diff = (J(q.double() + h * way, wq.double()) - J(q.double() - h * way, wq.double())) / (2 * h)
    assert abs(float((dq.double() * way).sum()) - diff) <= 1e-4 * (1 + abs(diff))
    diff = (J(q.double(), wq.double() + h * wway) - J(q.double(), wq.double() - h * wway)) / (2 * h)
    assert abs(float((dw.double() * wway).sum()) - diff) <= 1e-4 * (1 + abs(diff))


def test_refusals(enc):
    import torch
    import paper_2304_14698_amd as xrl
    q, k, pos, wq, wk = inputs(6, 5, 2, 1, 32, "bf16", 100)
    f = freqs_of(32)

    def refused(code, *a, **kw):
        with pytest.raises(xrl.XrlError) as e:
            enc.head_rotary(*a, **kw)
        assert e.value.code == xrl.ERR[code]
    refused("VALUE", q, k, pos, f, eps=-1.0)
    refused("VALUE", q, k, pos, f, eps=math.nan)
    refused("SHAPE", q, k, pos, freqs_of(34))
    big = torch.zeros(5, 1, 257, device="cuda")
    refused("UNSUPPORTED", big, None, pos, f)
    refused("SHAPE", q, k, pos, f, out=(q, k[:1].expand(5, 1, 32)))
    for bad in (lambda: enc.head_rotary(q, k[:4], pos, f), lambda: enc.head_rotary(q, k.float(), pos, f), lambda: enc.head_rotary(q, k, pos[:4], f),
                lambda: enc.head_rotary(q, k, pos.long(), f), lambda: enc.head_rotary(q, k, pos, f.double()), lambda: enc.head_rotary(q, k, pos, f, q_weight=wq[:31]),
                lambda: enc.head_rotary(q.cpu(), k, pos, f), lambda: enc.head_rotary(q, k, pos, f, out=(q.float(), k)),
                lambda: enc.head_rotary(q, k, pos, f, q_weight=wq.cpu())):
        with pytest.raises(ValueError):
            bad()
    assert enc.head_rotary(q[:0], k[:0], pos[:0], f)[0].shape == (0, 2, 32)


def test_recorded_in_a_graph():
    import torch
    import paper_2304_14698_amd as xrl
    stream = torch.cuda.Stream()
    model = dict(n_op_types=4, n_node_dense=0, d_edge=4, d_global=0, hidden=64, rounds=0)
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        enc = xrl.Encoder(model, np.zeros(xrl.weight_count(model), np.float32))
        q, k, pos, wq, wk = inputs(7, 300, 4, 2, 64, "bf16", 1000)
        f = freqs_of(64)
        dq, dk = torch.randn_like(q), torch.randn_like(k)
        dw = torch.zeros(2, 64, device="cuda")
        how = dict(q_weight=wq, k_weight=wk)
        z, g = enc.head_rotary(q, k, pos, f, **how), enc.head_rotary_backward(q, k, pos, f, dq, dk, dq_weight=dw[0], dk_weight=dw[1], **how)
        dw.zero_()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            enc.head_rotary(q, k, pos, f, out=z, **how)
            enc.head_rotary_backward(q, k, pos, f, dq, dk, dq_weight=dw[0], dk_weight=dw[1], out=g, **how)
        want_dw = torch.zeros(2, 64, device="cuda")
        for replay in range(3):
            q.mul_(1.25)
            graph.replay()
            stream.synchronize()
            a, b = enc.head_rotary(q, k, pos, f, **how), enc.head_rotary_backward(q, k, pos, f, dq, dk, dq_weight=want_dw[0], dk_weight=want_dw[1], **how)
            torch.zeros(1 << 20, device="cuda").add_(1.0).sum().item()
            for x, y in zip([*z, *g, dw], [*a, *b, want_dw]):
                assert torch.equal(x, y), replay
        enc.close()
