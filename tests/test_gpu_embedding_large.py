"""Embedding and its gradient where results or gradients are larger than the caches, with windows of both sizes and runs of many thousand windows.
Tolerances as at the smaller sizes: the lookup bit for bit, a gradient of k terms within (k + 2) 2^-24 of their sizes' sum and two roundings."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def enc():
    import torch
    assert torch.cuda.is_available(), "these tests need the GPU"
    import paper_2304_14698_amd as xrl
    model = dict(n_op_types=4, n_node_dense=0, d_edge=4, d_global=0, hidden=64, rounds=0)
    e = xrl.Encoder(model, np.zeros(xrl.weight_count(model), np.float32))
    yield e
    e.close()


def ids_of(g, n, vocab, kind):
    import torch
    u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
    if kind == "tail":
        ids = ((vocab + 1.0) ** u - 1).long().clamp_(max=vocab - 1)
    elif kind == "one":
        ids = torch.full((n,), vocab - 2, device="cuda")
    elif kind == "most":                              # one id, others strewn among it
        ids = torch.where(u < 0.97, vocab // 2, (u * 1e6).long() % vocab)
    else:
        ids = (u * vocab).long().clamp_(max=vocab - 1)
    ids[torch.rand(n, generator=g, device="cuda") < 0.01] = -1
    ids[n // 3] = vocab
    return ids.int()


def check_gradient(dout, ids, before, after, scale):
    """In 64 bits, some columns at a time, and the places of an id in many sums, which are then added up: one sum of a million terms takes minutes."""
    import torch
    vocab, dim = before.shape
    keep = (ids >= 0) & (ids < vocab)
    i = ids[keep].long()
    k = torch.bincount(i, minlength=vocab)[:, None]
    sums = max(1, min(1024, (1 << 21) // vocab))
    at = i * sums + torch.arange(i.numel(), device="cuda") % sums
    for lo in range(0, dim, 64):
        c = slice(lo, lo + 64)
        d = scale * dout[:, c][keep].double()
        add = lambda x: torch.zeros(vocab * sums, x.shape[1], dtype=torch.float64, device="cuda").index_add_(0, at, x).view(vocab, sums, -1).sum(1)  # noqa: E731
        want, size = before[:, c].double() + add(d), add(d.abs())
        bound = (k + 2) * U * size + 2 * U * (before[:, c].double().abs() + size)
        assert ((after[:, c].double() - want).abs() <= bound).all()
    assert torch.equal(after[k[:, 0] == 0], before[k[:, 0] == 0])


@pytest.mark.parametrize("kind", ["tail", "even", "most"])
@pytest.mark.parametrize("n,vocab,dim,type", [(65553, 50021, 1027, "bf16"), (65553, 3001, 1025, "fp32"), (77013, 5000, 130, "fp32"), (65535, 5000, 130, "fp32"),
                                              (65600, 5000, 300, "bf16"), (16383, 900, 1030, "fp32"), (300001, 20000, 60, "fp32"), (150001, 2000, 250, "bf16"),
                                              (40001, 70, 2100, "bf16")])
def test_gradients_larger_than_the_caches(enc, n, vocab, dim, type, kind):
    import torch
    dt = dict(fp32=torch.float32, bf16=torch.bfloat16)[type]
    g = torch.Generator(device="cuda").manual_seed(n + dim)
    dout = torch.randn(1 + n * (dim + 3), generator=g, device="cuda").to(dt)[1:].view(n, dim + 3)[:, :dim]   # rows apart, from an odd address
    before = torch.randn(vocab, dim, generator=g, device="cuda")
    ids = ids_of(g, n, vocab, kind)
    after = [enc.embedding_backward(dout, ids, before.clone(), scale=0.7) for _ in range(2)]
    torch.cuda.synchronize()
    assert torch.equal(after[0], after[1])
    check_gradient(dout, ids, before, after[0], float(np.float32(0.7)))


@pytest.mark.parametrize("kind", ["one", "most"])
@pytest.mark.parametrize("n,vocab,dim", [(140001, 90, 20), (1200007, 200, 9), (140001, 5000, 300), (4400001, 70, 3)])
def test_runs_of_many_thousand_windows(enc, n, vocab, dim, kind):
    """The number of a run's windows is found by probes of 64 windows, of 4096 and of more."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(n)
    dout, before = torch.randn(n, dim, generator=g, device="cuda"), torch.randn(vocab, dim, generator=g, device="cuda")
    ids = ids_of(g, n, vocab, kind)
    after = [enc.embedding_backward(dout, ids, before.clone()) for _ in range(2)]
    torch.cuda.synchronize()
    assert torch.equal(after[0], after[1])
    check_gradient(dout, ids, before, after[0], 1.0)


def test_a_sorted_gradient_behind_two_to_the_31st(enc):
    import torch
    rows, dim, vocab = (1 << 20) + 3, 2100, 500           # 2.2e9 entries
    dout = torch.zeros((rows, dim), dtype=torch.bfloat16, device="cuda")
    ids = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
    at = torch.tensor([5, 70, rows // 2, rows - 40, rows - 39, rows - 2, rows - 1], device="cuda")
    ids[at] = torch.tensor([7, 499, 7, 0, 7, 499, 7], dtype=torch.int32, device="cuda")
    dout[at] = torch.randn(7, dim, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").bfloat16()
    got = enc.embedding_backward(dout, ids, torch.zeros((vocab, dim), device="cuda"))
    ids[rows - 300000:] = 7                                # and a run whose carries lie there
    dout[rows - 300000:] = 1.0
    many = enc.embedding_backward(dout, ids, torch.zeros((vocab, dim), device="cuda"))
    torch.cuda.synchronize()
    want = torch.zeros((vocab, dim), dtype=torch.float64, device="cuda")
    first = torch.tensor([7, 499, 7, 0, 7, 499, 7], device="cuda")
    size = torch.zeros_like(want)
    values = torch.randn(7, dim, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").bfloat16().double()
    want.index_add_(0, first, values)
    size.index_add_(0, first, values.abs())
    assert ((got.double() - want).abs() <= 9 * U * size).all()
    early = values[0] + values[2]                          # places 5 and rows // 2
    assert ((many[7].double() - (300000 + early)).abs() <= 300004 * U * (300000 + values[0].abs() + values[2].abs())).all()
    assert torch.equal(many[499].double(), values[1]) and not many[0].any()


@pytest.mark.parametrize("types", ["fp32 fp32", "fp32 bf16", "bf16 fp32", "bf16 bf16"])
@pytest.mark.parametrize("n,dim,offset,apart", [(70001, 515, 0, 0), (70001, 515, 1, 5), (70000, 512, 0, 0), (35003, 1029, 3, 1), (9000001, 3, 0, 0)])
def test_lookups_larger_than_the_caches(enc, n, dim, offset, apart, types):
    import torch
    tt, to = (dict(fp32=torch.float32, bf16=torch.bfloat16)[x] for x in types.split())
    vocab = 3001
    g = torch.Generator(device="cuda").manual_seed(n + offset)
    table = torch.randn(offset + vocab * (dim + apart), generator=g, device="cuda").to(tt)[offset:].view(vocab, dim + apart)[:, :dim]
    ids = ids_of(g, n, vocab, "tail")
    outm = torch.full((offset + n * (dim + apart),), 7.0, device="cuda", dtype=to)
    out = outm[offset:].view(n, dim + apart)[:, :dim]
    enc.embedding(table, ids, scale=11.3, out=out)
    torch.cuda.synchronize()
    inside = (ids >= 0) & (ids < vocab)
    want = torch.where(inside[:, None], table[ids.long().clamp(0, vocab - 1)].float() * float(np.float32(11.3)), 0.0).to(to)
    assert torch.equal(out, want)
    assert (outm[:offset] == 7).all() and (outm[offset:].view(n, dim + apart)[:, dim:] == 7).all()
