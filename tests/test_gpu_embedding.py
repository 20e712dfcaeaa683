"""Embedding lookup and its gradient by sorted ids, against plain forms.

The lookup multiplies in fp32 and rounds once: the same bits as the plain form in fp32. The gradient is compared with sums in 64
bits: an fp32 sum of k terms in any order is off by at most k 2^-24 times the sum of their sizes, the scaling and the addition to
the row by two roundings more."""
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


def ids_of(rng, n, vocab, kind):
    if kind == "one":
        ids = np.full(n, vocab - 1)
    elif kind == "tail":
        ids = np.minimum((vocab + 1.0) ** rng.random(n) - 1, vocab - 1).astype(np.int64)
    elif kind == "up":
        ids = np.sort(rng.integers(0, vocab, n))
    else:
        ids = rng.integers(0, vocab, n)
    if kind == "pads":                       # ids outside the table, at both of its ends
        ids = np.where(rng.random(n) < 0.4, rng.choice([-1, vocab, -2 ** 31, 2 ** 31 - 1], n), ids)
    if kind == "none":
        ids = np.full(n, -1)
    return ids.astype(np.int32)


SHAPES = [(1, 7, 64), (1, 1, 1), (3, 5, 77), (64, 40, 128), (257, 1000, 100), (1025, 33, 48), (5000, 70001, 24), (33, 9, 2056), (4099, 3, 8)]


@pytest.mark.parametrize("n,vocab,dim", SHAPES)
@pytest.mark.parametrize("types", ["fp32 fp32", "fp32 bf16", "bf16 fp32", "bf16 bf16"])
def test_lookup_is_the_plain_form_bit_for_bit(enc, n, vocab, dim, types):
    import torch
    tt, to = (dict(fp32=torch.float32, bf16=torch.bfloat16)[x] for x in types.split())
    rng = np.random.Generator(np.random.PCG64(n + dim))
    table = torch.from_numpy(rng.standard_normal((vocab, dim)).astype(np.float32)).cuda().to(tt)
    for kind, scale in (("even", 1.0), ("pads", 11.3)):
        ids = torch.from_numpy(ids_of(rng, n, vocab, kind)).cuda()
        got = enc.embedding(table, ids, scale=scale, dtype=to)
        inside = (ids >= 0) & (ids < vocab)
        rows = table[ids.long().clamp(0, vocab - 1)].float() * np.float32(scale)
        want = torch.where(inside[:, None], rows, torch.zeros_like(rows)).to(to)
        torch.cuda.synchronize()
        assert torch.equal(got, want), kind


@pytest.mark.parametrize("offset", [0, 1, 3])
def test_lookup_of_rows_apart_and_at_any_address(enc, offset):
    import torch
    rng = np.random.Generator(np.random.PCG64(5))
    n, vocab, dim, ld, lo = 37, 11, 70, 75, 83
    for tt, to in ((torch.float32, torch.bfloat16), (torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32)):
        mem = torch.from_numpy(rng.standard_normal(offset + vocab * ld).astype(np.float32)).cuda().to(tt)
        table = mem[offset:].view(vocab, ld)[:, :dim]
        ids = torch.from_numpy(ids_of(rng, n, vocab, "pads")).cuda()
        outm = torch.full((offset + n * lo,), 7.0, device="cuda", dtype=to)
        out = outm[offset:].view(n, lo)[:, :dim]
        assert enc.embedding(table, ids, scale=2.5, out=out) is out
        rows = torch.where(((ids >= 0) & (ids < vocab))[:, None], table[ids.long().clamp(0, vocab - 1)].float() * 2.5, 0.0).to(to)
        torch.cuda.synchronize()
        assert torch.equal(out, rows)
        assert (outm[:offset] == 7).all() and (outm[offset:].view(n, lo)[:, dim:] == 7).all()


def check_gradient(dout, ids, before, after, scale):
    import torch
    vocab = before.shape[0]
    inside = (ids >= 0) & (ids < vocab)
    d, i = dout.double().cpu()[inside.cpu()], ids.long().cpu()[inside.cpu()]
    want = before.double().cpu().index_add(0, i, scale * d)
    size = torch.zeros_like(want).index_add_(0, i, abs(scale) * d.abs())
    k = torch.bincount(i, minlength=vocab).double()[:, None]
    bound = (k + 2) * U * size + 2 * U * (before.double().cpu().abs() + size)
    got = after.double().cpu()
    off = (got - want).abs()
    assert (off <= bound).all(), float((off / bound.clamp(min=1e-300)).max())
    untouched = (k[:, 0] == 0)
    assert torch.equal(after.cpu()[untouched], before.cpu()[untouched])


@pytest.mark.parametrize("n,vocab,dim", SHAPES)
@pytest.mark.parametrize("type", ["fp32", "bf16"])
@pytest.mark.parametrize("kind", ["even", "tail", "one", "pads", "up"])
def test_gradient_against_64_bits(enc, n, vocab, dim, type, kind):
    import torch
    dt = dict(fp32=torch.float32, bf16=torch.bfloat16)[type]
    rng = np.random.Generator(np.random.PCG64(n * 3 + dim))
    dout = torch.from_numpy(rng.standard_normal((n, dim)).astype(np.float32)).cuda().to(dt)
    ids = torch.from_numpy(ids_of(rng, n, vocab, kind)).cuda()
    before = torch.from_numpy(rng.standard_normal((vocab, dim)).astype(np.float32)).cuda()
    scale = 1.7
    after = [enc.embedding_backward(dout, ids, before.clone(), scale=scale) for _ in range(2)]
    torch.cuda.synchronize()
    assert torch.equal(after[0], after[1])               # the same bits again
    check_gradient(dout, ids, before, after[0], np.float32(scale).item())


@pytest.mark.parametrize("n", [30000, 200003])
def test_gradient_of_many_ids(enc, n):
    """Runs over many windows, ids of three radix passes' width, blocks that sort several steps."""
    import torch
    rng = np.random.Generator(np.random.PCG64(n))
    for vocab, kind, type in ((1 << 21, "tail", torch.bfloat16), (2, "even", torch.float32), (50021, "tail", torch.float32)):
        dim = 12
        dout = torch.from_numpy(rng.standard_normal((n, dim)).astype(np.float32)).cuda().to(type)
        ids = torch.from_numpy(ids_of(rng, n, vocab, kind)).cuda()
        before = torch.zeros((vocab, dim), device="cuda")
        after = enc.embedding_backward(dout, ids, before.clone())
        torch.cuda.synchronize()
        check_gradient(dout, ids, before, after, 1.0)


def test_gradient_of_rows_apart_and_at_any_address(enc):
    import torch
    rng = np.random.Generator(np.random.PCG64(8))
    n, vocab, dim = 300, 13, 70
    for dt, offset in ((torch.bfloat16, 1), (torch.float32, 3)):
        dout = torch.from_numpy(rng.standard_normal(offset + n * 75).astype(np.float32)).cuda().to(dt)[offset:].view(n, 75)[:, :dim]
        mem = torch.from_numpy(rng.standard_normal(1 + vocab * 83).astype(np.float32)).cuda()
        keep = mem.clone()
        ids = torch.from_numpy(ids_of(rng, n, vocab, "pads")).cuda()
        table = mem[1:].view(vocab, 83)[:, :dim]
        before = table.clone()
        enc.embedding_backward(dout, ids, table, scale=0.3)
        torch.cuda.synchronize()
        check_gradient(dout, ids, before, table.contiguous(), float(np.float32(0.3)))
        assert mem[0] == keep[0] and torch.equal(mem[1:].view(vocab, 83)[:, dim:], keep[1:].view(vocab, 83)[:, dim:])


def test_gradient_is_that_of_the_lookup(enc):
    """The lookup is linear in the table: <dout, lookup(D)> = <gradient, D> for any change D of the table."""
    import torch
    rng = np.random.Generator(np.random.PCG64(2))
    n, vocab, dim, scale = 1500, 90, 36, 3.0
    ids = torch.from_numpy(ids_of(rng, n, vocab, "pads")).cuda()
    D = torch.from_numpy(rng.standard_normal((vocab, dim)).astype(np.float32)).cuda()
    dout = torch.from_numpy(rng.standard_normal((n, dim)).astype(np.float32)).cuda()
    a = (enc.embedding(D, ids, scale=scale).double() * dout.double())
    g = enc.embedding_backward(dout, ids, torch.zeros_like(D), scale=scale).double() * D.double()
    # the lookup's products are rounded once, the sums of up to n / vocab * 3 terms as above
    bound = U * float(a.abs().sum()) * (1 + 3 * n / vocab + 3)
    assert abs(float(a.sum()) - float(g.sum())) <= bound


def test_nothing_to_do_and_refusals(enc):
    import torch
    import paper_2304_14698_amd as xrl
    table = torch.ones((5, 8), device="cuda")
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    assert enc.embedding(table, none).shape == (0, 8)
    assert torch.equal(enc.embedding_backward(torch.zeros((0, 8), device="cuda"), none, table.clone()), table)
    pads = torch.full((2000,), -1, dtype=torch.int32, device="cuda")
    assert not enc.embedding(table, pads).any()
    assert torch.equal(enc.embedding_backward(torch.ones((2000, 8), device="cuda"), pads, table.clone()), table)
    ids = torch.zeros(3, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        enc.embedding(table, ids.long())
    with pytest.raises(ValueError):
        enc.embedding(table.half(), ids)
    with pytest.raises(ValueError):
        enc.embedding(table.T, ids)
    with pytest.raises(ValueError):
        enc.embedding(table, ids, out=torch.empty((3, 9), device="cuda"))
    with pytest.raises(ValueError):
        enc.embedding_backward(torch.ones((3, 8), device="cuda"), ids, table.bfloat16())
    with pytest.raises(ValueError):
        enc.embedding_backward(torch.ones((4, 8), device="cuda"), ids, table)
    p = lambda x: x.data_ptr()  # noqa: E731
    out = torch.full((3, 8), 7.0, device="cuda")
    lib, h = xrl.load_library(), enc.handle
    for args, code in (((None, p(table), 0, 8, 5, 8, p(ids), 3, 1.0, p(out), 0, 8), "NULL"),
                       ((h, None, 0, 8, 5, 8, p(ids), 3, 1.0, p(out), 0, 8), "NULL"),
                       ((h, p(table), 2, 8, 5, 8, p(ids), 3, 1.0, p(out), 0, 8), "UNSUPPORTED"),
                       ((h, p(table), 0, 7, 5, 8, p(ids), 3, 1.0, p(out), 0, 8), "SHAPE"),
                       ((h, p(table), 0, 8, 5, 8, p(ids), -1, 1.0, p(out), 0, 8), "SHAPE"),
                       ((h, p(table) + 2, 0, 8, 5, 8, p(ids), 3, 1.0, p(out), 0, 8), "SHAPE")):
        assert lib.xrl_embedding(*args) == xrl.ERR[code]
    for args, code in (((h, p(out), 0, 8, p(ids), 3, 5, 8, 1.0, None, 8), "NULL"),
                       ((h, p(out), 0, 8, p(ids), 1 << 27, 5, 8, 1.0, p(table), 8), "UNSUPPORTED"),
                       ((h, p(out), 3, 8, p(ids), 3, 5, 8, 1.0, p(table), 8), "UNSUPPORTED"),
                       ((h, p(out), 0, 8, p(ids), 3, 5, 8, 1.0, p(table), 4), "SHAPE")):
        assert lib.xrl_embedding_backward(*args) == xrl.ERR[code]
    torch.cuda.synchronize()
    assert (out == 7).all() and (table == 1).all()


@pytest.mark.parametrize("vocab", [1, 2, 3, 23, 24, 25, 40, 63, 64, 65])
@pytest.mark.parametrize("n,dim,type", [(1025, 1, "fp32"), (1100, 2, "bf16"), (3000, 127, "bf16"), (2500, 128, "fp32"), (40000, 65, "fp32"),
                                        (9000, 513, "bf16"), (150000, 9, "fp32")])
def test_gradient_of_small_tables(enc, vocab, n, dim, type):
    """Tables that fit a wave's LDS, at the sizes where that changes: every id, one id of many, most ids never met, padding."""
    import torch
    dt = dict(fp32=torch.float32, bf16=torch.bfloat16)[type]
    rng = np.random.Generator(np.random.PCG64(vocab * 7 + n))
    dout = torch.from_numpy(rng.standard_normal((n, dim)).astype(np.float32)).cuda().to(dt)
    before = torch.from_numpy(rng.standard_normal((vocab, dim)).astype(np.float32)).cuda()
    for kind in ("even", "one", "pads", "up", "none"):
        ids = torch.from_numpy(ids_of(rng, n, vocab, kind)).cuda()
        after = [enc.embedding_backward(dout, ids, before.clone(), scale=0.7) for _ in range(2)]
        torch.cuda.synchronize()
        assert torch.equal(after[0], after[1])
        check_gradient(dout, ids, before, after[0], float(np.float32(0.7)))


@pytest.mark.parametrize("kind", ["tail", "one", "pads", "none"])
@pytest.mark.parametrize("vocab", [70, 1023, 1024, 9001])
@pytest.mark.parametrize("n,dim,type", [(768, 1100, "fp32"), (769, 1100, "fp32"), (2048, 250, "fp32"), (2049, 250, "fp32"), (8191, 66, "bf16"),
                                        (8192, 130, "fp32"), (8193, 130, "fp32"), (12288, 513, "bf16"), (12289, 515, "bf16"), (16001, 70, "fp32")])
def test_gradient_where_its_ways_change(enc, n, dim, type, vocab, kind):
    """Squares of ids, ranks, one and two passes of the sort; rows apart, from an address that is no multiple of 16."""
    import torch
    dt = dict(fp32=torch.float32, bf16=torch.bfloat16)[type]
    rng = np.random.Generator(np.random.PCG64(vocab + n))
    g = torch.Generator(device="cuda").manual_seed(n + dim)
    dout = torch.randn(1 + n * (dim + 3), generator=g, device="cuda").to(dt)[1:].view(n, dim + 3)[:, :dim]
    before = torch.randn(vocab, dim, generator=g, device="cuda")
    ids = torch.from_numpy(ids_of(rng, n, vocab, kind)).cuda()
    after = [enc.embedding_backward(dout, ids, before.clone(), scale=-0.7) for _ in range(2)]
    torch.cuda.synchronize()
    assert torch.equal(after[0], after[1])
    check_gradient(dout, ids, before, after[0], float(np.float32(-0.7)))
