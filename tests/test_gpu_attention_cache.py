"""The paged cache: writing new tokens into it bit for bit, and their attention over it against the formulas in 64 bits (bounds: tests/attention_checks.py)."""
import math

import numpy as np
import pytest

from attention_checks import close, one_head

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


class Case:
    """A cache of which only the named slots have numbers: all others are NaN."""

    def __init__(self, seed, new, lengths, heads, kv, dim, page, type, spare=2, cols=None, layout="slots"):
        import torch
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.r = lambda *s: torch.randn(*s, generator=g, device="cuda").to(dtype(type))  # noqa: E731
        self.new, self.lengths, self.page = list(new), list(lengths), page
        n = sum(new)
        per = [-(-max(m, 0) // page) for m in lengths]
        self.cols = max(per + [1]) if cols is None else cols
        order = np.random.Generator(np.random.PCG64(seed)).permutation(sum(per) + spare)
        self.table = np.full((len(new), self.cols), -1, np.int64)
        at = 0
        for s, c in enumerate(per):
            self.table[s, :min(c, self.cols)] = order[at:at + c][:self.cols]
            at += c
        pages = len(order)
        shape = (pages, page, kv, dim) if layout == "slots" else (pages, kv, page, dim)
        make = lambda: torch.full(shape, math.nan, device="cuda", dtype=dtype(type))  # noqa: E731
        turn = (lambda x: x) if layout == "slots" else (lambda x: x.transpose(1, 2))
        self.kc, self.vc = turn(make()), turn(make())
        self.q, self.k, self.v = self.r(n, heads, dim), self.r(n, kv, dim), self.r(n, kv, dim)
        i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()  # noqa: E731
        self.q_ptr = i32(np.concatenate([[0], np.cumsum(new)]))
        self.t, self.n = i32(self.table), i32(lengths)
        # tokens that were there before
        for s, m in enumerate(lengths):
            old = max(m - new[s], 0)
            js = np.arange(old)
            js = js[js // page < self.cols]
            pg = self.table[s, js // page]
            ok = (pg >= 0) & (pg < pages)
            js, pg = js[ok], pg[ok]
            if len(js):
                a, b = torch.from_numpy(pg).cuda(), torch.from_numpy(js % page).cuda()
                self.kc[a, b] = self.r(len(js), kv, dim)
                self.vc[a, b] = self.r(len(js), kv, dim)

    def places(self, s, upto):
        """(pages, slots, positions) of sequence s's tokens that are there."""
        js = np.arange(max(upto, 0))
        js = js[js // self.page < self.cols]
        pg = self.table[s, js // self.page]
        ok = (pg >= 0) & (pg < self.kc.shape[0])
        return pg[ok], js[ok] % self.page, js[ok]

    def write(self, enc):
        import torch
        want_k, want_v = self.kc.clone(), self.vc.clone()
        row = 0
        for s, (n, m) in enumerate(zip(self.new, self.lengths)):
            for i in range(n):
                j = m - n + i
                if 0 <= j and j // self.page < self.cols and 0 <= self.table[s, j // self.page] < self.kc.shape[0]:
                    at = int(self.table[s, j // self.page]), j % self.page
                    want_k[at], want_v[at] = self.k[row], self.v[row]
                row += 1
        enc.cache_write(self.k, self.v, self.q_ptr, self.kc, self.vc, self.t, self.n)
        torch.cuda.synchronize()
        bits = torch.int16 if self.kc.dtype == torch.bfloat16 else torch.int32
        for a, b in ((self.kc, want_k), (self.vc, want_v)):
            assert torch.equal(a.contiguous().view(bits), b.contiguous().view(bits))

    def want(self, scale):
        import torch
        half = 2.0 ** -8 if self.q.dtype == torch.bfloat16 else 0.0
        out = [torch.full(self.q.shape, math.nan, dtype=torch.float64, device="cuda") for _ in range(2)]
        heads, kv = self.q.shape[1], self.k.shape[1]
        row = 0
        for s, (n, m) in enumerate(zip(self.new, self.lengths)):
            pg, sl, js = (torch.from_numpy(np.ascontiguousarray(x)).cuda() for x in self.places(s, m))
            K, V = self.kc[pg, sl].double(), self.vc[pg, sl].double()
            for i in range(n):
                see = js <= m - n + i
                for h in range(kv):
                    for e in range(h * heads // kv, (h + 1) * heads // kv):
                        one = one_head(self.q[row:row + 1, e].double(), K[see][:, h], V[see][:, h], False, scale, half)["out"]
                        for x, y in zip(out, one):
                            x[row, e] = y[0]
                row += 1
        return out

    def check(self, enc, scale=None, out=None):
        import torch
        self.write(enc)
        got = enc.cache_attention(self.q, self.q_ptr, self.kc, self.vc, self.t, self.n, scale=scale, out=out)
        again = enc.cache_attention(self.q, self.q_ptr, self.kc, self.vc, self.t, self.n, scale=scale)
        torch.cuda.synchronize()
        assert torch.equal(got, again)
        close(got, self.want(float(np.float32(self.q.shape[2] ** -0.5 if scale is None else scale))), "out")
        return got


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("dim", [1, 8, 20, 32, 40, 63, 64, 96, 128])
@pytest.mark.parametrize("page", [1, 7, 16, 64])
def test_dims_and_pages(enc, type, dim, page):
    Case(dim, [1, 2, 1, 3], [1, 40, 133, 200], 4, 2, dim, page, type).check(enc)


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("new,lengths", [([1], [1]), ([1], [5000]), ([1] * 40, [17 * i + 1 for i in range(40)]), ([5], [3]), ([0, 1, 0], [7, 9, 0]), ([40], [40]), ([130], [130]),
                                         ([70, 33], [300, 1000]), ([1, 1], [0, -5]), ([3, 260], [2000, 260]), ([1, 1, 1], [2, 30000, 9])])
@pytest.mark.parametrize("heads,kv", [(2, 2), (8, 1), (6, 2), (40, 1)])
def test_lengths_and_groups(enc, type, new, lengths, heads, kv):
    """From one token to long contexts, chunks, whole prompts, sequences of nothing, fewer tokens than new ones, groups that cross a tile."""
    got = Case(sum(new), new, lengths, heads, kv, 32, 16, type).check(enc)
    row = 0
    for n, m in zip(new, lengths):
        assert not got[row:row + min(n, max(0, n - max(m, 0)))].any()
        row += n


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("dim", [64, 128])
def test_many_sequences(enc, type, dim):
    rng = np.random.Generator(np.random.PCG64(dim))
    Case(1, [1] * 150, rng.integers(1, 400, 150).tolist(), 2, 1, dim, 16, type).check(enc)


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("dim", [32, 20])
def test_pages_that_are_not_there(enc, type, dim):
    """Ids outside the cache, in the middle and at the start, and tokens behind the table's columns: not written, and not counted."""
    c = Case(3, [2, 1, 1, 3], [100, 100, 90, 300], 4, 2, dim, 16, type, cols=8)
    c.table[0, 2], c.table[1, 0], c.table[2, 5] = -7, 2 ** 31 - 1, c.kc.shape[0]
    c.table[3, :] = -1
    import torch
    c.t.copy_(torch.from_numpy(c.table.astype(np.int32)))
    got = c.check(enc)
    assert not got[4:].any()


@pytest.mark.parametrize("type", TYPES)
def test_layouts_strides_and_shared_pages(enc, type):
    """Pages of heads outside slots, a table whose rows lie apart, queries that are a part of wider rows, results in rows apart, two sequences with one prefix."""
    import torch
    c = Case(5, [1, 4, 1], [50, 300, 77], 4, 2, 64, 16, type, layout="heads")
    c.table[2, :2] = c.table[1, :2]
    wide = torch.full((3, c.cols + 5), -1, dtype=torch.int32, device="cuda")
    wide[:, :c.cols] = torch.from_numpy(c.table.astype(np.int32)).cuda()
    c.t = wide[:, :c.cols]
    qkv = c.r(6, 8, 64)
    c.q, c.k, c.v = qkv[:, :4], qkv[:, 4:6], qkv[:, 6:]
    out = torch.full((6, 8, 67), 7.0, device="cuda", dtype=dtype(type))
    c.check(enc, out=out[:, ::2, 1:65])
    assert (out[:, 1::2] == 7).all() and (out[..., 0] == 7).all() and (out[..., 65:] == 7).all()
    # one cache that holds both, at odd places
    both = torch.full((30, 16, 2, 2, 33), math.nan, device="cuda", dtype=dtype(type))
    c = Case(6, [1, 2], [90, 200], 2, 2, 32, 16, type)
    for x, i in (("kc", 0), ("vc", 1)):
        both[:c.kc.shape[0], :, i, :, 1:] = getattr(c, x)
        setattr(c, x, both[:c.kc.shape[0], :, i, :, 1:])
    c.check(enc)


@pytest.mark.parametrize("type", TYPES)
def test_rows_of_no_sequence_are_left(enc, type):
    import torch
    c = Case(7, [3, 5], [30, 60], 2, 1, 32, 16, type)
    c.q_ptr += 2
    pad = lambda x: torch.cat([torch.full((2, *x.shape[1:]), math.nan, device="cuda", dtype=x.dtype), x, torch.full((4, *x.shape[1:]), math.nan, device="cuda", dtype=x.dtype)])  # noqa: E731
    q, k, v = pad(c.q), pad(c.k), pad(c.v)
    out = torch.full_like(q, 7.0)
    enc.cache_write(k, v, c.q_ptr, c.kc, c.vc, c.t, c.n)
    enc.cache_attention(q, c.q_ptr, c.kc, c.vc, c.t, c.n, out=out)
    torch.cuda.synchronize()
    assert (out[:2] == 7).all() and (out[10:] == 7).all()
    close(out[2:10], c.want(32 ** -0.5), "out")


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("new,length", [(40, 200), (3, 3000)])
def test_what_a_token_does_not_see_reaches_nothing(enc, type, new, length):
    import torch
    c = Case(8, [new, 1], [length, 50], 2, 1, 32, 16, type)
    c.write(enc)
    clean = enc.cache_attention(c.q, c.q_ptr, c.kc, c.vc, c.t, c.n)
    j = length - 2                                           # seen by the last two new tokens
    at = int(c.table[0, j // 16]), j % 16
    for x in (c.kc, c.vc):
        old = x[at].clone()
        x[at] = math.nan
        got = enc.cache_attention(c.q, c.q_ptr, c.kc, c.vc, c.t, c.n)
        torch.cuda.synchronize()
        x[at] = old
        assert torch.equal(got[:new - 2], clean[:new - 2]) and torch.equal(got[new:], clean[new:]) and got[new - 2:new].isnan().all()


def test_a_step_after_a_prompt_is_a_longer_prompt(enc):
    """Packed attention over a prompt, and the same through the cache: in chunks, then token by token."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(4)
    n, heads, kv, dim, page = 150, 4, 2, 64, 16
    r = lambda h: torch.randn(n, h, dim, generator=g, device="cuda")  # noqa: E731
    q, k, v = r(heads), r(kv), r(kv)
    whole = enc.attention(q, k, v, torch.tensor([0, n], dtype=torch.int32, device="cuda"))["out"]
    kc, vc = (torch.full((12, page, kv, dim), math.nan, device="cuda") for _ in range(2))
    table = torch.randperm(12, generator=g, device="cuda").int()[None, :10]
    at = 0
    for step in [100, 30, 1, 1, 1, 16, 1]:
        ptr = torch.tensor([0, step], dtype=torch.int32, device="cuda")
        length = torch.tensor([at + step], dtype=torch.int32, device="cuda")
        enc.cache_write(k[at:at + step], v[at:at + step], ptr, kc, vc, table, length)
        out = enc.cache_attention(q[at:at + step], ptr, kc, vc, table, length)
        torch.cuda.synchronize()
        assert (out - whole[at:at + step]).abs().max() < 1e-5
        at += step
    assert at == n


def test_refusals(enc):
    import torch
    import paper_2304_14698_amd as xrl
    c = Case(9, [1, 2], [20, 30], 4, 2, 32, 16, "bf16")
    args = (c.q, c.q_ptr, c.kc, c.vc, c.t, c.n)
    for scale in (0.0, -1.0, math.nan, math.inf):
        with pytest.raises(xrl.XrlError) as e:
            enc.cache_attention(*args, scale=scale)
        assert e.value.code == xrl.ERR["VALUE"]
    big = torch.zeros(3, 1, 130, device="cuda")
    cache = torch.zeros(2, 16, 1, 130, device="cuda")
    with pytest.raises(xrl.XrlError) as e:
        enc.cache_attention(big, c.q_ptr, cache, cache, c.t, c.n)
    assert e.value.code == xrl.ERR["UNSUPPORTED"]
    one = c.kc[:1].expand(8, 16, 2, 32)
    with pytest.raises(xrl.XrlError) as e:                   # every page the same memory: not to be written
        enc.cache_write(c.k, c.v, c.q_ptr, one, one, c.t, c.n)
    assert e.value.code == xrl.ERR["SHAPE"]
    for bad in (lambda: enc.cache_attention(c.q.float(), *args[1:]), lambda: enc.cache_attention(c.q[:, :3], *args[1:]), lambda: enc.cache_attention(*args[:4], c.t[:1], c.n),
                lambda: enc.cache_attention(*args[:4], c.t.long(), c.n), lambda: enc.cache_attention(*args[:5], c.n[:1]), lambda: enc.cache_attention(*args[:3], c.vc[:1], *args[4:]),
                lambda: enc.cache_attention(*args[:4], c.t.T, c.n), lambda: enc.cache_attention(c.q.cpu(), *args[1:]), lambda: enc.cache_write(c.k[:, :1], c.v, *args[1:]),
                lambda: enc.cache_write(c.k, c.v[:2], *args[1:]), lambda: enc.cache_attention(*args, out=c.q[:1])):
        with pytest.raises(ValueError):
            bad()
    empty = torch.zeros(0, 16, 2, 32, device="cuda", dtype=torch.bfloat16)
    out = enc.cache_attention(c.q, c.q_ptr, empty, empty, c.t, c.n)
    torch.cuda.synchronize()
    assert not out.any()


def test_recorded_in_a_graph():
    """Replays while lengths grow: a rollout whose steps are one graph."""
    import torch
    import paper_2304_14698_amd as xrl
    stream = torch.cuda.Stream()
    model = dict(n_op_types=4, n_node_dense=0, d_edge=4, d_global=0, hidden=64, rounds=0)
    c = Case(10, [1, 1, 1], [20, 500, 1000], 4, 2, 64, 16, "bf16", cols=80)
    spare = torch.arange(c.kc.shape[0], c.kc.shape[0] + 30, device="cuda", dtype=torch.int32).view(3, 10)
    grown = lambda x: torch.cat([x, torch.zeros(30, *x.shape[1:], device="cuda", dtype=x.dtype)])  # noqa: E731
    kc, vc = grown(c.kc), grown(c.vc)
    for s, m in enumerate(c.lengths):
        first = -(-m // 16)
        c.t[s, first:first + 10] = spare[s]
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        enc = xrl.Encoder(model, np.zeros(xrl.weight_count(model), np.float32))
        step = lambda: (enc.cache_write(c.k, c.v, c.q_ptr, kc, vc, c.t, c.n), enc.cache_attention(c.q, c.q_ptr, kc, vc, c.t, c.n, out=out))  # noqa: E731
        out = torch.empty_like(c.q)
        step()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            step()
        for replay in range(5):
            c.n.add_(1)
            c.k.mul_(-1.01)
            graph.replay()
            got = out.clone()
            want = enc.cache_attention(c.q, c.q_ptr, kc, vc, c.t, c.n)
            torch.zeros(1 << 20, device="cuda").add_(1.0).sum().item()
            assert torch.equal(got, want) and got.isfinite().all(), replay
        enc.close()


def test_a_cache_behind_two_to_the_31st(enc):
    """Offsets that pass 32 bits: 2.4e9 elements a tensor, pages at its end and its start."""
    import torch
    pages, page, kv, dim = 18500, 128, 8, 128
    g = torch.Generator(device="cuda").manual_seed(2)
    kc = torch.zeros(pages, page, kv, dim, device="cuda", dtype=torch.bfloat16)
    vc = torch.zeros_like(kc)
    table = torch.tensor([[pages - 1, 0, pages - 2, 5]], dtype=torch.int32, device="cuda")
    r = lambda n, h: torch.randn(n, h, dim, generator=g, device="cuda").bfloat16()  # noqa: E731
    k, v, q = r(400, kv), r(400, kv), r(400, 16)
    ptr, n = torch.tensor([0, 400], dtype=torch.int32, device="cuda"), torch.tensor([400], dtype=torch.int32, device="cuda")
    enc.cache_write(k, v, ptr, kc, vc, table, n)
    out = enc.cache_attention(q[399:], torch.tensor([0, 1], dtype=torch.int32, device="cuda"), kc, vc, table, n)
    torch.cuda.synchronize()
    assert torch.equal(kc[pages - 1], k[:128]) and torch.equal(vc[0], v[128:256]) and torch.equal(kc[pages - 2], k[256:384]) and torch.equal(vc[5, :16], v[384:])
    for e in range(16):
        close(out[:, e], one_head(q[399:, e].double(), k[:, e // 2].double(), v[:, e // 2].double(), False, 128 ** -0.5, 2.0 ** -8)["out"], e)
