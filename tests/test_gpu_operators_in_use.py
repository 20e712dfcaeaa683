"""The operators over a vocabulary as a program uses them: recorded in a graph, on a stream that is not torch's current one, in tensors of
more than 2^31 entries, and in sums that the listed tests do not reach. Tolerances as in their own tests."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def encoder(**kw):
    import paper_2304_14698_amd as xrl
    model = dict(n_op_types=4, n_node_dense=0, d_edge=4, d_global=0, hidden=64, rounds=0)
    return xrl.Encoder(model, np.zeros(xrl.weight_count(model), np.float32), **kw)


def everything(enc, s, out=None):
    """One pass through all operators; results as a list."""
    import torch
    e = enc.embedding(s["table"], s["ids"], scale=2.0, out=out and out["e"])
    f = enc.token_logp(s["logits"], s["given"], top_k=5, out=out and out["f"])
    d = enc.token_logp_backward(s["logits"], s["given"], f, s["dlogp"], s["dent"], out=out and out["d"])
    enc.embedding_backward(s["dout"], s["ids"], s["dtable"], scale=2.0)
    enc.embedding_backward(s["dout"][:500], s["ids"][:500], s["dtable"])
    enc.muon_step(s["W"], s["G"], s["M"], s["mats"], lr=0.02)
    enc.muon_step(s["W"], s["G"], s["M"], s["small"], lr=0.02)
    return dict(e=e, f=f, d=d)


def state(seed):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    randn = lambda *n: torch.randn(*n, generator=g, device="cuda")  # noqa: E731
    ids = lambda n, v: torch.randint(-1, v, (n,), generator=g, device="cuda").int()  # noqa: E731
    mats = np.array([(0, 300, 128), (38400, 70, 3000)])
    return dict(table=randn(900, 72), ids=ids(5000, 900), logits=randn(6, 9000).bfloat16(), given=ids(6, 9000), dlogp=randn(6), dent=randn(6),
                dout=randn(5000, 72), dtable=randn(900, 72), W=randn(260000), G=randn(260000), M=randn(260000), mats=mats,
                small=np.array([(248400, 33, 100)]))


def flat(s, out):
    return [out["e"], out["d"], s["dtable"], s["W"], s["M"]] + [out["f"][k] for k in sorted(out["f"])]


def test_recorded_in_a_graph():
    """Replays against eager calls on copies, with eager work of the program and of the library in between."""
    import torch
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        enc, s, eager = encoder(), state(1), state(1)
        out = everything(enc, s)                               # (the workspace grows to its size)
        everything(enc, eager)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            everything(enc, s, out)
        for replay in range(4):
            graph.replay()
            want = everything(enc, eager)
            stream.synchronize()
            for a, b in zip(flat(s, out), flat(eager, want)):
                assert torch.equal(a, b), replay
            # a call that needs a larger workspace leaves the graph's in place
            if replay == 1:
                big = torch.randn(100000, 64, device="cuda")
                at = torch.randint(0, 50, (100000,), device="cuda").int()
                enc.embedding_backward(big, at, torch.zeros(50, 64, device="cuda"))
            torch.zeros(1 << 20, device="cuda").add_(1.0).sum().item()
        enc.close()


def test_a_workspace_that_would_have_to_grow_is_refused_in_a_capture():
    import torch
    import paper_2304_14698_amd as xrl
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        enc = encoder()
        dout, ids, dtable = torch.ones(5000, 64, device="cuda"), torch.zeros(5000, dtype=torch.int32, device="cuda"), torch.zeros(9, 64, device="cuda")
        stream.synchronize()
        graph, code = torch.cuda.CUDAGraph(), None
        with torch.cuda.graph(graph, stream=stream):
            dtable.mul_(1.0)
            try:
                enc.embedding_backward(dout, ids, dtable)
            except xrl.XrlError as e:
                code = e.code
        assert code == xrl.ERR["HIP"]
        graph.replay()                                         # what was recorded around it stands
        enc.embedding_backward(dout, ids, dtable)              # and outside it the call works
        stream.synchronize()
        assert (dtable[0] == 5000).all() and not dtable[1:].any()
        enc.close()


def test_on_a_stream_of_its_own():
    import torch
    side = torch.cuda.Stream()
    enc, here = encoder(stream=side), encoder()
    s, t = state(3), state(3)
    torch.cuda.synchronize()
    a, b = everything(enc, s), everything(here, t)
    torch.cuda.synchronize()
    for x, y in zip(flat(s, a), flat(t, b)):
        assert torch.equal(x, y)
    enc.close()
    here.close()


def test_entries_behind_two_to_the_31st():
    import torch
    enc = encoder()
    rows, dim = (1 << 20) + 3, 2100                            # 2.2e9 entries of a table, and of a gradient
    table = torch.zeros((rows, dim), dtype=torch.bfloat16, device="cuda")
    table[-1] = torch.arange(dim, device="cuda").bfloat16()
    ids = torch.tensor([rows - 1, 0, rows - 1], dtype=torch.int32, device="cuda")
    got = enc.embedding(table, ids)
    torch.cuda.synchronize()
    assert torch.equal(got[0], table[-1]) and torch.equal(got[2], table[-1]) and not got[1].any()
    at = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
    at[-1], at[5] = 2, 2
    dtable = torch.zeros((3, dim), device="cuda")
    enc.embedding_backward(table, at, dtable)
    torch.cuda.synchronize()
    assert torch.equal(dtable[2], table[-1].float()) and not dtable[:2].any()
    del got, dtable
    logits = table                                             # the same memory as rows of logits
    given = torch.full((rows,), 7, dtype=torch.int32, device="cuda")
    first = int((table[-1] == table[-1].max()).nonzero()[0])   # (bf16 holds several of the arange as one value)
    f = enc.token_logp(logits, given, top_k=1)
    d = enc.token_logp_backward(logits, given, f, torch.ones(rows, device="cuda"), out=logits)
    torch.cuda.synchronize()
    assert abs(float(f["logp"][0]) + math.log(dim)) < 1e-4 and int(f["top_ids"][-1, 0]) == first
    assert abs(float(d[0, 7]) - (1 - 1 / dim)) < 1e-2 and float(d[-2, 8]) == float(torch.tensor(-1 / dim).bfloat16())
    assert float(d[-1, 7]) == 1.0 and float(d[-1, 8]) <= 0.0
    del table, logits, d, f
    torch.cuda.empty_cache()
    # a matrix behind two to the 31st of the flat vector
    n = (1 << 31) + 5000
    W, G, M = (torch.zeros(n, device="cuda") for _ in range(3))
    G[-4000:] = torch.randn(4000, device="cuda")
    enc.muon_step(W, G, M, [(n - 4000, 40, 100)], lr=1.0, beta=0.0, nesterov=False, rms=0.1)
    torch.cuda.synchronize()
    sv = torch.linalg.svdvals(W[-4000:].view(40, 100).double().cpu())
    assert not W[:-4000].any() and float(sv.min()) > 0.6 and float(sv.max()) < 1.3
    enc.close()


@pytest.mark.parametrize("shapes", [[(1, 2342)], [(2859, 89), (70, 3001)], [(700, 1500)], [(2049, 2100)], [(2990, 300), (2960, 2960)], [(33, 513), (513, 64), (64, 514)]])
def test_long_sums_and_many_tiles_of_the_update(shapes):
    """Sums cut into parts, tiles of both sizes and their edges, matrices just over what one block takes: against 64 bits on the GPU."""
    import torch
    enc = encoder()
    g = torch.Generator(device="cuda")
    g.manual_seed(sum(r * c for r, c in shapes))
    mats, at = [], 0
    for r, c in shapes:
        mats.append((at, r, c))
        at += r * c
    W, G, M = (torch.randn(at, generator=g, device="cuda") for _ in range(3))
    w0, m0 = W.double(), M.double()
    copies = [x.clone() for x in (W, G, M)]
    enc.muon_step(W, G, M, mats, lr=0.02, weight_decay=0.1)
    enc.muon_step(*copies, mats, lr=0.02, weight_decay=0.1)
    torch.cuda.synchronize()
    assert torch.equal(W, copies[0]) and torch.equal(M, copies[2])
    f = lambda v: float(np.float32(v))  # noqa: E731
    a, b, c5 = 3.4445, -4.7750, 2.0315
    for o, r, c in mats:
        s = slice(o, o + r * c)
        m = f(0.95) * m0[s] + G[s].double()
        assert ((M[s].double() - m).abs() <= 2.0 ** -23 * (G[s].abs() + m0[s].abs())).all()
        x = (G[s].double() + f(0.95) * m).view(r, c)
        x = x / (x.norm() + 1e-7)
        x = x.T if r > c else x
        for _ in range(5):
            k = x @ x.T
            x = a * x + (b * k + c5 * (k @ k)) @ x
        update = f(0.02) * f(0.2) * math.sqrt(max(r, c)) * (x.T if r > c else x).reshape(-1)
        want = (1 - f(0.02) * f(0.1)) * w0[s] - update
        off = float((W[s].double() - want).norm())
        assert off <= 3 * 2.0 ** -22 * a ** 5 * float(update.norm()) + 3 * 2.0 ** -24 * float(w0[s].norm()), (r, c)
    enc.close()


def test_rows_of_few_and_of_many_parts():
    """Log-probabilities in every way the rows are shared out: by waves, by blocks, in parts of a wave and of a block."""
    import torch
    enc = encoder()
    g = torch.Generator(device="cuda")
    g.manual_seed(9)
    for rows, cols in ((1, 131072), (1, 131073), (40, 30000), (300, 9000), (1500, 5000), (7, 400001), (5000, 1024)):
        x = torch.randn(rows, cols, generator=g, device="cuda").bfloat16()
        ids = torch.randint(0, cols, (rows,), generator=g, device="cuda").int()
        f = enc.token_logp(x, ids, top_k=3)
        torch.cuda.synchronize()
        lp = torch.log_softmax(x.double(), 1)
        n = (3 * (cols / 64 + 8) + 64 + 4 * math.log2(cols)) * 2.0 ** -24
        assert (f["logp"].double() - lp.gather(1, ids.long()[:, None])[:, 0]).abs().max() <= n + 6 * 2.0 ** -24 * 40
        best = x.float().sort(dim=1, descending=True, stable=True)
        assert torch.equal(f["top_ids"].long(), best[1][:, :3]), (rows, cols)
    enc.close()


@pytest.mark.parametrize("type", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,cols,k", [(1700, 2049, 0), (1700, 4097, 0), (1700, 8191, 2), (1700, 8193, 2), (1400, 4000, 2), (3, 8192, 5), (3, 8193, 5),
                                         (3, 40960, 0), (3, 40961, 0), (400, 41000, 0), (5, 200000, 0), (5, 131073, 5)])
def test_rows_where_their_ways_change(type, rows, cols, k):
    """Waves of several steps, blocks uncut and cut, with their gradient: against 64 bits."""
    import torch
    enc = encoder()
    g = torch.Generator(device="cuda").manual_seed(cols)
    x = torch.randn(rows, cols, generator=g, device="cuda").to(dict(fp32=torch.float32, bf16=torch.bfloat16)[type])
    ids = torch.randint(0, cols, (rows,), generator=g, device="cuda").int()
    f = enc.token_logp(x, ids, top_k=k)
    dlogp = torch.ones(rows, device="cuda")
    d = enc.token_logp_backward(x, ids, f, dlogp)
    torch.cuda.synchronize()
    u, at = 2.0 ** -24, ids.long()[:, None]
    D = (3 * (cols / 64 + 8) + 64 + 4 * math.log2(cols)) * u
    for r in range(0, rows, 200):                        # a part of the rows at a time: they are held in 64 bits
        s = slice(r, r + 200)
        lp = torch.log_softmax(x[s].double(), 1)
        assert (f["logp"][s].double() - lp.gather(1, at[s])[:, 0]).abs().max() <= D + 6 * u * 40
        H = -(lp.exp() * lp).sum(1)
        assert (f["entropy"][s].double() - H).abs().max() <= D * (1 + 2 * (math.log(cols) + 12)) + 8 * u * 24
        if k:
            assert torch.equal(f["top_ids"][s].long(), x[s].float().sort(dim=1, descending=True, stable=True)[1][:, :k])
        want = -lp.exp()
        want.scatter_add_(1, at[s], torch.ones_like(at[s], dtype=torch.float64))
        bound = want.abs() * (2 * D + (24 + 8 * lp.abs()) * u + (2.0 ** -8 if type == "bf16" else 0)) + 16 * u * (want > 0) + 1e-38
        assert ((d[s].double() - want).abs() <= bound).all()
    enc.close()


@pytest.mark.parametrize("type,cols", [("fp32", 1023), ("fp32", 1024), ("fp32", 1025), ("bf16", 2047), ("bf16", 2048), ("bf16", 2049), ("bf16", 131)])
@pytest.mark.parametrize("rows", [1, 3, 4, 5, 1001])
def test_gradient_of_rows_by_waves_and_by_blocks(rows, type, cols):
    """The last rows of a block of four, in place and into rows apart: as in float64."""
    import torch
    enc = encoder()
    g = torch.Generator(device="cuda").manual_seed(cols + rows)
    x = torch.randn(rows, cols, generator=g, device="cuda").to(dict(fp32=torch.float32, bf16=torch.bfloat16)[type])
    ids = torch.randint(0, cols, (rows,), generator=g, device="cuda").int()
    f, dlogp = enc.token_logp(x, ids), torch.ones(rows, device="cuda")
    wide = torch.full((rows, cols + 3), 7.0, device="cuda").to(x.dtype)
    enc.token_logp_backward(x, ids, f, dlogp, out=wide[:, :cols])
    y = x.clone()
    enc.token_logp_backward(y, ids, f, dlogp, out=y)
    torch.cuda.synchronize()
    assert torch.equal(y, wide[:, :cols]) and (wide[:, cols:] == 7).all()
    lp, at = torch.log_softmax(x.double(), 1), ids.long()[:, None]
    want = -lp.exp()
    want.scatter_add_(1, at, torch.ones_like(at, dtype=torch.float64))
    u = 2.0 ** -24
    D = (3 * (cols / 64 + 8) + 64 + 4 * math.log2(cols)) * u
    bound = want.abs() * (2 * D + (24 + 8 * lp.abs()) * u + (2.0 ** -8 if type == "bf16" else 0)) + 16 * u * (want > 0) + 1e-38
    assert ((y.double() - want).abs() <= bound).all()
    enc.close()
