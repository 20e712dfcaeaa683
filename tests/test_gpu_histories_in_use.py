"""The operators over histories as a program uses them together: a rollout token by token over a paged cache with entries drawn of each step's logits, the update over
the same histories packed, recorded in graphs that share a workspace, and on a stream of its own."""
import math

import numpy as np
import pytest

from test_gpu_token_sample import check, draw

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
INF = math.inf
HEADS, KV, DIM, VOCAB, PAGE = 6, 2, 40, 700, 7


def encoder(**kw):
    import paper_2304_14698_amd as xrl
    model = dict(n_op_types=4, n_node_dense=0, d_edge=4, d_global=0, hidden=64, rounds=0)
    return xrl.Encoder(model, np.zeros(xrl.weight_count(model), np.float32), **kw)


def policy(seed, dtype=None):
    """A policy of one layer: tables of a token's query, key and value, weights of the norms, and rows of logits (in 64 bits, so that a step's and a history's agree)."""
    import torch
    import paper_2304_14698_amd as xrl
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *n: torch.randn(*n, generator=g, device="cuda")  # noqa: E731
    t = dtype or torch.float32
    return dict(q=r(VOCAB, HEADS * DIM).to(t), k=r(VOCAB, KV * DIM).to(t), v=r(VOCAB, KV * DIM).to(t), wq=1 + 0.1 * r(DIM), wk=1 + 0.1 * r(DIM),
                head=r(HEADS * DIM, VOCAB).double() / 4, freqs=torch.from_numpy(xrl.rotary_freqs(DIM, factor=4.0, length=30.0)).cuda())


def qkv(enc, p, ids, positions):
    q, k, v = (enc.embedding(p[x], ids).view(len(ids), -1, DIM) for x in "qkv")
    raw = q, k
    q, k = enc.head_rotary(q, k, positions, p["freqs"], q_weight=p["wq"], k_weight=p["wk"])
    return q, k, v, raw


def logits_of(p, out):
    return (out.double().flatten(1) @ p["head"]).float()


def test_a_rollout_and_the_update_over_its_histories():
    """Log-probabilities of the drawn entries, step by step over the cache and over the packed histories: the same to twice what one may be off by; and the gradients of
    a loss of them, down to the tables, against 64 bits."""
    import torch
    enc, p = encoder(), policy(1)
    i32 = dict(dtype=torch.int32, device="cuda")
    prompts = [3, 1, 40, 9, 65]
    steps, n = 12, len(prompts)
    g = torch.Generator(device="cuda").manual_seed(2)
    histories = [torch.randint(0, VOCAB, (m,), generator=g, device="cuda").int() for m in prompts]
    most = max(prompts) + steps
    cols = -(-most // PAGE)
    table = torch.randperm(n * cols, generator=g, device="cuda").int().view(n, cols)
    cache = [torch.full((n * cols, PAGE, KV, DIM), math.nan, device="cuda") for _ in range(2)]
    lengths = torch.tensor(prompts, **i32)
    ends = lambda x: torch.tensor(np.concatenate([[0], np.cumsum(x)]), **i32)  # noqa: E731
    new, logp = histories, []
    drawn = []
    for step in range(steps):
        counts = [len(x) for x in new]
        ids, ptr = torch.cat(new), ends(counts)
        at = torch.cat([torch.arange(int(m) - c, int(m), **i32) for m, c in zip(lengths, counts)])
        q, k, v, _ = qkv(enc, p, ids, at)
        enc.cache_write(k, v, ptr, *cache, table=table, lengths=lengths)
        out = enc.cache_attention(q, ptr, *cache, table=table, lengths=lengths, scale=DIM ** -0.5)
        rows = logits_of(p, out[ptr[1:].long() - 1])
        got = enc.token_sample(rows, torch.rand(n, generator=g, device="cuda"), top_k=50, top_p=0.95)
        drawn.append(got["ids"])
        logp.append(got["logp"])
        new = [got["ids"][i:i + 1] for i in range(n)]
        histories = [torch.cat([h, x]) for h, x in zip(histories, new)]
        lengths += 1
    logp, drawn = torch.stack(logp, 1), torch.stack(drawn, 1)
    assert (drawn >= 0).all()
    # the same histories, all rows at once: row `prompt - 1 + step` of each gave step's logits
    ids = torch.cat([h[:-1] for h in histories])
    counts = [len(h) - 1 for h in histories]
    ptr = ends(counts)
    at = torch.cat([torch.arange(c, **i32) for c in counts])
    q, k, v, raw = qkv(enc, p, ids, at)
    f = enc.attention(q, k, v, ptr, scale=DIM ** -0.5)
    rows = torch.cat([int(ptr[i]) + m - 1 + torch.arange(steps, device="cuda") for i, m in enumerate(prompts)])
    x = logits_of(p, f["out"][rows])
    given = enc.token_logp(x, drawn.flatten())
    torch.cuda.synchronize()
    # one side's out, by attention's bounds: probabilities are off by 2 (rel + (m + 16) u) of themselves, rel = (dim + 4) u of the scores' sizes + 16 u + 8 u of the scores
    size = DIM ** -0.5 * float((q.abs().amax(0).amax(0) * k.abs().amax(0).amax(0)).sum())
    rel = 2 * ((DIM + 4 + 8) * U * size + 24 * U + (most + 16) * U)
    off = rel * float(v.abs().max()) * float(p["head"].abs().sum(0).max())
    own = (3 * (VOCAB / 64 + 8) + 64 + 4 * math.log2(VOCAB)) * U + 6 * U * 40
    assert (given["logp"].view(n, steps) - logp).abs().max() <= 2 * (2 * off + 2 * U * float(x.abs().max()) + own)
    # the update
    dlogp, dent = (torch.randn(n * steps, generator=g, device="cuda") for _ in range(2))
    dx = enc.token_logp_backward(x, drawn.flatten(), given, dlogp, dent)
    dout = torch.zeros_like(f["out"])
    dout[rows] = (dx.double() @ p["head"].T).float().view(-1, HEADS, DIM)
    dq, dk, dv = enc.attention_backward(q, k, v, ptr, f, dout, scale=DIM ** -0.5)
    dw = [torch.zeros(DIM, device="cuda") for _ in range(2)]
    dq, dk = enc.head_rotary_backward(*raw, at, p["freqs"], dq, dk, dq_weight=dw[0], dk_weight=dw[1], q_weight=p["wq"], k_weight=p["wk"])
    tables = [torch.zeros_like(p[x]) for x in "qkv"]
    for d, to in zip((dq, dk, dv), tables):
        enc.embedding_backward(d.reshape(len(ids), -1), ids, to)
    torch.cuda.synchronize()
    # in 64 bits, by automatic differentiation on the host
    leaves = [p[x].double().cpu().requires_grad_() for x in ("q", "k", "v", "wq", "wk")]
    angle = at.cpu().double()[:, None, None] * p["freqs"].cpu().double()

    def turned(y, w):
        y = y * w / (y.square().mean(-1, keepdim=True) + float(np.float32(1e-6))).sqrt()
        a, b = y[..., :DIM // 2], y[..., DIM // 2:]
        return torch.cat([a * angle.cos() - b * angle.sin(), a * angle.sin() + b * angle.cos()], -1)
    at_ids = ids.cpu().long()
    Q, K, V = (leaves[i][at_ids].view(len(ids), -1, DIM) for i in range(3))
    Q, K = turned(Q, leaves[3]), turned(K, leaves[4])
    outs = []
    for a, b in zip(ptr[:-1].tolist(), ptr[1:].tolist()):
        for h in range(HEADS):
            s = float(np.float32(DIM ** -0.5)) * Q[a:b, h] @ K[a:b, h * KV // HEADS].T
            s = s.masked_fill(torch.ones(b - a, b - a).tril() == 0, -math.inf)
            outs.append(s.softmax(1) @ V[a:b, h * KV // HEADS])
    outs = torch.cat([torch.stack(outs[i:i + HEADS], 1) for i in range(0, len(outs), HEADS)])
    lp = (outs[rows.cpu()].flatten(1) @ p["head"].cpu()).log_softmax(1)
    loss = (lp.gather(1, drawn.flatten().cpu().long()[:, None])[:, 0] * dlogp.cpu().double()).sum() - ((lp.exp() * lp).sum(1) * dent.cpu().double()).sum()
    loss.backward()
    # five operators, each of which adds at most (its longest sum + 64) u of the sizes that it sums; differences among these cost at most another 2^4
    bound = 16 * U * (5 * 64 + DIM + most + 2 * DIM + VOCAB / 64 + HEADS * DIM + len(ids))
    for leaf, got, name in zip(leaves, tables + dw, ("q", "k", "v", "wq", "wk")):
        off = float((got.double().cpu() - leaf.grad).norm() / leaf.grad.norm())
        assert off <= bound, (name, off, bound)
    enc.close()


def test_gradients_in_bf16_lose_little():
    """Relative errors over whole gradients against 64 bits. A result rounded once has at most 2^-8 / sqrt(3) (a value's error is even over half a step that is at most 2^-8 of it); so has
    each factor of a product that is rounded once, which errors of signs of their own carry over to the sum. dv has two such roundings (p, dv), dk has ds and its own, and
    dq its own and that of out in D: no more than twice the one."""
    import torch
    enc = encoder()
    g = torch.Generator(device="cuda").manual_seed(5)
    n, dim = 700, 64
    q, k, v, dout = (torch.randn(n, 2, dim, generator=g, device="cuda").bfloat16() for _ in range(4))
    ptr = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    f = enc.attention(q, k, v, ptr, scale=0.125)
    got = enc.attention_backward(q, k, v, ptr, f, dout, scale=0.125)
    torch.cuda.synchronize()
    leaves = [x.double().cpu().requires_grad_() for x in (q, k, v)]
    for h in range(2):
        s = 0.125 * leaves[0][:, h] @ leaves[1][:, h].T
        out = s.masked_fill(torch.ones(n, n).tril() == 0, -math.inf).softmax(1) @ leaves[2][:, h]
        (out * dout[:, h].double().cpu()).sum().backward()
    for x, leaf, name in zip(got, leaves, ("dq", "dk", "dv")):
        off = float((x.double().cpu() - leaf.grad).norm() / leaf.grad.norm())
        assert off <= 2 * 2.0 ** -8 / math.sqrt(3), (name, off)
    enc.close()


def everything(enc, p, s, out=None):
    """One pass through all operators, for single new tokens and for a history; out: an earlier pass's results, written again."""
    o = out or dict.fromkeys(("step", "c", "ids", "qk", "f", "d", "back"))
    step = enc.head_rotary(s["q1"], s["k1"], s["at1"], p["freqs"], q_weight=p["wq"], k_weight=p["wk"], out=o["step"])
    how = dict(table=s["table"], lengths=s["lengths"])
    enc.cache_write(step[1], s["v1"], s["ptr1"], s["kc"], s["vc"], **how)
    c = enc.cache_attention(step[0], s["ptr1"], s["kc"], s["vc"], scale=0.2, out=o["c"], **how)
    ids = enc.token_sample(s["logits"], s["u"], top_k=9, out=o["ids"])
    qk = enc.head_rotary(s["q"], s["k"], s["at"], p["freqs"], q_weight=p["wq"], k_weight=p["wk"], out=o["qk"])
    f = enc.attention(*qk, s["v"], s["ptr"], scale=0.2, out=o["f"])
    d = enc.attention_backward(*qk, s["v"], s["ptr"], f, s["dout"], scale=0.2, out=o["d"])
    back = enc.head_rotary_backward(s["q"], s["k"], s["at"], p["freqs"], d[0], d[1], dq_weight=s["dwq"], dk_weight=s["dwk"], q_weight=p["wq"], k_weight=p["wk"], out=o["back"])
    return dict(step=step, c=c, ids=ids, qk=qk, f=f, d=d, back=back)


def state(seed, dtype, seqs=5, keys=900, rows=500):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *n: torch.randn(*n, generator=g, device="cuda").to(dtype)  # noqa: E731
    i = lambda *n, high: torch.randint(0, high, n, generator=g, device="cuda").int()  # noqa: E731
    cols = -(-keys // PAGE)
    return dict(q1=r(seqs, HEADS, DIM), k1=r(seqs, KV, DIM), v1=r(seqs, KV, DIM), at1=i(seqs, high=5000), ptr1=torch.arange(seqs + 1, dtype=torch.int32, device="cuda"),
                table=torch.randperm(seqs * cols, generator=g, device="cuda").int().view(seqs, cols), lengths=keys // 2 + i(seqs, high=keys // 2) + 1,
                kc=r(seqs * cols, PAGE, KV, DIM), vc=r(seqs * cols, PAGE, KV, DIM), logits=r(4, 20000), u=torch.rand(4, generator=g, device="cuda"),
                q=r(rows, HEADS, DIM), k=r(rows, KV, DIM), v=r(rows, KV, DIM), at=i(rows, high=5000), dout=r(rows, HEADS, DIM),
                ptr=torch.tensor([0, 3, 3, rows // 2, rows], dtype=torch.int32, device="cuda"), dwq=r(DIM).float(), dwk=r(DIM).float())


def flat(s, out):
    return [s[x] for x in ("kc", "vc", "dwq", "dwk")] + [*out["step"], out["c"], out["ids"]["ids"], out["ids"]["logp"], *out["qk"], out["f"]["out"], out["f"]["lse"], *out["d"],
                                                         *out["back"]]


@pytest.mark.parametrize("type", ["fp32", "bf16"])
def test_two_graphs_that_share_a_workspace(type):
    """Two recorded passes of one context over other sizes, replayed in turn with eager passes in between: every replay equals the eager results."""
    import torch
    t = dict(fp32=torch.float32, bf16=torch.bfloat16)[type]
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        enc, p = encoder(), policy(3)
        sizes = [dict(seqs=5, keys=900, rows=500), dict(seqs=9, keys=300, rows=77)]
        states, eager = ([state(7 + i, t, **z) for i, z in enumerate(sizes)] for _ in range(2))
        outs = [everything(enc, p, s) for s in states]          # (the workspace grows to its size)
        for e in eager:
            everything(enc, p, e)
        stream.synchronize()
        graphs = [torch.cuda.CUDAGraph() for _ in sizes]
        for g, s, o in zip(graphs, states, outs):
            with torch.cuda.graph(g, stream=stream):
                everything(enc, p, s, o)
        for replay in range(4):
            for s, e in zip(states, eager):                     # other inputs in the same memory
                for x in (s, e):
                    x["lengths"].sub_(1)
                    x["q1"].mul_(0.5)
                    x["q"].mul_(-1.0)
            for g in graphs:
                g.replay()
            want = [everything(enc, p, e) for e in eager]
            stream.synchronize()
            for i in range(2):
                for k, (a, b) in enumerate(zip(flat(states[i], outs[i]), flat(eager[i], want[i]))):
                    assert torch.equal(a, b), (replay, i, k)
            torch.zeros(1 << 20, device="cuda").add_(1.0).sum().item()
        enc.close()


def test_on_a_stream_of_its_own():
    import torch
    side, p = torch.cuda.Stream(), policy(4)
    enc, here = encoder(stream=side), encoder()
    s, t = state(11, torch.bfloat16), state(11, torch.bfloat16)
    torch.cuda.synchronize()
    a, b = everything(enc, p, s), everything(here, p, t)
    torch.cuda.synchronize()
    for x, y in zip(flat(s, a), flat(t, b)):
        assert torch.equal(x, y)
    enc.close()
    here.close()


def test_a_workspace_that_would_have_to_grow_is_refused_in_a_capture():
    import torch
    import paper_2304_14698_amd as xrl
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        enc, s = encoder(), state(12, torch.bfloat16)
        out = torch.empty_like(s["q1"])
        how = dict(table=s["table"], lengths=s["lengths"], scale=0.2)
        stream.synchronize()
        graph, code = torch.cuda.CUDAGraph(), None
        with torch.cuda.graph(graph, stream=stream):
            s["kc"].mul_(1.0)
            try:
                enc.cache_attention(s["q1"], s["ptr1"], s["kc"], s["vc"], out=out, **how)
            except xrl.XrlError as e:
                code = e.code
        assert code == xrl.ERR["HIP"]
        graph.replay()
        enc.cache_attention(s["q1"], s["ptr1"], s["kc"], s["vc"], out=out, **how)
        stream.synchronize()
        assert out.isfinite().all()
        enc.close()


def test_tables_whose_rows_share_memory_are_refused():
    """A row of a table for all sequences (stride 0), and rows that overlap: the library takes rows at least their length apart."""
    import torch
    enc, s = encoder(), state(13, torch.float32)
    wide = s["table"].contiguous()
    for bad in (wide[:1].expand(5, -1), wide.as_strided((5, wide.shape[1]), (wide.shape[1] - 1, 1)), wide.T.contiguous().T):
        how = dict(table=bad, lengths=s["lengths"])
        with pytest.raises(ValueError, match="table"):
            enc.cache_attention(s["q1"], s["ptr1"], s["kc"], s["vc"], **how)
        with pytest.raises(ValueError, match="table"):
            enc.cache_write(s["k1"], s["v1"], s["ptr1"], s["kc"], s["vc"], **how)
    apart = torch.full((5, wide.shape[1] + 3), -1, dtype=torch.int32, device="cuda")
    apart[:, :wide.shape[1]] = wide
    a, b = (enc.cache_attention(s["q1"], s["ptr1"], s["kc"], s["vc"], table=t, lengths=s["lengths"]) for t in (wide, apart[:, :wide.shape[1]]))
    torch.cuda.synchronize()
    assert torch.equal(a, b)
    enc.close()


@pytest.mark.parametrize("type", ["fp32", "bf16"])
@pytest.mark.parametrize("how", [dict(), dict(top_k=3), dict(top_k=40, top_p=0.8), dict(min_p=0.1), dict(top_p=0.7), dict(top_k=9, min_p=0.2)])
@pytest.mark.parametrize("masked", ["own", "shared", "odd"])
def test_drawing_of_long_masked_rows(type, how, masked):
    """Rows of more than 8192 entries with masks: none, one and few entries left, NaN and infinities under the mask and beside it, ties over the whole row."""
    import torch
    enc = encoder()
    rows, cols = 7, 24583
    x, u, g = draw(31, rows, cols, type)
    mask = torch.rand(rows, cols, generator=g, device="cuda") < 0.3
    if masked == "odd":                                         # rows at odd places
        wide = torch.zeros(rows, cols + 1, dtype=x.dtype, device="cuda")
        wide[:, 1:] = x
        x = wide[:, 1:]
    if masked == "shared":
        mask = mask[0].clone()
        x[1, mask.nonzero()[5]] = math.nan
        x[2, (~mask).nonzero()[7]] = math.nan
        x[3, mask.nonzero()[-1]] = math.inf
        x[4] = 1.25
    else:
        mask[0] = False
        mask[1] = False
        mask[1, cols - 1] = True
        mask[2] = False
        mask[2, 8190:8195] = True
        x[3, ~mask[3]] = math.nan
        x[4, mask[4].nonzero()[11]] = math.nan
        x[5, mask[5].nonzero()[0]] = -math.inf
        x[6] = -2.5
    check(enc, x, u, mask=mask.to(torch.uint8), **how)
    enc.close()


@pytest.mark.parametrize("cols", [8193, 16384, 30000])
@pytest.mark.parametrize("how", [dict(top_k=3), dict(min_p=0.1), dict(top_k=7, top_p=0.9)])
def test_drawing_of_long_rows_that_hold_no_number(cols, how):
    """A NaN or an infinity at a row's ends and at the borders of its parts, or nothing but the lowest values."""
    import torch
    enc = encoder()
    x, u, _ = draw(41, 9, cols, "fp32")
    for r, (at, what) in enumerate([(0, math.nan), (cols - 1, math.nan), (8191, math.inf), (min(8192, cols - 1), math.nan), (5, -math.inf), (cols - 1, -math.inf)]):
        x[r, at] = what
    x[6] = -math.inf
    x[7] = torch.finfo(torch.float32).min
    x[8] = -math.inf
    x[8, cols - 2] = torch.finfo(torch.float32).min
    check(enc, x, u, **how)
    enc.close()


def test_drawing_of_more_rows_than_compute_units():
    import torch
    enc = encoder()
    for rows, cols in ((300, 4500), (700, 4097)):
        x, u, _ = draw(51, rows, cols, "bf16")
        check(enc, x, u, top_k=40, top_p=0.9)
        check(enc, x, u, temperature=0.8)
    enc.close()


@pytest.mark.parametrize("type", ["fp32", "bf16"])
@pytest.mark.parametrize("cols", [257, 1025, 2043])
@pytest.mark.parametrize("how", [dict(), dict(top_k=3), dict(top_k=700), dict(top_p=0.6), dict(min_p=0.02), dict(top_k=300, top_p=0.9, min_p=0.01), dict(top_k=16, top_p=0.5)])
def test_drawing_of_many_middling_rows(type, cols, how):
    """So many rows that each has one wave: random ones, ties, masked ones, what is not finite."""
    import torch
    enc = encoder()
    rows = 530
    x, u, g = draw(61 + cols, rows, cols, type)
    mask = torch.rand(rows, cols, generator=g, device="cuda") < 0.7
    x[3] = 0.5
    x[4, :cols // 2] = 2.0
    x[4, cols // 2:] = -INF
    x[5] = -INF
    x[6, cols - 1] = math.nan
    x[7, 0] = INF
    mask[8] = False
    mask[9] = False
    mask[9, cols - 1] = True
    keep = torch.cat([torch.arange(40, device="cuda"), torch.arange(rows - 20, rows, device="cuda")])
    for m in (None, mask.to(torch.uint8)):
        got = enc.token_sample(x, u, mask=m, **how)
        check_rows(enc, x, u, m, got, keep, how)
    enc.close()


def check_rows(enc, x, u, mask, got, keep, how):
    """Some rows of a call against the oracle."""
    import torch
    from test_gpu_token_sample import one_row
    torch.cuda.synchronize()
    kw = dict(temperature=1.0, top_k=0, top_p=1.0, min_p=0.0) | how
    for r in keep.tolist():
        X = x[r].double().cpu().numpy()
        id, lp, _ = one_row(X, None if mask is None else mask[r].cpu().numpy(), float(u[r]), kw["top_k"], kw["top_p"], kw["min_p"], kw["temperature"])
        assert int(got["ids"][r]) == id, r
        g, n = float(got["logp"][r]), max(2, len(X))
        if math.isfinite(lp):
            assert abs(g - lp) <= (3 * (n / 64 + 8) + 64 + 4 * math.log2(n)) * U + 6 * U * (abs(lp) + math.log(n)), r
        else:
            assert g == lp or (math.isnan(lp) and math.isnan(g)), r
