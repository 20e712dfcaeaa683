"""Operators of a policy that reads a history in order: the norm of queries and keys with the rotation by position, attention over packed
sequences, attention of new tokens over a paged cache, and drawing from a row of logits.

The inputs are what a program holds that rolls such a policy out and trains it: histories of different lengths packed one behind
another, a cache whose pages lie in any order, gradients of a loss, logits with the masks of a state's slots and given random numbers.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
INF = math.inf
_encoder = None


def _rotary(name, op, tokens, heads, kv_heads, dim, rotary, type, norm, interleaved, far):
    return dict(name=name, op=op, tokens=tokens, heads=heads, kv_heads=kv_heads, dim=dim, rotary=rotary, type=type, norm=norm,
                interleaved=interleaved, far=far)


def _attn(name, op, seqs, tokens, spread, heads, kv_heads, dim, type, causal=True, keys=0):
    return dict(name=name, op=op, seqs=seqs, tokens=tokens, spread=spread, heads=heads, kv_heads=kv_heads, dim=dim, type=type,
                causal=causal, keys=keys)


def _cache(name, seqs, new, keys, spread, heads, kv_heads, dim, page, type):
    return dict(name=name, op="cache", seqs=seqs, new=new, keys=keys, spread=spread, heads=heads, kv_heads=kv_heads, dim=dim, page=page,
                type=type)


def _sample(name, rows, cols, type, mask, top_k, top_p, min_p, temperature=1.0, ragged=False):
    return dict(name=name, op="sample", rows=rows, cols=cols, type=type, mask=mask, top_k=top_k, top_p=top_p, min_p=min_p,
                temperature=temperature, ragged=ragged)


def listed():
    return [
        # the next tokens of 32 environments, at positions of a long context
        _rotary("rotary_step_bf16", "rotary", 32, 32, 8, 128, 128, "bf16", True, False, 1 << 17),
        # an update over packed histories, half of each head rotated: forward and gradients
        _rotary("rotary_update_bf16", "rotary_grad", 16384, 32, 8, 128, 64, "bf16", True, True, 8192),
        # histories of 1 to 24 rules in a minibatch of a small policy, in single precision: forward and gradients
        _attn("attn_histories_fp32", "attn_grad", 1024, 8192, 24.0, 4, 4, 32, "fp32"),
        # one long prompt
        _attn("attn_prompt_bf16", "attn", 1, 8192, 1.0, 32, 8, 128, "bf16"),
        # a minibatch of episodes of very different lengths
        _attn("attn_episodes_bf16", "attn_grad", 16, 16381, 20.0, 16, 4, 64, "bf16"),
        # an update over long sequences
        _attn("attn_update_bf16", "attn_grad", 2, 8192, 1.0, 32, 8, 128, "bf16"),
        # one rule more in 64 environments of a small policy
        _cache("cache_step_small_fp32", 64, 1, 64 * 24, 12.0, 4, 4, 32, 16, "fp32"),
        # one token more in 32 sequences, 1 to 30 thousand tokens each
        _cache("cache_step_bf16", 32, 1, 262144, 24.0, 32, 8, 128, 16, "bf16"),
        # a chunk of new tokens each over long contexts
        _cache("cache_chunk_bf16", 4, 509, 32768, 3.0, 32, 8, 128, 64, "bf16"),
        # a rollout step of 32 environments: the slots of their states with their masks
        _sample("sample_slots_fp32", 32, 65, "fp32", "own", 0, 1.0, 0.0, 1.0, True),
        # the next token of eight sequences
        _sample("sample_next_bf16", 8, 128256, "bf16", "none", 50, 0.95, 0.0, 0.7),
        # a rollout of many sequences at once
        _sample("sample_rollout_bf16", 2048, 32003, "bf16", "none", 0, 0.9, 0.02),
    ]


def draw(rng):
    def size(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    op = rng.choice(["rotary", "rotary_grad", "attn", "attn_grad", "cache", "sample"])
    type = rng.choice(["bf16", "bf16", "fp32"])
    dim = rng.choice([16, 32, 40, 64, 64, 80, 96, 128, 128, rng.randint(2, 64) * 2, rng.randint(1, 128)])
    kv, group = size(1, 8), rng.choice([1, 1, 2, 4, 8, rng.randint(1, 8)])
    if op in ("rotary", "rotary_grad"):
        dim += dim % 2
        rotary = rng.choice([dim, dim, 2 * rng.randint(1, dim // 2)])
        tokens = size(1, max(1, min(32768, (1 << 26) // (dim * kv * (group + 1)))))
        c = _rotary("", op, tokens, kv * group, kv, dim, rotary, type, rng.random() < 0.7, rng.random() < 0.5, size(64, 1 << 20))
    elif op in ("attn", "attn_grad"):
        seqs = size(1, 512)
        # scores of all pairs, and operations of the largest listed case
        tokens = size(seqs, max(seqs, min(16384, int(math.sqrt(2e9 * seqs / (16 * kv * group))))))
        causal = rng.random() < 0.7
        keys = 0 if causal or rng.random() < 0.5 else size(seqs, 2 * tokens)
        c = _attn("", op, seqs, tokens, rng.choice([1.0, 4.0, 16.0]), kv * group, kv, dim, type, causal, keys)
    elif op == "cache":
        seqs, new = size(1, 128), rng.choice([1, 1, 1, size(1, 512)])
        most = min(262144, int(1e9 / (dim * kv)), int(1e9 / (new * kv * group)))
        keys = size(seqs * new, max(seqs * new, most))
        c = _cache("", seqs, new, keys, rng.choice([1.0, 4.0, 16.0]), kv * group, kv, dim, rng.choice([1, 8, 16, 16, 64, 100, 256]), type)
    else:
        ragged = rng.random() < 0.25
        cols = size(2, 1024) if ragged else size(16, 131072)
        rows = size(1, 4096) if ragged else size(1, min(8192, (1 << 26) // cols))
        c = _sample("", rows, cols, type, rng.choice(["none", "own", "shared"] if not ragged else ["none", "own"]),
                    rng.choice([0, 0, 1, 20, 64, size(1, 2000)]), rng.choice([1.0, 0.95, 0.9, 0.5]), rng.choice([0.0, 0.0, 0.02, 0.1]),
                    rng.choice([1.0, 0.7, 1.5]), ragged)
    c.pop("name", None)
    return c


def _lengths(seqs, total, spread, least=0):
    """Lengths of `seqs` sequences, `total` in all, the longest about `spread` times the shortest."""
    f = np.exp(np.linspace(0.0, math.log(spread), seqs)) if seqs > 1 else np.ones(1)
    end = least * np.arange(1, seqs + 1) + np.rint(np.cumsum(f) / f.sum() * (total - least * seqs)).astype(np.int64)
    return np.diff(end, prepend=0)


def _case_lengths(case):
    if case["op"] == "cache":
        return np.full(case["seqs"], case["new"]), _lengths(case["seqs"], case["keys"], case["spread"], case["new"])
    n = _lengths(case["seqs"], case["tokens"], case["spread"])
    return n, _lengths(case["seqs"], case["keys"], case["spread"]) if case["keys"] else n


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _ptr(lengths):
    return torch.from_numpy(np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)).cuda()


def prepare(case, seed):
    g, op, s = _gen(seed), case["op"], dict(case=case)
    randn = lambda *n: torch.randn(*n, generator=g, device="cuda")  # noqa: E731
    if op == "sample":
        rows, cols = case["rows"], case["cols"]
        s["row_ptr"], s["width"], shape = None, cols, (rows, cols)
        if case["ragged"]:
            u = torch.rand(rows, generator=g, device="cuda", dtype=torch.float64) + 0.02
            end = (u.cumsum(0) / u.sum() * (rows * (cols - 1))).long().clamp_(max=rows * (cols - 1))
            end[-1] = rows * (cols - 1)
            s["row_ptr"] = torch.cat([end.new_zeros(1), end + 1 + torch.arange(rows, device="cuda")]).int()
            s["width"], shape = int(torch.diff(s["row_ptr"].long()).max()), (rows * cols,)
        s["logits"] = (2.5 * randn(*shape)).to(TYPES[case["type"]])
        s["uniforms"] = torch.rand(rows, generator=g, device="cuda")
        s["mask"] = None
        if case["mask"] == "own":
            s["mask"] = (torch.rand(*shape, generator=g, device="cuda") < 0.6).to(torch.uint8)
            if case["ragged"]:
                s["mask"][s["row_ptr"][:-1].long()] = 1                 # each state's first slot may always be taken
            elif rows > 8:
                s["mask"][3] = 0                                        # nothing applies
        elif case["mask"] == "shared":
            s["mask"] = (torch.rand(cols, generator=g, device="cuda") < 0.6).to(torch.uint8)
            s["mask"][0] = 1
        return s
    type, heads, kv, dim = TYPES[case["type"]], case["heads"], case["kv_heads"], case["dim"]
    if op in ("rotary", "rotary_grad"):
        n, half = case["tokens"], case["rotary"] // 2
        qkv = (3.0 * randn(n, heads + 2 * kv, dim)).to(type)            # what one product with the weights of all three gives
        s["q"], s["k"] = qkv[:, :heads], qkv[:, heads:heads + kv]
        s["positions"] = torch.randint(0, case["far"], (n,), generator=g, device="cuda").int()
        s["freqs"] = (10000.0 ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)).float()
        s["q_weight"] = s["k_weight"] = None
        if case["norm"]:
            s["q_weight"], s["k_weight"] = 1.0 + 0.1 * randn(dim), 1.0 + 0.1 * randn(dim)
        if op == "rotary_grad":
            s["dq"], s["dk"] = (1e-3 * randn(n, heads, dim)).to(type), (1e-3 * randn(n, kv, dim)).to(type)
            if case["norm"]:
                s["dq_weight"], s["dk_weight"] = 1e-3 * randn(dim), 1e-3 * randn(dim)     # of the micro-batch before
        return s
    nq, nk = _case_lengths(case)
    order = np.random.Generator(np.random.PCG64(seed)).permutation(case["seqs"])
    nq, nk = nq[order], nk[order]
    s["q_ptr"], s["longest"] = _ptr(nq), (int(nq.max()), int(nk.max()))
    s["scale"] = dim ** -0.5
    s["q"] = (1.5 * randn(int(nq.sum()), heads, dim)).to(type)
    if op == "cache":
        page, total = case["page"], int(nq.sum())
        per = -(-nk // page)
        width = int(per.max())
        shuffled = torch.randperm(int(per.sum()) + 3, generator=g, device="cuda").int()
        at = torch.from_numpy(np.cumsum(per) - per).cuda()[:, None] + torch.arange(width, device="cuda")
        s["table"] = torch.where(torch.arange(width, device="cuda") < torch.from_numpy(per).cuda()[:, None],
                                 shuffled[at.clamp(max=shuffled.numel() - 1)], -1)
        s["k_cache"], s["v_cache"] = ((1.5 * torch.randn(shuffled.numel(), page, kv, dim, generator=g, device="cuda", dtype=type))
                                      for _ in range(2))
        s["k"], s["v"] = (1.5 * randn(total, kv, dim)).to(type), (1.5 * randn(total, kv, dim)).to(type)
        s["lengths"] = torch.from_numpy(nk.astype(np.int32)).cuda()     # with the new tokens
        return s
    s["k_ptr"] = _ptr(nk) if case["keys"] else None
    s["k"], s["v"] = (1.5 * randn(int(nk.sum()), kv, dim)).to(type), randn(int(nk.sum()), kv, dim).to(type)
    if op == "attn_grad":
        s["dout"] = (1e-2 * randn(int(nq.sum()), heads, dim)).to(type)
    return s


def _own():
    """The library's context: one for the program, on its stream."""
    global _encoder
    if _encoder is None:
        import paper_2304_14698_amd as xrl
        model = dict(n_op_types=40, n_node_dense=0, d_edge=4, d_global=0, hidden=64, rounds=0)
        _encoder = xrl.Encoder(model, np.zeros(xrl.weight_count(model), np.float32))
    return _encoder


def _run_own(s):
    c, enc, op = s["case"], _own(), s["case"]["op"]
    if op == "sample":
        return enc.token_sample(s["logits"], s["uniforms"], mask=s["mask"], row_ptr=s["row_ptr"], temperature=c["temperature"],
                                top_k=c["top_k"], top_p=c["top_p"], min_p=c["min_p"])
    if op in ("rotary", "rotary_grad"):
        how = dict(q_weight=s["q_weight"], k_weight=s["k_weight"], interleaved=c["interleaved"])
        q, k = enc.head_rotary(s["q"], s["k"], s["positions"], s["freqs"], **how)
        if op == "rotary":
            return dict(q=q, k=k)
        grads = dict(dq_weight=s["dq_weight"], dk_weight=s["dk_weight"]) if c["norm"] else {}
        dq, dk = enc.head_rotary_backward(s["q"], s["k"], s["positions"], s["freqs"], s["dq"], s["dk"], **grads, **how)
        return dict(q=q, k=k, dq=dq, dk=dk, **grads)
    if op == "cache":
        where = dict(table=s["table"], lengths=s["lengths"])
        enc.cache_write(s["k"], s["v"], s["q_ptr"], s["k_cache"], s["v_cache"], **where)
        out = enc.cache_attention(s["q"], s["q_ptr"], s["k_cache"], s["v_cache"], scale=s["scale"], **where)
        return dict(out=out, k_cache=s["k_cache"], v_cache=s["v_cache"])
    how = dict(k_ptr=s["k_ptr"], causal=c["causal"], scale=s["scale"])
    f = enc.attention(s["q"], s["k"], s["v"], s["q_ptr"], **how)
    if op == "attn":
        return f
    dq, dk, dv = enc.attention_backward(s["q"], s["k"], s["v"], s["q_ptr"], f, s["dout"], **how)
    return dict(f, dq=dq, dk=dk, dv=dv)


def _turn(y, c, positions, freqs, sign):
    """The first `rotary` columns of y [n, heads, dim] turned by positions * freqs."""
    a = positions.double()[:, None] * freqs.double()
    cos, sin = a.cos().float()[:, None], sign * a.sin().float()[:, None]
    r, n, heads, _ = c["rotary"], *y.shape
    pair = y[..., :r].reshape(n, heads, r // 2, 2) if c["interleaved"] else y[..., :r].reshape(n, heads, 2, r // 2).transpose(2, 3)
    z = torch.stack([pair[..., 0] * cos - pair[..., 1] * sin, pair[..., 0] * sin + pair[..., 1] * cos], -1)
    z = z if c["interleaved"] else z.transpose(2, 3)
    return torch.cat([z.reshape(n, heads, r), y[..., r:]], -1)


def _plain_rotary(s, x, weight, dz, dweight):
    c, x32 = s["case"], x.float()
    r = torch.ones_like(x32[..., :1]) if weight is None else ((x32 * x32).mean(-1, keepdim=True) + 1e-6).rsqrt()
    w = 1.0 if weight is None else weight
    z = _turn(x32 * r * w, c, s["positions"], s["freqs"], 1.0).to(x.dtype)
    if dz is None:
        return z, None
    g = _turn(dz.float(), c, s["positions"], s["freqs"], -1.0)
    if weight is None:
        return z, g.to(x.dtype)
    dweight += (g * x32 * r).sum((0, 1))
    gw = g * w
    return z, (r * (gw - x32 * (r * r * (gw * x32).mean(-1, keepdim=True)))).to(x.dtype)


def _padded(x, ptr, longest, kv):
    """Packed rows [n, heads, dim] as [seqs, kv heads, group, longest, dim] in fp32, zeros behind a sequence's end, and where each row went."""
    ptr = ptr.long()
    at = ptr[:-1, None] + torch.arange(longest, device="cuda")
    inside = at < ptr[1:, None]
    row = torch.arange(x.shape[0], device="cuda")
    seq = torch.searchsorted(ptr[1:], row, right=True)
    place = seq * longest + row - ptr[seq]
    y = torch.where(inside[..., None, None], x[at.clamp(max=max(x.shape[0] - 1, 0))].float(), 0.0)
    b, n, heads, dim = y.shape
    return y.view(b, n, kv, heads // kv, dim).permute(0, 2, 3, 1, 4).contiguous(), place


def _packed(y, place, dtype):
    b, kv, group, n, dim = y.shape
    return y.permute(0, 3, 1, 2, 4).reshape(b * n, kv * group, dim)[place].to(dtype)


def _softmax(q, k, v, seen, scale):
    """q [b, kv, group, n, dim], k and v [b, kv, 1, m, dim], seen [b, n, m]: out, ln of the sums, and the probabilities."""
    b, kv, group, n, dim = q.shape
    S = (q.view(b, kv, group * n, dim) @ k[:, :, 0].transpose(2, 3)).view(b, kv, group, n, -1) * scale
    S = S.masked_fill_(~seen[:, None, None], -INF)
    top = S.amax(-1, keepdim=True).clamp_(min=-3e38)
    P = S.sub_(top).exp_()
    total = P.sum(-1, keepdim=True)
    P = P.div_(torch.where(total > 0, total, 1.0))
    out = (P.view(b, kv, group * n, -1) @ v[:, :, 0]).view(q.shape)
    return out, torch.where(total > 0, top + total.log(), -INF)[..., 0], P


def _seen(nq, nk, n, m, causal):
    i, j = torch.arange(n, device="cuda")[:, None], torch.arange(m, device="cuda")
    seen = (i < nq[:, None, None]) & (j < nk[:, None, None])
    return seen & (j <= i + (nk - nq)[:, None, None]) if causal else seen


def _plain_attn(s):
    c, kv, type = s["case"], s["case"]["kv_heads"], s["q"].dtype
    q_ptr = s["q_ptr"]
    k_ptr = q_ptr if s["k_ptr"] is None else s["k_ptr"]
    (q, qi), (k, ki), (v, _) = (_padded(s[x], p, m, kv) for x, p, m in
                                (("q", q_ptr, s["longest"][0]), ("k", k_ptr, s["longest"][1]), ("v", k_ptr, s["longest"][1])))
    b, _, group, n, dim = q.shape
    seen = _seen(torch.diff(q_ptr.long()), torch.diff(k_ptr.long()), n, k.shape[3], c["causal"])
    out, lse, P = _softmax(q, k, v, seen, s["scale"])
    res = dict(out=_packed(out, qi, type), lse=lse.permute(0, 3, 1, 2).reshape(b * n, kv * group)[qi])
    if c["op"] == "attn":
        return res
    do = _padded(s["dout"], q_ptr, n, kv)[0]
    flat = lambda x: x.reshape(b, kv, group * n, x.shape[-1])  # noqa: E731
    res["dv"] = _packed((flat(P).transpose(2, 3) @ flat(do))[:, :, None], ki, type)
    dS = (flat(do) @ v[:, :, 0].transpose(2, 3)).view(P.shape)
    dS = dS.sub_((do * out).sum(-1, keepdim=True)).mul_(P).mul_(s["scale"])
    res["dq"] = _packed((flat(dS) @ k[:, :, 0]).view(q.shape), qi, type)
    res["dk"] = _packed((flat(dS).transpose(2, 3) @ flat(q))[:, :, None], ki, type)
    return res


def _plain_cache(s):
    c, kv, type = s["case"], s["case"]["kv_heads"], s["q"].dtype
    n, m = s["longest"]
    q, qi = _padded(s["q"], s["q_ptr"], n, kv)
    nq, nk, table, page = torch.diff(s["q_ptr"].long()), s["lengths"].long(), s["table"].long(), c["page"]
    seq = torch.repeat_interleave(torch.arange(c["seqs"], device="cuda"), nq, output_size=s["k"].shape[0])
    at = (nk - nq)[seq] + torch.arange(s["k"].shape[0], device="cuda") - s["q_ptr"].long()[seq]
    s["k_cache"][table[seq, at // page], at % page] = s["k"]
    s["v_cache"][table[seq, at // page], at % page] = s["v"]
    j = torch.arange(m, device="cuda")
    there = j < nk[:, None]
    row = table[:, j // page].clamp(min=0) * page + j % page
    read = lambda x: torch.where(there[..., None, None], x.view(-1, kv, c["dim"])[row].float(), 0.0).transpose(1, 2)[:, :, None].contiguous()  # noqa: E731
    out = _softmax(q, read(s["k_cache"]), read(s["v_cache"]), _seen(nq, nk, n, m, True), s["scale"])[0]
    return dict(out=_packed(out, qi, type), k_cache=s["k_cache"], v_cache=s["v_cache"])


def _dense(s, flat, fill):
    """Ragged rows as a dense matrix, `fill` behind a row's end."""
    ptr = s["row_ptr"].long()
    at = ptr[:-1, None] + torch.arange(s["width"], device="cuda")
    return torch.where(at < ptr[1:, None], flat[at.clamp(max=flat.numel() - 1)], fill)


def _plain_sample(s):
    """In 64 bits: which entries are kept and which one is drawn goes by sums next to a border."""
    c, f32 = s["case"], np.float32
    x = s["logits"].float()
    x = _dense(s, x, -INF) if c["ragged"] else x
    if s["mask"] is not None:
        x = torch.where((_dense(s, s["mask"], 0) if c["ragged"] else s["mask"]) != 0, x, -INF)
    n, width = x.shape
    top = x.amax(1, keepdim=True).clamp(min=-3e38).double()
    t = (x.double() - top) / float(f32(c["temperature"]))
    w = t.exp()
    kept = w > 0
    if c["top_k"] or c["top_p"] < 1.0:
        order = x.sort(dim=1, descending=True, stable=True)[1]
        ranked = w.gather(1, order)
        if c["top_k"]:
            ranked[:, c["top_k"]:] = 0.0
        upto = ranked.cumsum(1)
        stays = ranked > 0
        if c["top_p"] < 1.0:
            stays &= upto - ranked < float(f32(c["top_p"])) * upto[:, -1:]
        kept &= torch.zeros_like(kept).scatter_(1, order, stays)
    if c["min_p"] > 0.0:
        kept &= w >= float(f32(c["min_p"]))
    upto = torch.where(kept, w, 0.0).cumsum(1)
    beyond = kept & (upto > s["uniforms"].double()[:, None] * upto[:, -1:])
    j = torch.arange(width, device="cuda")
    last = torch.where(kept, j, -1).amax(1)
    first = torch.where(beyond, j, width).amin(1)
    ids = torch.where(first < width, first, last)
    logp = t.gather(1, ids.clamp(min=0)[:, None])[:, 0] - w.sum(1).log()
    return dict(ids=ids.int(), logp=torch.where(ids < 0, -INF, logp).float())


def run(state):
    s, op = state, state["case"]["op"]
    if own:
        return _run_own(s)
    if op == "sample":
        return _plain_sample(s)
    if op == "cache":
        return _plain_cache(s)
    if op in ("attn", "attn_grad"):
        return _plain_attn(s)
    q, dq = _plain_rotary(s, s["q"], s["q_weight"], s.get("dq"), s.get("dq_weight"))
    k, dk = _plain_rotary(s, s["k"], s["k_weight"], s.get("dk"), s.get("dk_weight"))
    if op == "rotary":
        return dict(q=q, k=k)
    more = dict(dq_weight=s["dq_weight"], dk_weight=s["dk_weight"]) if s["case"]["norm"] else {}
    return dict(q=q, k=k, dq=dq, dk=dk, **more)


def work(case):
    size, op = {"fp32": 4, "bf16": 2}[case["type"]], case["op"]
    if op == "sample":
        n = case["rows"] * case["cols"]
        mask = {"none": 0, "own": n, "shared": case["cols"]}[case["mask"]]
        return {"bytes": n * size + mask + 12 * case["rows"], "flops": 8 * n}
    rows = case["heads"] + case["kv_heads"]
    if op in ("rotary", "rotary_grad"):
        n = case["tokens"] * rows * case["dim"]
        back = op == "rotary_grad"
        return {"bytes": n * size * (4 if back else 2) + 4 * case["tokens"] + (16 * case["dim"] if case["norm"] else 0),
                "flops": n * (18 if back else 6)}
    nq, nk = _case_lengths(case)
    if op != "cache" and not case["causal"]:
        pairs = int((nq * nk).sum())
    else:                        # row i of a sequence sees i + 1 + nk - nq keys (none of fewer keys than rows is listed or drawn)
        pairs = int((nq * (nk - nq) + nq * (nq + 1) // 2).sum())
    q, k = int(nq.sum()) * case["heads"] * case["dim"] * size, int(nk.sum()) * case["kv_heads"] * case["dim"] * size
    flops = 4.0 * case["dim"] * case["heads"] * pairs
    if op == "cache":
        new = int(nq.sum()) * case["kv_heads"] * case["dim"] * size
        return {"bytes": 2 * q + 2 * k + 2 * new, "flops": flops}
    if op == "attn":
        return {"bytes": 2 * q + 2 * k, "flops": flops}
    return {"bytes": 4 * q + 4 * k, "flops": 3.5 * flops}


def exact(case, seed):
    s, op, c = prepare(case, seed), case["op"], case
    if op == "sample":
        return _exact_sample(s)
    if op in ("rotary", "rotary_grad"):
        out = {}
        half = c["rotary"] // 2
        a = s["positions"].cpu().numpy().astype(np.float64)[:, None] * s["freqs"].cpu().numpy().astype(np.float64)
        turn = torch.complex(torch.from_numpy(np.cos(a)).cuda(), torch.from_numpy(np.sin(a)).cuda())[:, None]
        first = torch.arange(half, device="cuda") * (2 if c["interleaved"] else 1)
        second = first + (1 if c["interleaved"] else half)

        def turned(y, by):
            z = torch.complex(y[..., first], y[..., second]) * by
            y = y.clone()
            y[..., first], y[..., second] = z.real, z.imag
            return y
        for x in "qk":
            v = s[x].double()
            w = torch.ones(c["dim"], dtype=torch.float64, device="cuda") if not c["norm"] else s[x + "_weight"].double()
            r = 1.0 / torch.sqrt(v.square().sum(-1, keepdim=True) / c["dim"] + 1e-6) if c["norm"] else torch.ones_like(v[..., :1])
            out[x] = turned(v * r * w, turn)
            if op == "rotary_grad":
                back = turned(s["d" + x].double(), turn.conj())
                if c["norm"]:
                    unit = v * r
                    out["d%s_weight" % x] = s["d%s_weight" % x].double() + torch.einsum("nhd,nhd->d", back, unit)
                    # of u = v / |v|: what the gradient has along v goes, but for eps' share
                    along = (back * w * unit).sum(-1, keepdim=True) / c["dim"]
                    back = r * (back * w - unit * along)
                out["d" + x] = back
        return out
    # one sequence and one head of keys at a time
    heads, kv = c["heads"], c["kv_heads"]
    group = heads // kv
    q = s["q"].double()
    q_ptr = s["q_ptr"].tolist()
    new = lambda x: torch.zeros(x.shape, dtype=torch.float64, device="cuda")  # noqa: E731
    out, lse = new(q), torch.zeros(q.shape[:2], dtype=torch.float64, device="cuda")
    back = op == "attn_grad"
    if op == "cache":
        kc, vc, page = s["k_cache"], s["v_cache"], c["page"]
        lengths, table = s["lengths"].tolist(), s["table"].cpu().numpy()
        for b in range(c["seqs"]):
            for i in range(q_ptr[b], q_ptr[b + 1]):
                at = lengths[b] - (q_ptr[b + 1] - i)
                kc[int(table[b, at // page]), at % page] = s["k"][i]
                vc[int(table[b, at // page]), at % page] = s["v"][i]
    else:
        k_ptr = q_ptr if s["k_ptr"] is None else s["k_ptr"].tolist()
        dq, dk, dv = new(q), new(s["k"]), new(s["v"])
    for b in range(c["seqs"]):
        rows = slice(q_ptr[b], q_ptr[b + 1])
        n = rows.stop - rows.start
        if op == "cache":
            m = lengths[b]
            pages = torch.from_numpy(table[b, :-(-m // page)].astype(np.int64)).cuda()
            K, V = (x[pages].reshape(-1, kv, c["dim"])[:m].double() for x in (kc, vc))
        else:
            keys = slice(k_ptr[b], k_ptr[b + 1])
            m = keys.stop - keys.start
            K, V = s["k"][keys].double(), s["v"][keys].double()
        if n == 0 or m == 0:
            lse[rows] = -INF
            continue
        causal = op == "cache" or c["causal"]
        late = torch.ones(n, m, dtype=torch.bool, device="cuda").triu(m - n + 1) if causal else None
        for h in range(kv):
            for e in range(h * group, (h + 1) * group):
                y = q[rows, e] @ K[:, h].T * s["scale"]
                if late is not None:
                    y = y.masked_fill(late, -INF)
                l = torch.logsumexp(y, 1)
                p = torch.exp(y - l[:, None])
                lse[rows, e] = l
                out[rows, e] = p @ V[:, h]
                if back:
                    do = s["dout"][rows, e].double()
                    dv[keys, h] += p.T @ do
                    dp = do @ V[:, h].T
                    ds = p * (dp - (p * dp).sum(1, keepdim=True)) * s["scale"]
                    dq[rows, e] = ds @ K[:, h]
                    dk[keys, h] += ds.T @ q[rows, e]
    if op == "cache":
        return dict(out=out, k_cache=None, v_cache=None)
    return dict(out=out, lse=lse, dq=dq, dk=dk, dv=dv) if back else dict(out=out, lse=lse)


def _exact_sample(s):
    """A row at a time, on the host: entries in order of size, the filters one after another, and the first whose sum passes."""
    c, f32 = s["case"], lambda v: float(np.float32(v))  # noqa: E731
    rows = c["rows"]
    if rows * c["cols"] >= 7e7:
        return None
    logits, u = s["logits"].float().cpu().numpy().astype(np.float64), s["uniforms"].cpu().numpy().astype(np.float64)
    mask = None if s["mask"] is None else s["mask"].cpu().numpy()
    ptr = s["row_ptr"].tolist() if c["ragged"] else None
    ids, logp = np.full(rows, -1, np.int32), np.full(rows, -INF)
    for r in range(rows):
        x = logits[ptr[r]:ptr[r + 1]] if ptr else logits[r]
        ok = np.ones(len(x), bool) if mask is None else (mask[ptr[r]:ptr[r + 1]] if ptr else mask if mask.ndim == 1 else mask[r]) != 0
        at = np.flatnonzero(ok)
        if not len(at):
            continue
        y = (x[at] - x[at].max()) / f32(c["temperature"])
        p = np.exp(y)
        whole = p.sum()
        rank = np.lexsort((at, -x[at]))
        rank = rank[:c["top_k"]] if c["top_k"] else rank
        if c["top_p"] < 1.0:
            before = np.cumsum(p[rank]) - p[rank]
            rank = rank[before < f32(c["top_p"]) * p[rank].sum()]
        rank = np.sort(rank[p[rank] >= f32(c["min_p"])])
        upto = np.cumsum(p[rank])
        pick = rank[min(int(np.searchsorted(upto, u[r] * upto[-1], side="right")), len(rank) - 1)]
        ids[r], logp[r] = at[pick], y[pick] - math.log(whole)
    return dict(ids=torch.from_numpy(ids), logp=torch.from_numpy(logp))
