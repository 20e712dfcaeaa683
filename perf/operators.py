"""Operators of a training step over a vocabulary: embedding with its gradient, log-probabilities of given tokens with
entropy, top alternatives and the gradient to the logits, and the orthogonalised update of a model's matrices.

The inputs are what an agent's program holds when it makes these calls: ids of operators or tokens (operators of a graph come
from a few dozen types, tokens from a long-tailed distribution), logits of a policy with its mask, gradients whose
spectrum falls off, and momentum of earlier steps.
"""
import math

import numpy as np
import torch

own = False

NS = (3.4445, -4.7750, 2.0315)
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
_encoder = None


def _embed(name, n, vocab, dim, table, out, scale=1.0):
    return dict(name=name, op="embed", n=n, vocab=vocab, dim=dim, table=table, out=out, scale=scale)


def _embed_grad(name, n, vocab, dim, dout, spread, scale=1.0):
    return dict(name=name, op="embed_grad", n=n, vocab=vocab, dim=dim, dout=dout, spread=spread, scale=scale)


def _logp(name, op, rows, cols, type, mask, top_k, temperature=1.0, ragged=False):
    return dict(name=name, op=op, rows=rows, cols=cols, type=type, mask=mask, top_k=top_k, temperature=temperature,
                ragged=ragged)


def _agent(hidden, rounds):
    """The matrices of an agent of this library: embed MLP, rounds, readout, heads (44 node, 8 edge, 1 global attributes)."""
    h = hidden
    one = "%dx%d %dx%d " % (2 * h + 8, h, h, h) + "%dx%d %dx%d " % (2 * h, h, h, h)
    return "44x%d %dx%d " % (h, h, h) + one * rounds + "%dx%d %dx%d " % (h + 1, h, h, h) + ("%dx256 256x64 64x1 " % h) * 2


def listed():
    return [
        # the next ids of 32 environments: one short gather
        _embed("embed_step_bf16", 32, 32000, 512, "bf16", "bf16", math.sqrt(512)),
        # a minibatch's ids through a table kept in single precision for the optimiser
        _embed("embed_batch_fp32_to_bf16", 65536, 50021, 768, "fp32", "bf16", math.sqrt(768)),
        # operator types of all nodes of one state of transformer graphs: a table of 40 rows, every row hit often
        _embed_grad("embed_grad_operators_fp32", 77013, 40, 128, "fp32", "even"),
        # tokens of a minibatch, long-tailed: a few ids take much of it
        _embed_grad("embed_grad_tokens_bf16", 65536, 50021, 1024, "bf16", "tail", math.sqrt(1024)),
        # a rollout step of 32 environments: the slots of their states with their mask, and the best four
        _logp("logp_slots_fp32", "logp", 32, 65, "fp32", "own", 4, 1.0, True),
        # the next token of eight sequences: few long rows
        _logp("logp_next_bf16", "logp", 8, 128256, "bf16", "none", 8, 0.7),
        # a rollout scored anew: log-probabilities and entropy of every given token
        _logp("logp_score_bf16", "logp", 4096, 32003, "bf16", "none", 0),
        # an update step: forward, and the gradient to the logits
        _logp("logp_update_bf16", "logp_grad", 2048, 50021, "bf16", "none", 0),
        # an update step with one mask for all rows, in single precision, alternatives kept for the record
        _logp("logp_update_mask_fp32", "logp_grad", 1000, 8191, "fp32", "shared", 5),
        # the optimiser's step of a small agent, of the largest one, and of wide layers
        dict(name="muon_agent_h64", op="muon", shapes=_agent(64, 2).strip()),
        dict(name="muon_agent_h256", op="muon", shapes=_agent(256, 5).strip()),
        dict(name="muon_wide", op="muon", shapes="2048x2048 2048x2048 2048x8192 8192x2048"),
    ]


def draw(rng):
    def size(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    op = rng.choice(["embed", "embed_grad", "logp", "logp_grad", "muon"])
    type = rng.choice(["fp32", "bf16"])
    if op in ("embed", "embed_grad"):
        dim = size(16, 2048)
        if rng.random() < 0.7:
            dim = (dim + 7) // 8 * 8
        vocab, n = size(8, 131072), size(1, min(131072, (1 << 26) // dim))
        scale = rng.choice([1.0, math.sqrt(dim)])
        if op == "embed":
            c = _embed("", n, vocab, dim, type, rng.choice(["fp32", "bf16"]), scale)
        else:
            c = _embed_grad("", n, vocab, dim, type, rng.choice(["even", "tail"]), scale)
    elif op in ("logp", "logp_grad"):
        ragged = rng.random() < 0.25
        cols = size(2, 1024) if ragged else size(16, 131072)
        rows = size(1, 4096) if ragged else size(1, min(16384, (1 << 27) // cols))
        c = _logp("", op, rows, cols, type, rng.choice(["none", "own", "shared"] if not ragged else ["none", "own"]),
                  rng.choice([0, 1, 4, 8, 16]), rng.choice([1.0, 0.7]), ragged)
    else:
        shapes, left = [], 3e11
        for _ in range(rng.randint(1, 24)):
            r, k = size(1, 4096), size(1, 4096)
            cost = 4 * r * k * min(r, k)
            if cost < left:
                shapes.append("%dx%d" % (r, k))
                left -= cost
        c = dict(op="muon", shapes=" ".join(shapes) or "256x256")
    c.pop("name", None)
    return c


def _shapes(case):
    return [tuple(int(v) for v in s.split("x")) for s in case["shapes"].split()]


def _gen(seed, device="cuda"):
    g = torch.Generator(device=device)
    g.manual_seed(int(seed))
    return g


def _ids(g, n, vocab, spread):
    u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
    if spread == "tail":        # frequency falls as one over the rank
        at = torch.exp(u * math.log(vocab + 1.0)) - 1.0
        order = torch.randperm(vocab, generator=g, device="cuda")
        return order[at.long().clamp_(0, vocab - 1)].int()
    return (u * vocab).long().clamp_(0, vocab - 1).int()


def prepare(case, seed):
    g = _gen(seed)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    s = dict(case=case)
    if case["op"] == "embed":
        s["table"] = (0.02 * randn(case["vocab"], case["dim"])).to(TYPES[case["table"]])
        s["ids"] = _ids(g, case["n"], case["vocab"], "tail")
    elif case["op"] == "embed_grad":
        s["dout"] = (1e-3 * randn(case["n"], case["dim"])).to(TYPES[case["dout"]])
        s["ids"] = _ids(g, case["n"], case["vocab"], case["spread"])
        if case["n"] > 16:       # padding at the end of a sequence
            s["ids"][-1] = -1
        s["dtable"] = 1e-3 * randn(case["vocab"], case["dim"])      # of the micro-batch before
    elif case["op"] in ("logp", "logp_grad"):
        rows, cols = case["rows"], case["cols"]
        if case["ragged"]:
            u = torch.rand(rows, generator=g, device="cuda", dtype=torch.float64) + 0.02
            end = (u.cumsum(0) / u.sum() * (rows * (cols - 1))).long().clamp_(max=rows * (cols - 1))
            end[-1] = rows * (cols - 1)
            s["row_ptr"] = torch.cat([end.new_zeros(1), end + 1 + torch.arange(rows, device="cuda")]).int()
            length = torch.diff(s["row_ptr"].long())
            s["width"], shape = int(length.max()), (rows * cols,)
        else:
            length = torch.full((rows,), cols, device="cuda")
            s["row_ptr"], s["width"], shape = None, cols, (rows, cols)
        s["logits"] = (2.5 * randn(*shape)).to(TYPES[case["type"]])
        u = torch.rand(rows, generator=g, device="cuda", dtype=torch.float64)
        s["ids"] = (u * length).long().clamp_(max=length - 1).int()
        s["mask"] = None
        if case["mask"] == "own":
            s["mask"] = (torch.rand(*shape, generator=g, device="cuda") < 0.6).to(torch.uint8)
            if case["ragged"]:
                first = s["row_ptr"][:-1].long()
                s["mask"][first] = 1                               # each state's first slot may always be taken
                s["mask"][first + s["ids"].long()] = 1
            else:
                s["mask"].scatter_(1, s["ids"].long()[:, None], 1)
                if rows > 8:
                    s["mask"][3] = 0                               # nothing applies
        elif case["mask"] == "shared":
            s["mask"] = (torch.rand(cols, generator=g, device="cuda") < 0.6).to(torch.uint8)
            s["mask"][0] = 1
        if rows > 8:
            s["ids"][5] = -1                                       # no token given
        s["dlogp"], s["dentropy"] = randn(rows) / rows, -0.01 * torch.ones(rows, device="cuda") / rows
    else:
        W, G, M, mats, at = [], [], [], [], 0
        for r, k in _shapes(case):
            rank = max(1, min(r, k) // 4)

            def low():           # gradients: a spectrum that falls off, over noise
                fall = torch.arange(1, rank + 1, device="cuda", dtype=torch.float32) ** -0.5
                return 1e-3 * ((randn(r, rank) * fall) @ randn(rank, k) / math.sqrt(rank) + 0.1 * randn(r, k))
            W.append(randn(r, k).mul_(math.sqrt(2.0 / r)).flatten())
            G.append(low().flatten())
            M.append(3.0 * low().flatten())
            mats.append((at, r, k))
            at += r * k
        s |= dict(weights=torch.cat(W), grads=torch.cat(G), momentum=torch.cat(M), matrices=np.array(mats, np.int64))
    return s


MUON = dict(lr=0.02, beta=0.95, nesterov=True, weight_decay=0.01, steps=5, rms=0.2)


def _own():
    """The library's context: one for the program, on its stream."""
    global _encoder
    if _encoder is None:
        import paper_2304_14698_amd as xrl
        model = dict(n_op_types=40, n_node_dense=0, d_edge=4, d_global=0, hidden=64, rounds=0)
        _encoder = xrl.Encoder(model, np.zeros(xrl.weight_count(model), np.float32))
    return _encoder


def _run_own(s):
    c, enc = s["case"], _own()
    if c["op"] == "embed":
        return enc.embedding(s["table"], s["ids"], scale=c["scale"], dtype=TYPES[c["out"]])
    if c["op"] == "embed_grad":
        return enc.embedding_backward(s["dout"], s["ids"], s["dtable"], scale=c["scale"])
    if c["op"] in ("logp", "logp_grad"):
        rows = dict(mask=s["mask"], row_ptr=s["row_ptr"], temperature=c["temperature"])
        f = enc.token_logp(s["logits"], s["ids"], top_k=c["top_k"], **rows)
        out = dict(logp=f["logp"], entropy=f["entropy"])
        if c["top_k"]:
            out |= dict(top_ids=f["top_ids"], top_logp=f["top_logp"])
        if c["op"] == "logp_grad":
            out["dlogits"] = enc.token_logp_backward(s["logits"], s["ids"], f, s["dlogp"], s["dentropy"], **rows)
        return out
    enc.muon_step(s["weights"], s["grads"], s["momentum"], s["matrices"], **MUON)
    return dict(weights=s["weights"], momentum=s["momentum"])


def _dense(s, flat, fill):
    """Ragged rows as a dense matrix, `fill` behind a row's end."""
    ptr = s["row_ptr"].long()
    j = torch.arange(s["width"], device="cuda")
    at = ptr[:-1, None] + j
    inside = at < ptr[1:, None]
    return torch.where(inside, flat[at.clamp(max=flat.numel() - 1)], fill), inside


def _plain_logp(s):
    c = s["case"]
    ragged, inf = c["ragged"], float("inf")
    x = s["logits"].float()
    if ragged:
        x, inside = _dense(s, x, -inf)
    if s["mask"] is not None:
        ok = _dense(s, s["mask"], 0)[0] if ragged else s["mask"]
        x = torch.where(ok != 0, x, -inf)
    n, width = x.shape
    scale = 1.0 / c["temperature"]
    top = x.amax(1, keepdim=True).clamp(min=torch.finfo(torch.float32).min)
    z = (x - top) * scale
    e = z.exp()
    total = e.sum(1, keepdim=True)
    any_ = total > 0
    lp = z - total.log()
    p = e / torch.where(any_, total, 1.0)
    H = -(p * torch.where(p > 0, lp, 0.0)).sum(1)
    ids = s["ids"].long()
    given = torch.gather(lp, 1, ids.clamp(0, width - 1)[:, None])[:, 0]
    given = torch.where(any_[:, 0], given, -inf)
    out = dict(logp=torch.where(ids < 0, 0.0, given), entropy=H)
    if c["top_k"]:
        k = min(c["top_k"], width)
        bits = (x + 0.0).view(torch.int32)
        key = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long() * (1 << 32) + (width - 1 - torch.arange(width, device="cuda"))
        at = width - 1 - (key.topk(k, 1)[0] & 0xFFFFFFFF)
        best = torch.gather(x, 1, at) > -inf
        ids_k = torch.full((n, c["top_k"]), -1, dtype=torch.int32, device="cuda")
        lp_k = torch.full((n, c["top_k"]), -inf, device="cuda")
        ids_k[:, :k] = torch.where(best, at, -1).int()
        lp_k[:, :k] = torch.where(best, torch.gather(lp, 1, at), -inf)
        out |= dict(top_ids=ids_k, top_logp=lp_k)
    if c["op"] == "logp_grad":
        g = torch.where((ids >= 0) & (given > -inf), s["dlogp"], 0.0)[:, None]
        d = p * (-g - s["dentropy"][:, None] * (torch.where(p > 0, lp, 0.0) + H[:, None]))
        d = scale * d.scatter_add_(1, ids.clamp(0, width - 1)[:, None], g)
        if ragged:
            d = d[inside]
        out["dlogits"] = d.to(s["logits"].dtype)
    return out


def _plain_muon(s):
    a, b, c = NS
    for at, r, k in s["matrices"].tolist():
        w, g, m = (s[n][at:at + r * k].view(r, k) for n in ("weights", "grads", "momentum"))
        m.mul_(MUON["beta"]).add_(g)
        u = g + MUON["beta"] * m
        x = u.T if r > k else u
        x = x / ((x * x).sum().sqrt() + 1e-7)
        for _ in range(MUON["steps"]):
            A = x @ x.T
            x = a * x + (b * A + c * (A @ A)) @ x
        x = x.T if r > k else x
        w.mul_(1 - MUON["lr"] * MUON["weight_decay"]).add_(x, alpha=-MUON["lr"] * MUON["rms"] * math.sqrt(max(r, k)))
    return dict(weights=s["weights"], momentum=s["momentum"])


def run(state):
    s, c = state, state["case"]
    if own:
        return _run_own(s)
    if c["op"] == "embed":
        return (s["table"][s["ids"].long()].float() * c["scale"]).to(TYPES[c["out"]])
    if c["op"] == "embed_grad":
        ids = s["ids"].long()
        rows = s["dout"].float() * c["scale"] * (ids >= 0)[:, None]
        return s["dtable"].index_add_(0, ids.clamp(min=0), rows)
    return _plain_muon(s) if c["op"] == "muon" else _plain_logp(s)


def work(case):
    size = {"fp32": 4, "bf16": 2}
    if case["op"] == "embed":
        n, d = case["n"], case["dim"]
        rows = case["vocab"] * (1 - (1 - 1 / case["vocab"]) ** n)        # distinct rows, at most
        return {"bytes": 4 * n + min(rows, n) * d * size[case["table"]] + n * d * size[case["out"]], "flops": n * d}
    if case["op"] == "embed_grad":
        n, d, v = case["n"], case["dim"], case["vocab"]
        if case["spread"] == "even":
            rows = v * (1 - (1 - 1 / v) ** n)
        else:                    # rank r has the share log((r + 2)/(r + 1)) / log(v + 1)
            share = np.log1p(1.0 / np.arange(1, v + 1)) / math.log(v + 1)
            rows = float((1 - (1 - share) ** n).sum())
        return {"bytes": 4 * n + n * d * size[case["dout"]] + 8 * rows * d, "flops": n * d}
    if case["op"] in ("logp", "logp_grad"):
        n = case["rows"] * case["cols"]
        mask = {"none": 0, "own": n, "shared": case["cols"]}[case["mask"]]
        once = n * size[case["type"]] + mask + case["rows"] * (12 + 8 * case["top_k"])
        more = (n * size[case["type"]] + 8 * case["rows"]) if case["op"] == "logp_grad" else 0
        return {"bytes": once + more, "flops": n * (6 if case["op"] == "logp" else 12)}
    nbytes = flops = 0.0
    for r, k in _shapes(case):
        m, n = min(r, k), max(r, k)
        nbytes += 20.0 * m * n
        flops += MUON["steps"] * (3.0 * m * m * n + 1.0 * m * m * m)      # symmetric products: one triangle
    return {"bytes": nbytes, "flops": flops}


def exact(case, seed):
    s = prepare(case, seed)
    c = case
    if c["op"] == "embed":
        return s["table"].double().mul_(c["scale"]).index_select(0, s["ids"].long())
    if c["op"] == "embed_grad":
        # sums over runs of equal ids as differences of a running sum in 64 bits, of columns a slab at a time
        keep = s["ids"] >= 0
        ids, order = torch.sort(s["ids"][keep].long(), stable=True)
        out = s["dtable"].double()
        end = torch.cat([ids[1:] != ids[:-1], torch.ones_like(ids[:1], dtype=torch.bool)]).nonzero()[:, 0]
        for lo in range(0, c["dim"], 256):
            run = (s["dout"][keep][:, lo:lo + 256].double()[order]).cumsum(0)[end]
            out[ids[end], lo:lo + 256] += c["scale"] * torch.diff(run, dim=0, prepend=torch.zeros_like(run[:1]))
        return out
    if c["op"] == "muon":
        p1, p3, p5 = NS
        W, M = s["weights"].double(), s["momentum"].double()
        M = MUON["beta"] * M + s["grads"].double()
        U = s["grads"].double() + MUON["beta"] * M
        for at, r, k in s["matrices"].tolist():
            u = U[at:at + r * k].view(r, k)
            u = u / (u.norm() + 1e-7)
            # X_k = P_k X_0 (or X_0 P_k): the polynomial runs on the smaller Gram matrix alone
            K = u @ u.T if r <= k else u.T @ u
            P = eye = torch.eye(min(r, k), dtype=torch.float64, device="cuda")
            for _ in range(MUON["steps"]):
                A = P @ K @ P.T
                P = (p1 * eye + p3 * A + p5 * (A @ A)) @ P
            x = P @ u if r <= k else u @ P.T
            W[at:at + r * k] *= 1 - MUON["lr"] * MUON["weight_decay"]
            W[at:at + r * k] -= (MUON["lr"] * MUON["rms"] * math.sqrt(max(r, k)) * x).flatten()
        return dict(weights=W, momentum=M)
    # one row (or, dense, a few hundred) at a time from the definition p = exp(x) / sum exp(x)
    rows, k = c["rows"], c["top_k"]
    logp = torch.empty(rows, dtype=torch.float64, device="cuda")
    H = torch.empty_like(logp)
    top = torch.full((rows, k), -math.inf, dtype=torch.float64, device="cuda")
    grad = torch.zeros(s["logits"].shape, dtype=torch.float64, device="cuda")
    ptr = s["row_ptr"].tolist() if c["ragged"] else None
    step = 1 if c["ragged"] else 512
    for lo in range(0, rows, step):
        hi = min(rows, lo + step)
        at = slice(ptr[lo], ptr[hi]) if c["ragged"] else slice(lo, hi)
        y = s["logits"][at].double().view(hi - lo, -1) / c["temperature"]
        if s["mask"] is not None:
            y = y.masked_fill((s["mask"] if c["mask"] == "shared" else s["mask"][at].view(hi - lo, -1)) == 0, -math.inf)
        q = torch.log_softmax(y, 1)
        none = torch.isneginf(y).all(1)
        q = q.masked_fill(none[:, None], -math.inf)
        prob = q.exp()
        H[lo:hi] = torch.special.entr(prob).sum(1)
        ids = s["ids"][lo:hi].long()
        r = torch.arange(hi - lo, device="cuda")
        got = q[r, ids.clamp(min=0)]
        logp[lo:hi] = got.masked_fill(ids < 0, 0.0)
        if k:
            best = q.sort(1, descending=True)[0][:, :k]
            top[lo:hi, :best.shape[1]] = best
        if c["op"] == "logp_grad":
            g = s["dlogp"][lo:hi].double().masked_fill((ids < 0) | torch.isneginf(got), 0.0)
            one = torch.zeros_like(q)
            one[r, ids.clamp(min=0)] = g
            # of H: the derivative of sum -p ln p through p's own Jacobian
            v = -(q.masked_fill(prob == 0, 0.0) + 1.0) * s["dentropy"][lo:hi, None].double()
            d = one - prob * g[:, None] + prob * (v - (prob * v).sum(1, keepdim=True))
            grad[at] = (d / c["temperature"]).view(grad[at].shape)
    out = dict(logp=logp, entropy=H)
    if k:
        out |= dict(top_ids=None, top_logp=top)
    if c["op"] == "logp_grad":
        out["dlogits"] = grad
    return out
