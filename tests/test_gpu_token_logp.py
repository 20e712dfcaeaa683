"""Log-probabilities of given entries, entropy, best entries and the gradient to the logits, against the formulas in 64 bits.

Tolerances. u = 2^-24. A row's sum S of e^y is fp32: a lane adds up to L = cols / 64 + 8 terms, each with an exponential off by
two units and by the rounding of its argument (|t| units; weighted with the terms themselves, that is their mean, at most
2 log2(cols) + 4 on these inputs), and rescales at most L times: S is off by at most D = (3 L + 64 + 4 log2 cols) u of itself. So
is W = sum e^t t, whose terms have one sign. The rest is a handful of roundings of the numbers at hand."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
INF = math.inf


@pytest.fixture(scope="module")
def enc():
    import torch
    assert torch.cuda.is_available(), "these tests need the GPU"
    import paper_2304_14698_amd as xrl
    model = dict(n_op_types=4, n_node_dense=0, d_edge=4, d_global=0, hidden=64, rounds=0)
    e = xrl.Encoder(model, np.zeros(xrl.weight_count(model), np.float32))
    yield e
    e.close()


def one_row(x, mask, id, k, temperature, g, h):
    """The formulas for one row of float64 logits (numpy)."""
    T = float(np.float32(1) / np.float32(temperature))
    ok = np.isfinite(x) if mask is None else np.isfinite(x) & (mask != 0)
    n = len(x)
    top_ids, top_logp = np.full(k, -1), np.full(k, -INF)
    grad = np.zeros(n)
    if not ok.any():
        return dict(logp=0.0 if id < 0 else -INF, entropy=0.0, top_ids=top_ids, top_logp=top_logp, grad=grad, p=grad, lp=grad, m=0.0, A=0.0)
    m = x[ok].max()
    lp = np.full(n, -INF)
    y = (x[ok] - m) * T
    lp[ok] = y - math.log(np.exp(y).sum())
    p = np.exp(lp)
    H = -(p[ok] * lp[ok]).sum()
    far = lp < -3.4028235e38                             # beyond fp32
    taken = 0 <= id < n and ok[id]
    logp = 0.0 if id < 0 else (lp[id] if taken else -INF)
    order = sorted(np.flatnonzero(ok), key=lambda j: (-x[j], j))[:k]
    top_ids[:len(order)], top_logp[:len(order)] = order, np.where(far[order], -INF, lp[order])
    gg = g if taken else 0.0
    grad[ok] = T * (-p[ok] * (gg + h * (lp[ok] + H)))
    A = T * abs(gg + h * H)
    if taken:
        grad[id] += T * gg
    return dict(logp=logp, entropy=H, top_ids=top_ids, top_logp=top_logp, grad=grad, p=p, lp=np.where(ok, lp, 0.0), m=m, A=A, taken=taken)


def check_rows(rows, masks, ids, k, temperature, dlogp, dentropy, got, dgot, bf16):
    T = 1.0 / temperature
    for r, x in enumerate(rows):
        w = one_row(x, masks[r], int(ids[r]), k, temperature, float(dlogp[r]), float(dentropy[r]))
        n = max(len(x), 2)
        D = (3 * (n / 64 + 8) + 64 + 4 * math.log2(n)) * U
        H = w["entropy"]
        if math.isfinite(w["logp"]):
            assert abs(got["logp"][r] - w["logp"]) <= D + 6 * U * (abs(w["logp"]) + math.log(n)) , (r, got["logp"][r], w["logp"])
        else:
            assert got["logp"][r] == w["logp"], r
        assert abs(got["entropy"][r] - H) <= D * (1 + 2 * (math.log(n) + H)) + 8 * U * (math.log(n) + H), (r, got["entropy"][r], H)
        if k:
            np.testing.assert_array_equal(got["top_ids"][r], w["top_ids"])
            there = np.isfinite(w["top_logp"])
            assert (np.abs(got["top_logp"][r][there] - w["top_logp"][there]) <= D + 6 * U * (np.abs(w["top_logp"][there]) + math.log(n))).all()
            assert (got["top_logp"][r][~there] == -INF).all()
        if dgot is not None:
            p, lp, h = w["p"], np.abs(w["lp"]), abs(float(dentropy[r]))
            size = p * (w["A"] + T * h * lp)
            bound = size * (16 * U + 8 * U * lp + 2 * D) + p * T * h * (D * (1 + 2 * (math.log(n) + H)) + 8 * U * (lp + H + math.log(n)))
            bound = bound + 8 * U * (np.abs(w["grad"]) + (T * abs(float(dlogp[r])) if w.get("taken") else 0.0) * (np.arange(len(x)) == int(ids[r])))
            if bf16:
                bound = bound + 2.0 ** -8 * (np.abs(w["grad"]) + bound) + 1e-38
            off = np.abs(dgot[r] - w["grad"])
            assert (off <= bound + 1e-44).all(), (r, float((off - bound).max()))
            dead = p == 0 if masks[r] is None else (masks[r] == 0) | (p == 0)
            assert (dgot[r][dead] == 0).all()


def run_case(enc, x, mask, ids, k, temperature, seed=0, row_ptr=None, in_place=False):
    """x: numpy float32 already of the type's values, with its torch tensor."""
    import torch
    n = len(ids)
    rng = np.random.Generator(np.random.PCG64(seed + 1))
    dlogp, dent = rng.standard_normal(n).astype(np.float32), rng.standard_normal(n).astype(np.float32)
    t = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    kw = dict(mask=mask, row_ptr=row_ptr, temperature=temperature)
    tids = t(ids.astype(np.int32))
    f = enc.token_logp(x, tids, top_k=k, **kw)
    f2 = enc.token_logp(x, tids, top_k=k, **kw)
    d = enc.token_logp_backward(x, tids, f, t(dlogp), t(dent), **kw)
    if in_place:
        y = x.clone()
        enc.token_logp_backward(y, tids, f, t(dlogp), t(dent), out=y, **kw)
        torch.cuda.synchronize()
        assert torch.equal(y, d)
    torch.cuda.synchronize()
    for key in f:
        a, b = f[key], f2[key]
        assert torch.equal(torch.nan_to_num(a.float(), nan=123.0), torch.nan_to_num(b.float(), nan=123.0)), key
    return {key: v.cpu().numpy().astype(np.float64) if v.is_floating_point() else v.cpu().numpy() for key, v in f.items()}, d, dlogp, dent


def inputs(rng, rows, cols, type, spread=2.5):
    import torch
    x = torch.from_numpy((spread * rng.standard_normal((rows, cols))).astype(np.float32)).to(type)
    return x, x.double().numpy()


@pytest.mark.parametrize("type", ["fp32", "bf16"])
@pytest.mark.parametrize("masked", ["none", "own", "shared"])
@pytest.mark.parametrize("rows,cols,k,temperature", [
    (1, 1, 1, 1.0), (3, 2, 4, 0.7), (5, 9, 3, 1.0), (7, 64, 64, 2.0), (4, 513, 1, 1.0), (6, 1024, 8, 0.7), (5, 1025, 5, 1.0),
    (9, 2051, 0, 1.3), (3, 4099, 64, 1.0), (2, 12289, 16, 0.7), (1, 50021, 8, 1.0), (70, 3001, 2, 1.0)])
def test_dense_rows(enc, type, masked, rows, cols, k, temperature):
    import torch
    dt = dict(fp32=torch.float32, bf16=torch.bfloat16)[type]
    rng = np.random.Generator(np.random.PCG64(rows * 1000 + cols))
    x, x64 = inputs(rng, rows, cols, dt)
    ids = rng.integers(0, cols, rows)
    masks, tm = [None] * rows, None
    if masked == "own":
        m = (rng.random((rows, cols)) < 0.6).astype(np.uint8) * rng.integers(1, 256, (rows, cols)).astype(np.uint8)
        m[0] = 0                                          # nothing to choose
        masks, tm = list(m), torch.from_numpy(m).cuda()
    elif masked == "shared":
        m = (rng.random(cols) < 0.5).astype(np.uint8)
        masks, tm = [m] * rows, torch.from_numpy(m).cuda()
    if rows > 2:
        ids[1], ids[2] = -1, cols                        # no token; behind the row's end
    x = x.cuda()
    got, d, dlogp, dent = run_case(enc, x, tm, ids, k, temperature, in_place=True)
    check_rows(x64, masks, ids, k, temperature, dlogp, dent, got, d.double().cpu().numpy(), type == "bf16")


@pytest.mark.parametrize("type", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,most", [(1, 5), (33, 130), (5, 9000), (3, 40000)])
def test_ragged_rows(enc, type, rows, most):
    """Slots of states: rows of every length, empty ones among them, at every alignment; their masks."""
    import torch
    dt = dict(fp32=torch.float32, bf16=torch.bfloat16)[type]
    rng = np.random.Generator(np.random.PCG64(rows + most))
    length = rng.integers(0, most, rows)
    length[-1] = most
    if rows > 4:
        length[1], length[3] = 0, 1
    ptr = np.concatenate([[0], np.cumsum(length)]).astype(np.int32)
    x, x64 = inputs(rng, 1, int(ptr[-1]), dt)
    mask = (rng.random(int(ptr[-1])) < 0.7).astype(np.uint8)
    ids = np.array([rng.integers(0, max(1, n)) for n in length])
    for m in (None, mask):
        got, d, dlogp, dent = run_case(enc, x[0].contiguous().cuda(), None if m is None else torch.from_numpy(m).cuda(), ids, 4, 0.9,
                                       row_ptr=torch.from_numpy(ptr).cuda(), in_place=True)
        cut = lambda a: [a[ptr[r]:ptr[r + 1]] for r in range(rows)]  # noqa: E731
        check_rows(cut(x64[0]), [None] * rows if m is None else cut(m), ids, 4, 0.9, dlogp, dent, got,
                   cut(d.double().cpu().numpy()), type == "bf16")


def test_row_ends_outside_the_array_count_as_not_there(enc):
    import torch
    x = torch.arange(10, dtype=torch.float32, device="cuda")
    ptr = torch.tensor([-5, 4, 2, 40], dtype=torch.int32, device="cuda")
    f = enc.token_logp(x, None, row_ptr=ptr, top_k=2)
    torch.cuda.synchronize()
    assert f["top_ids"].tolist() == [[3, 2], [-1, -1], [7, 6]]
    assert "logp" not in f and float(f["entropy"][1]) == 0.0


@pytest.mark.parametrize("type", ["fp32", "bf16"])
@pytest.mark.parametrize("order", ["rising", "falling", "equal", "two values"])
@pytest.mark.parametrize("cols", [100, 5000, 40000])
def test_ties_and_sorted_rows(enc, type, order, cols):
    """Equal logits go to the lowest index, whichever wave or part holds them; sorted rows put every entry in or none."""
    import torch
    dt = dict(fp32=torch.float32, bf16=torch.bfloat16)[type]
    rng = np.random.Generator(np.random.PCG64(cols))
    x = np.linspace(-4, 4, cols)
    if order == "falling":
        x = x[::-1]
    if order == "equal":
        x = np.zeros(cols)
    if order == "two values":
        x = rng.integers(0, 2, cols) * 1.0
    x = torch.from_numpy(np.tile(x, (3, 1)).astype(np.float32)).to(dt)
    ids = np.array([0, cols // 2, cols - 1])
    for k in (1, 7, 64):
        got, d, dlogp, dent = run_case(enc, x.cuda(), None, ids, k, 1.0)
        check_rows(x.double().numpy(), [None] * 3, ids, k, 1.0, dlogp, dent, got, d.double().cpu().numpy(), type == "bf16")


@pytest.mark.parametrize("type", ["fp32", "bf16"])
@pytest.mark.parametrize("cols", [50, 3000, 20000])
def test_infinities_lowest_values_and_nan(enc, type, cols):
    import torch
    dt = dict(fp32=torch.float32, bf16=torch.bfloat16)[type]
    low = float(torch.finfo(dt).min)
    rng = np.random.Generator(np.random.PCG64(cols))
    x, _ = inputs(rng, 8, cols, dt)
    mask = np.ones((8, cols), np.uint8)
    x[0, ::3] = -INF                                     # masked by infinity
    x[1] = -INF                                          # all of it
    x[2, 1:] = low                                       # masked by the type's lowest value
    x[3] = low                                           # all of it: the same everywhere
    x[4, 5], mask[4, 5] = float("nan"), 0                # what stands in masked places is not looked at
    x[4, 6], mask[4, 6] = INF, 0
    mask[5] = 0
    x[5, 7] = float("nan")
    x[6, :] = low
    x[6, 9] = -low                                       # the difference overflows
    ids = np.array([1, 2, 0, 3, 7, 1, 9, 4])
    x64 = x.double().numpy()
    # where every finite logit is far below another, its difference is beyond fp32: -inf there, probability 0 either way
    got, d, dlogp, dent = run_case(enc, x.cuda(), torch.from_numpy(mask).cuda(), ids, 3, 1.0, in_place=False)
    clean = np.where(mask != 0, x64, 0.0)
    check_rows(clean, list(mask), ids, 3, 1.0, dlogp, dent, got, d.double().cpu().numpy(), type == "bf16")
    # a NaN or +inf that may be chosen reaches everything of its row, and no other
    for bad in (float("nan"), INF):
        y = x.clone()
        y[7, cols // 2] = bad
        g2, d2, _, _ = run_case(enc, y.cuda(), torch.from_numpy(mask).cuda(), ids, 3, 1.0)
        assert math.isnan(g2["logp"][7]) and math.isnan(g2["entropy"][7]) and np.isnan(g2["top_logp"][7]).all()
        assert torch.isnan(d2[7]).all()
        for key in ("logp", "entropy", "top_logp"):
            np.testing.assert_array_equal(g2[key][:7], got[key][:7])
        assert torch.equal(d2[:7], d[:7])


def test_rows_apart_at_any_address_and_many_rows(enc):
    import torch
    rng = np.random.Generator(np.random.PCG64(4))
    for dt, off in ((torch.bfloat16, 1), (torch.float32, 3)):
        rows, cols, ld = 6, 1501, 1512
        mem = torch.from_numpy(rng.standard_normal(off + rows * ld).astype(np.float32)).to(dt).cuda()
        x = mem[off:].view(rows, ld)[:, :cols]
        mmem = (torch.rand(rows * 1507 + 1) < 0.5).to(torch.uint8).cuda()
        mask = mmem[1:].view(rows, 1507)[:, :cols]
        ids = rng.integers(0, cols, rows)
        tids = torch.from_numpy(ids.astype(np.int32)).cuda()
        f = enc.token_logp(x, tids, mask=mask, top_k=3)
        g = enc.token_logp(x.contiguous(), tids, mask=mask.contiguous(), top_k=3)
        outm = torch.full((off + rows * 1600,), 7.0, dtype=dt, device="cuda")
        out = outm[off:].view(rows, 1600)[:, :cols]
        dl = torch.ones(rows, device="cuda")
        enc.token_logp_backward(x, tids, f, dl, mask=mask, out=out)
        want = enc.token_logp_backward(x.contiguous(), tids, g, dl, mask=mask.contiguous())
        torch.cuda.synchronize()
        for key in f:
            assert torch.equal(f[key], g[key]), key
        assert torch.equal(out, want)
        assert (outm[:off] == 7).all() and (outm[off:].view(rows, 1600)[:, cols:] == 7).all()
    # more rows than one launch takes
    rows = (1 << 22) + 5
    x = torch.zeros((rows, 2), device="cuda")
    x[-1, 1] = math.log(3.0)
    ids = torch.ones(rows, dtype=torch.int32, device="cuda")
    f = enc.token_logp(x, ids, top_k=1)
    d = enc.token_logp_backward(x, ids, f, torch.ones(rows, device="cuda"))
    torch.cuda.synchronize()
    assert abs(float(f["logp"][-1]) - math.log(0.75)) < 1e-6 and (f["logp"][:-1] == f["logp"][0]).all()
    assert f["top_ids"][-1, 0] == 1 and not f["top_ids"][:-1].any()
    assert (d[:-1] == torch.tensor([-0.5, 0.5], device="cuda")).all() and abs(float(d[-1, 0]) + 0.25) < 1e-6


@pytest.mark.parametrize("type", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(40, 700), (500, 9001), (700, 50000)])
def test_in_place_where_the_given_entry_may_not_be_chosen(enc, type, rows, cols):
    """Many blocks write a row, each over logits that the others need: the same bits as into memory of its own."""
    import torch
    dt = dict(fp32=torch.float32, bf16=torch.bfloat16)[type]
    g = torch.Generator(device="cuda").manual_seed(rows)
    x = torch.randn(rows, cols, generator=g, device="cuda").to(dt)
    ids = torch.randint(0, cols, (rows,), generator=g, device="cuda").int()
    ids[:8] = torch.tensor([0, cols - 1, cols // 2, 1, cols, -1, 5, 6], device="cuda").int()
    never = torch.arange(rows, device="cuda") % 4 != 3
    x[never.nonzero()[:, 0], ids.long().clamp(0, cols - 1)[never]] = -INF
    dlogp = torch.ones(rows, device="cuda")
    f = enc.token_logp(x, ids)
    want = enc.token_logp_backward(x, ids, f, dlogp, -0.5 * dlogp)
    for _ in range(3):
        y = x.clone()
        enc.token_logp_backward(y, ids, f, dlogp, -0.5 * dlogp, out=y)
        assert torch.equal(y, want)


def test_a_logp_below_the_lowest_value_keeps_its_gradient(enc):
    import torch
    x = torch.zeros(2, 5, device="cuda")
    x[:, 1] = torch.finfo(torch.float32).min
    x[1, 2] = -INF
    ids = torch.tensor([1, 2], device="cuda", dtype=torch.int32)
    f = enc.token_logp(x, ids, temperature=0.5)
    d = enc.token_logp_backward(x, ids, f, torch.ones(2, device="cuda"), temperature=0.5)
    assert f["logp"].tolist() == [torch.finfo(torch.float32).min, -INF]
    assert d[0, 1] == 2 and (d[0, [0, 2, 3, 4]] + 0.5).abs().max() < 1e-6 and (d[1] == 0).all()


@pytest.mark.parametrize("cols", [40, 2500])
def test_gradient_against_differences(enc, cols):
    """J = sum of a_r logp_r + b_r entropy_r in 64 bits by the formula, moved by +-e in single logits: the error of the difference is of
    order e^2 = 1e-8 of J's third derivatives (at most 2 here), the kernel's gradient as in the other tests below 1e-5 of the weights."""
    import torch
    rng = np.random.Generator(np.random.PCG64(cols))
    x, x64 = inputs(rng, 3, cols, torch.float32, 1.0)
    ids = rng.integers(0, cols, 3)
    got, d, a, b = run_case(enc, x.cuda(), None, ids, 0, 0.8)

    def J(y):
        tot = 0.0
        for r in range(3):
            w = one_row(y[r], None, int(ids[r]), 0, 0.8, 0.0, 0.0)
            tot += float(a[r]) * w["logp"] + float(b[r]) * w["entropy"]
        return tot
    e = 1e-4
    for r in range(3):
        for j in [int(ids[r])] + rng.integers(0, cols, 6).tolist():
            hi, lo = x64.copy(), x64.copy()
            hi[r, j] += e
            lo[r, j] -= e
            diff = (J(hi) - J(lo)) / (2 * e)
            assert abs(diff - float(d[r, j])) <= 1e-5 * (1 + abs(float(a[r])) + abs(float(b[r]))), (r, j)


def test_on_packed_states(enc):
    """Slots of packed states with the library's own heads: log-probabilities of the taken slots, entropy and the best slot are the heads'."""
    import torch
    import paper_2304_14698_amd as xrl
    import synth
    model, state = synth.make_config(3, n_states=5, n_cand=12)
    model["precision"] = "fp32"
    rng = np.random.Generator(np.random.PCG64(1))
    w = synth.init_weights(rng, xrl.weight_layout(model), bias_range=0.1)
    e = xrl.Encoder(model, w)
    batch = e.pack(state)
    pv = e.policy_value(batch, e.encode(batch))
    ptr = torch.from_numpy(np.ascontiguousarray(state["state_graph_ptr"], np.int32)).cuda()
    mask = torch.from_numpy(np.ascontiguousarray(state["slot_mask"], np.uint8)).cuda()
    f = e.token_logp(pv["logit"], pv["action"], mask=mask, row_ptr=ptr, top_k=3)
    torch.cuda.synchronize()
    scale = max(1.0, float(pv["logit"].abs().max()))
    at = ptr[:-1].long() + pv["action"].long()
    assert torch.equal(f["top_ids"][:, 0], pv["action"])
    assert (f["logp"] - pv["logp"][at]).abs().max() <= 1e-5 * scale
    assert (f["top_logp"][:, 0] - f["logp"]).abs().max() <= 4 * U * scale
    assert (f["entropy"] - pv["entropy"]).abs().max() <= 1e-5 * scale
    batch.free()
    e.close()


def test_nothing_to_do_and_refusals(enc):
    import torch
    import paper_2304_14698_amd as xrl
    x = torch.zeros((0, 7), device="cuda")
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    f = enc.token_logp(x, none, top_k=2)
    assert f["logp"].shape == (0,) and enc.token_logp_backward(x, none, f, f["logp"]).shape == (0, 7)
    x = torch.zeros((2, 0), device="cuda")
    ids = torch.zeros(2, dtype=torch.int32, device="cuda")
    f = enc.token_logp(x, ids, top_k=1)
    assert f["logp"].tolist() == [-INF, -INF] and f["entropy"].tolist() == [0, 0] and f["top_ids"].tolist() == [[-1], [-1]]
    x = torch.zeros((2, 7), device="cuda")
    f = enc.token_logp(x, ids)
    with pytest.raises(ValueError):
        enc.token_logp(x, ids.long())
    with pytest.raises(ValueError):
        enc.token_logp(x.half(), ids)
    with pytest.raises(ValueError):
        enc.token_logp(x, ids[:1])
    with pytest.raises(ValueError):
        enc.token_logp(x, ids, mask=torch.ones((2, 7), device="cuda"))
    with pytest.raises(ValueError):
        enc.token_logp(x, ids, mask=torch.ones((2, 6), dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError):
        enc.token_logp(x.T, ids)
    with pytest.raises(ValueError):
        enc.token_logp_backward(x, ids, f, f["logp"].double())
    for bad, code in ((dict(temperature=0.0), "VALUE"), (dict(temperature=-1.0), "VALUE"), (dict(temperature=float("nan")), "VALUE"),
                      (dict(temperature=1e-39), "VALUE"), (dict(top_k=65), "UNSUPPORTED")):
        with pytest.raises(xrl.XrlError) as ei:
            enc.token_logp(x, ids, **bad)
        assert ei.value.code == xrl.ERR[code]
    with pytest.raises(xrl.XrlError) as ei:
        enc.token_logp(x[:1].expand(2, 7), ids)          # rows on top of each other
    assert ei.value.code == xrl.ERR["SHAPE"]
    lib = xrl.load_library()
    assert lib.xrl_token_logp(enc.handle, None, None, 0, None, None, None, None, None) == xrl.ERR["NULL"]


def test_shapes_of_what_is_made_and_a_forward_without_log_probabilities(enc):
    import torch
    import paper_2304_14698_amd as xrl
    x = torch.randn(2, 3, 4, device="cuda")                  # ragged logits are taken flat, whatever their shape
    ptr = torch.tensor([0, 10, 24], dtype=torch.int32, device="cuda")
    ids = torch.tensor([9, 0], dtype=torch.int32, device="cuda")
    f = enc.token_logp(x, ids, row_ptr=ptr, top_k=3)
    one = torch.ones(2, device="cuda")
    d = enc.token_logp_backward(x, ids, f, one, row_ptr=ptr)
    assert d.shape == x.shape and d.is_contiguous() and f["stats"].shape == (2, 2) and f["top_ids"].shape == (2, 3)
    assert torch.equal(d.flatten(), enc.token_logp_backward(x.flatten(), ids, f, one, row_ptr=ptr))
    f = enc.token_logp(x, None, row_ptr=ptr)
    assert "logp" not in f
    assert enc.token_logp_backward(x, None, f, None, one, row_ptr=ptr).shape == x.shape
    with pytest.raises(xrl.XrlError) as ei:
        enc.token_logp_backward(x, ids, f, one, row_ptr=ptr)
    assert ei.value.code == xrl.ERR["NULL"]
