"""The gradient to ragged logits at entries that no row covers: 0, wherever they lie. Rows themselves have the bits that they have without such
entries around them (a row's sums do not depend on where it lies)."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def enc():
    import torch
    assert torch.cuda.is_available(), "these tests need the GPU"
    import paper_2304_14698_amd as xrl
    model = dict(n_op_types=4, n_node_dense=0, d_edge=4, d_global=0, hidden=64, rounds=0)
    e = xrl.Encoder(model, np.zeros(xrl.weight_count(model), np.float32))
    yield e
    e.close()


def gradients(enc, x, ids, ptr, dlogp, dentropy, **kw):
    """Into memory that held 7s, over the logits, and as the method makes it."""
    import torch
    f = enc.token_logp(x, ids, row_ptr=ptr, **kw)
    out = [enc.token_logp_backward(x, ids, f, dlogp, dentropy, row_ptr=ptr, out=torch.full_like(x, 7.0), **kw)]
    y = x.clone()
    out.append(enc.token_logp_backward(y, ids, f, dlogp, dentropy, row_ptr=ptr, out=y, **kw))
    held = torch.full_like(x, float("nan"))              # what the allocator hands out next
    del held
    out.append(enc.token_logp_backward(x, ids, f, dlogp, dentropy, row_ptr=ptr, **kw))
    torch.cuda.synchronize()
    return out


@pytest.mark.parametrize("type", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,length,front,behind", [(1, 5, 3, 0), (1, 5, 0, 1), (32, 65, 7, 100), (33, 64, 0, 5001), (5, 9000, 1201, 333), (3000, 9, 1, 70001),
                                                      (2, 3, 100003, 100001), (7, 0, 40, 9)])
def test_slack_around_the_rows(enc, type, rows, length, front, behind):
    import torch
    dt = dict(fp32=torch.float32, bf16=torch.bfloat16)[type]
    g = torch.Generator(device="cuda").manual_seed(rows + front)
    n = rows * length
    x = torch.randn(front + n + behind, generator=g, device="cuda").to(dt)
    mask = (torch.rand(x.numel(), generator=g, device="cuda") < 0.7).to(torch.uint8)
    ids = torch.randint(0, max(1, length), (rows,), generator=g, device="cuda").int()
    ptr = (torch.arange(rows + 1, device="cuda") * length + front).int()
    dlogp, dentropy = torch.randn(rows, generator=g, device="cuda"), torch.randn(rows, generator=g, device="cuda")
    inner = slice(front, front + n)
    for m in (None, mask):
        kw = dict(mask=None if m is None else m[inner].clone(), temperature=0.8)
        alone, tight = x[inner].clone(), ptr - front
        want = enc.token_logp_backward(alone, ids, enc.token_logp(alone, ids, row_ptr=tight, **kw), dlogp, dentropy, row_ptr=tight, **kw)
        for d in gradients(enc, x, ids, ptr, dlogp, dentropy, mask=m, temperature=0.8):
            assert torch.equal(d[inner], want)
            assert not d[:front].any() and not d[front + n:].any()


@pytest.mark.parametrize("type", ["fp32", "bf16"])
@pytest.mark.parametrize("n", [1, 10, 3001, 1 << 20])
def test_no_rows_at_all(enc, type, n):
    import torch
    dt = dict(fp32=torch.float32, bf16=torch.bfloat16)[type]
    none, f = torch.zeros(0, dtype=torch.int32, device="cuda"), torch.zeros(0, device="cuda")
    for end in (0, 5, -3, n):
        for d in gradients(enc, torch.randn(n, device="cuda").to(dt), none, torch.full((1,), end, dtype=torch.int32, device="cuda"), f, f):
            assert d.shape == (n,) and not d.any()


@pytest.mark.parametrize("ends", [[-5, 4, 4, 7], [2, 6, 40, 41], [-9, -2, 3, 5], [13, 0, 5], [5, 0, 2, 2, 30], [13, 2, 9, 0, 1], [10, 14, 2, 6], [50, 60], [-4, -1], [12, 3]])
def test_ends_outside_and_ends_that_fall(enc, ends):
    """Rows that do not overlap, wherever their ends lie: each entry has its row's gradient, or 0."""
    import torch
    n = 16
    x = torch.randn(n, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda")
    rows = len(ends) - 1
    ids, ptr = torch.zeros(rows, dtype=torch.int32, device="cuda"), torch.tensor(ends, dtype=torch.int32, device="cuda")
    a, b = torch.linspace(0.5, 2.0, rows, device="cuda"), torch.linspace(-1.0, 1.0, rows, device="cuda")
    want, at = torch.zeros(n, dtype=torch.float64), x.double().cpu()
    for r in range(rows):
        s = slice(min(max(ends[r], 0), n), min(max(ends[r + 1], 0), n))
        if s.start < s.stop:
            y = at[s].clone().requires_grad_()
            lp = torch.log_softmax(y, 0)
            (float(a[r]) * lp[0] - float(b[r]) * (lp.exp() * lp).sum()).backward()
            want[s] = y.grad
    # rows of at most 16 logits of size 4: sums and exponentials of a few dozen roundings, of terms below 10
    for d in gradients(enc, x, ids, ptr, a, b):
        d = d.double().cpu()
        assert (d - want).abs().max() < 200 * 2.0 ** -24 * 10
        assert not d[want == 0].any()


def test_many_rows_whose_ends_fall(enc):
    """Every second row lies backwards, rows of the second half in front of the first end."""
    import torch
    rows, length = 700, 3
    at = np.concatenate([np.arange(rows // 2) + 1000, np.arange(rows // 2)])   # where row r's three entries lie, in threes
    ends = np.empty(2 * rows, np.int32)
    ends[0::2], ends[1::2] = at * length, at * length + length                 # row 2 i covers; the way to the next is a row too, forwards or back
    ptr = torch.from_numpy(ends).cuda()
    n = 1500 * length
    x = torch.randn(n, device="cuda")
    ids = torch.zeros(2 * rows - 1, dtype=torch.int32, device="cuda")
    one = torch.ones(2 * rows - 1, device="cuda")
    cover = np.zeros(n, bool)
    for b, e in zip(ends[:-1], ends[1:]):
        cover[b:e] = True
    for d in gradients(enc, x, ids, ptr, one, None):
        got = d.cpu().numpy()
        assert not got[~cover].any() and (got[cover] != 0).all()
