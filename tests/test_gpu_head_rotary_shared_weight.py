"""One weight for the norms of queries and keys, whose gradient is one vector: both sums are added to it, in turn."""
import pytest

from test_gpu_head_rotary import TYPES, enc, freqs_of, inputs  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("n,heads,kv,dim", [(1, 1, 1, 8), (37, 5, 2, 20), (300, 4, 4, 64), (3000, 6, 2, 128), (50, 3, 1, 7)])
def test_one_vector_for_both(enc, type, n, heads, kv, dim):  # noqa: F811
    import torch
    q, k, pos, w, _ = inputs(n, n, heads, kv, dim, type, 1000)
    f = freqs_of(dim // 4 * 2)
    g = torch.Generator(device="cuda").manual_seed(n)
    dq, dk = (torch.randn(x.shape, generator=g, device="cuda").to(x.dtype) for x in (q, k))
    first = torch.randn(dim, generator=g, device="cuda")
    want, both = first.clone(), [first.clone() for _ in range(5)]
    # q's part, then k's: the same sums in the same order
    gq, _ = enc.head_rotary_backward(q, k, pos, f, dq, dk, q_weight=w, k_weight=w, dq_weight=want)
    _, gk = enc.head_rotary_backward(q, k, pos, f, dq, dk, q_weight=w, k_weight=w, dk_weight=want)
    for x in both:
        hq, hk = enc.head_rotary_backward(q, k, pos, f, dq, dk, q_weight=w, k_weight=w, dq_weight=x, dk_weight=x)
    torch.cuda.synchronize()
    assert torch.equal(gq, hq) and torch.equal(gk, hk)
    for x in both:
        assert torch.equal(x, want)


def test_parts_of_each_other_are_refused(enc):  # noqa: F811
    import torch
    import paper_2304_14698_amd as xrl
    q, k, pos, w, _ = inputs(1, 5, 2, 1, 32, "bf16", 100)
    v = torch.zeros(64, device="cuda")
    f = freqs_of(32)
    for a, b in ((0, 1), (31, 0)):
        with pytest.raises(xrl.XrlError) as e:
            enc.head_rotary_backward(q, k, pos, f, q, k, q_weight=w, k_weight=w, dq_weight=v[a:a + 32], dk_weight=v[b:b + 32])
        assert e.value.code == xrl.ERR["SHAPE"]
    enc.head_rotary_backward(q, k, pos, f, q, k, q_weight=w, k_weight=w, dq_weight=v[:32], dk_weight=v[32:])
    torch.cuda.synchronize()
    assert v.isfinite().all() and v.any()
