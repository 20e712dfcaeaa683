"""Packed attention where a block has nothing to go over, and where the ends of sequences are wrong. Oracle and tolerances: attention_checks.py."""
import pytest

from test_gpu_attention_packed import check, enc, ptr, tensors  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("type", ["fp32", "bf16"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dim", [64, 96, 128])
@pytest.mark.parametrize("nq,nk", [([0, 500], [300, 500]), ([500, 0, 200], [500, 400, 200]), ([600, 0], [600, 129]), ([0, 0], [300, 128]), ([700, 0, 1, 0], [200, 500, 300, 1])])
def test_keys_that_no_query_has(enc, type, causal, dim, nq, nk):  # noqa: F811
    """Sequences of many keys without queries, in front, between and behind: blocks of 128 keys that sum over nothing. Their gradients are 0, whatever lies beside them."""
    q_ptr, k_ptr = ptr(nq), ptr(nk)
    got = check(enc, *tensors(dim, sum(nq), sum(nk), 4, 2, dim, type), q_ptr, k_ptr, causal)
    for n, a, b in zip(nq, k_ptr[0][:-1], k_ptr[0][1:]):
        if n == 0:
            assert not got["dk"][a:b].any() and not got["dv"][a:b].any()
