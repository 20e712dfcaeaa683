"""Numbers of entries to keep that are larger than a row: the largest there are among them, which programs pass for "no limit"."""
import numpy as np
import pytest

from test_gpu_token_sample import check, draw, enc  # noqa: F401

pytestmark = pytest.mark.gpu
LARGE = [20000, 1 << 27, 1 << 28, (1 << 31) - 1]


@pytest.mark.parametrize("type", ["fp32", "bf16"])
@pytest.mark.parametrize("rest", [dict(), dict(top_p=0.9), dict(min_p=0.05), dict(top_p=0.8, min_p=0.01)])
def test_more_than_a_row_has_is_no_limit(enc, type, rest):  # noqa: F811
    import torch
    x, u, _ = draw(3, 4, 20000, type)
    want = check(enc, x, u, **rest)
    for k in LARGE:
        assert np.array_equal(check(enc, x, u, top_k=k, **rest), want), k
    ragged = torch.tensor([0, 20000, 20001, 20001, 80000], dtype=torch.int32, device="cuda")
    want = check(enc, x.reshape(-1), u, row_ptr=ragged, **rest)
    assert np.array_equal(check(enc, x.reshape(-1), u, row_ptr=ragged, top_k=LARGE[-1], **rest), want)


@pytest.mark.parametrize("k", LARGE)
def test_no_workspace_is_taken_for_them(k):
    """Looking at groups of entries first, which needs a workspace, is for the few that can be kept: a capture by a context that has none yet goes through."""
    import torch
    import paper_2304_14698_amd as xrl
    stream = torch.cuda.Stream()
    model = dict(n_op_types=4, n_node_dense=0, d_edge=4, d_global=0, hidden=64, rounds=0)
    x, u, _ = draw(5, 6, 20000, "bf16")
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        enc = xrl.Encoder(model, np.zeros(xrl.weight_count(model), np.float32))  # noqa: F811
        want = enc.token_sample(x, u)
        out = {name: torch.zeros_like(t) for name, t in want.items()}
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            enc.token_sample(x, u, top_k=k, out=out)
        for _ in range(3):
            for t in out.values():
                t.zero_()
            graph.replay()
            stream.synchronize()
            assert torch.equal(out["ids"], want["ids"]) and torch.equal(out["logp"], want["logp"])
        enc.close()


def test_numbers_past_32_bits(enc):  # noqa: F811
    """Are not read without their upper bits: no limit, and refused below 0."""
    import paper_2304_14698_amd as xrl
    x, u, _ = draw(7, 8, 500, "fp32")
    want = check(enc, x, u)
    for k in (1 << 31, (1 << 32) + 1, (1 << 40) + 3):
        assert np.array_equal(check(enc, x, u, top_k=k), want), k
    for k in (-(1 << 31), 1 - (1 << 32), -(1 << 40)):
        with pytest.raises(xrl.XrlError) as e:
            enc.token_sample(x, u, top_k=k)
        assert e.value.code == xrl.ERR["VALUE"]
