"""Keys of score -inf in the cache do not count, whatever the heads' size, the column that holds the infinity, and where the cache lies: as in packed attention. Oracle and
tolerances: attention_checks.py, over the other keys."""
import math

import pytest

from attention_checks import close, one_head
from test_gpu_attention_cache import TYPES, Case, enc  # noqa: F401

pytestmark = pytest.mark.gpu


def oddly(x):
    """The same cache at addresses that are no multiples of 16 bytes."""
    import torch
    y = torch.zeros(*x.shape[:3], x.shape[3] + 1, dtype=x.dtype, device="cuda")[..., 1:]
    y.copy_(x)
    return y


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("dim", [8, 32, 40, 64, 80, 96, 128])
@pytest.mark.parametrize("column", [0, 3, 7])
@pytest.mark.parametrize("new,lengths", [([1, 2], [60, 40]), ([1, 2], [700, 300]), ([70, 3], [90, 200]), ([70, 90], [700, 300])])
def test_keys_of_no_weight(enc, type, dim, column, new, lengths):  # noqa: F811
    import torch
    heads, kv = 4, 2
    c = Case(dim + column, new, lengths, heads, kv, dim, 16, type)
    c.q[..., column] = c.q[..., column].abs() + 0.25
    c.write(enc)
    gone = [torch.arange(2 + s, m - new[s], 7) for s, m in enumerate(lengths)]      # of the tokens that were there before
    for s, js in enumerate(gone):
        c.kc[torch.from_numpy(c.table[s])[js // 16].cuda(), (js % 16).cuda(), :, column] = -math.inf
    got = enc.cache_attention(c.q, c.q_ptr, c.kc, c.vc, c.t, c.n)
    odd = enc.cache_attention(c.q, c.q_ptr, oddly(c.kc), oddly(c.vc), c.t, c.n)
    places = [[torch.from_numpy(x).cuda() for x in c.places(s, m)[:2]] for s, m in enumerate(lengths)]
    k, v = (torch.cat([x[pg, sl] for pg, sl in places]) for x in (c.kc, c.vc))
    k_ptr = torch.tensor([0, lengths[0], sum(lengths)], dtype=torch.int32, device="cuda")
    packed = enc.attention(c.q, k, v, c.q_ptr, k_ptr=k_ptr)["out"]
    torch.cuda.synchronize()
    half = 2.0 ** -8 if type == "bf16" else 0.0
    row = at = 0
    for s, (n, m) in enumerate(zip(new, lengths)):
        keep = torch.ones(m, dtype=torch.bool)
        keep[gone[s]] = False
        keep[m - n:] = False
        for h in range(heads):
            K, V = k[at:at + m, h * kv // heads].double(), v[at:at + m, h * kv // heads].double()
            for i in sorted({0, n // 2, n - 1}):
                see = keep.clone()
                see[m - n:m - n + i + 1] = True
                want = one_head(c.q[row + i:row + i + 1, h].double(), K[see.cuda()], V[see.cuda()], False, dim ** -0.5, half)["out"]
                for what, x in (("aligned", got), ("odd", odd), ("packed", packed)):
                    close(x[row + i:row + i + 1, h], want, (what, s, h, i))
        row, at = row + n, at + m
