"""Attention over the paged caches with scores as large as the operators take them: 2^28 times log2 e over a bf16 cache, 2^22 over 8-bit
ones.  Their rounding is as large as what softmax tells apart, so which keys have the weight is open; but a result is a mean of
values that its query sees, within the roundings of weights and result."""
import math

import pytest
import torch

from test_gpu_paged_attention_q8 import E4, I8, PagedQ8

pytestmark = pytest.mark.gpu


def largest_score(q, keys, group):
    """Of all queries and keys, in powers of two."""
    k = keys.repeat_interleave(group, 1).double()
    return (torch.einsum("thd,jhd->htj", q.double(), k).abs().max() * q.shape[2] ** -0.5 / math.log(2)).item()


def in_hull(out, v, group):
    v = v.repeat_interleave(group, 1).double()
    slack = 2 ** -7 * v.abs().amax(0)
    assert bool(((out.double() <= v.amax(0) + slack) & (out.double() >= v.amin(0) - slack)).all())
    assert bool(out.any(-1).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, I8, E4], ids=["bf16", "int8", "e4m3"])
@pytest.mark.parametrize("heads,heads_kv,d", [(8, 2, 64), (8, 2, 128), (24, 4, 128), (5, 1, 64)])
@pytest.mark.parametrize("tokens", [1, 3, 5, 16, 40, 100])
def test_largest_scores(tokens, heads, heads_kv, d, dtype):
    from paper_2511_03586_b200 import api
    group, kv = heads // heads_kv, 700
    if dtype == torch.bfloat16:
        g = torch.Generator(device="cuda").manual_seed(tokens)
        keys, values = (torch.randn(kv, heads_kv, d, generator=g, device="cuda").bfloat16() for _ in range(2))
        q = torch.randn(tokens, heads, d, generator=g, device="cuda").bfloat16()
        pages = -(-kv // 16)
        caches = [torch.zeros(pages * 16, heads_kv, d, dtype=dtype, device="cuda") for _ in range(2)]
        for c, x in zip(caches, (keys, values)):
            c[:kv] = x
        table = torch.arange(pages, dtype=torch.int32, device="cuda")[None]
        ints = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
        limit = 2.0 ** 28
    else:
        p = PagedQ8([(tokens, kv)], heads, heads_kv, d, 16, seed=tokens, dtype=dtype)
        keys, values, q, limit = p.k_seq[0], p.v_seq[0], p.q, 2.0 ** 22
    for gain in (0.99, 0.7, 0.3):
        grown = (q.float() * (gain * limit / largest_score(q, keys, group))).bfloat16()
        assert largest_score(grown, keys, group) < limit
        if dtype == torch.bfloat16:
            out = api.pd_attention_paged_fwd(grown, *(c.view(pages, 16, heads_kv, d) for c in caches), table, ints(0, tokens), ints(kv),
                                             max_q_len=tokens, max_kv_len=kv)
        else:
            p.q = grown
            out = p.attend()
        assert api.pd_get_device_status() == 0
        in_hull(out, values, group)
