"""Queries rotated in place where the units of a head do not divide a warp (and where they do), in every layout of pairs: bit for bit what
the call that writes elsewhere gives, which the operator's own tests hold to the definition."""
import pytest
import torch

from test_gpu_rope_append import E4, I8, Append

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,rotary,interleaved", [(24, 24, False), (40, 40, False), (48, 16, True), (80, 80, False), (96, 96, False), (96, 64, True),
                                                  (112, 112, True), (160, 160, False), (192, 192, False), (248, 248, False), (8, 8, False),
                                                  (64, 64, False), (256, 256, False)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, I8, E4], ids=["bf16", "int8", "e4m3"])
@pytest.mark.parametrize("lens", [[(1, 9), (1, 500)], [(60, 100), (1, 20), (33, 90)], [(1000, 1003)]], ids=["single", "some", "long"])
def test_in_place(lens, dtype, d, rotary, interleaved):
    from paper_2511_03586_b200 import api
    if dtype != torch.bfloat16 and d % 16:
        pytest.skip("strides of an 8-bit cache are multiples of 16")
    a, b = (Append(lens, 10, 2, d, 16, dtype=dtype, rotary=rotary, interleaved=interleaved, seed=d, pad=2) for _ in range(2))
    b.q = b.q.clone()
    want = b.run(q_out=b.q.clone())
    args, named = a.args()
    assert api.pd_rope_kv_cache_append(*args, q=a.q, q_out=a.q, **named) is a.q
    assert torch.equal(a.q, want)
    for x, y in ((a.k_cache, b.k_cache), (a.v_cache, b.v_cache)):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
