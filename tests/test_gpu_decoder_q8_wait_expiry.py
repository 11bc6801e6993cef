"""Bounded waits of the attention over 8-bit caches that run out: a code is recorded, the kernel drains and returns, and the next call
is right.  The loads are switched off (pd_debug_withhold_loads) and the limit is cut to one millisecond; nothing faults or hangs,
since no copy is in flight when the waits give up."""
import pytest
import torch

from test_gpu_decoder_wait_expiry import expired_code, withheld_loads
from test_gpu_paged_attention_q8 import E4, I8, PagedQ8

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [I8, E4], ids=["int8", "e4m3"])
@pytest.mark.parametrize("lens,codes", [([(1, 100), (1, 70)], (302,)), ([(1, 3000), (2, 40), (0, 0)], (302,)), ([(5, 900)], (302,)),
                                        ([(100, 300), (40, 40)], (312, 313)), ([(40, 4000)], (312, 313))],
                         ids=["rows", "rows joined", "more rows", "chunk", "chunk split"])
@pytest.mark.parametrize("heads", [(8, 2, 64), (8, 4, 128), (5, 1, 128)], ids=str)
def test_attention_whose_keys_do_not_arrive(lens, codes, heads, dtype):
    from paper_2511_03586_b200 import api
    p = PagedQ8(lens, *heads, 16, pad=3, dtype=dtype)
    out = torch.full_like(p.q, 3.0)
    with withheld_loads():
        p.attend(out=out)
        assert expired_code() in codes
    assert bool((out[sum(n for n, _ in lens):] == 3.0).all())      # padding stays as it was
    p.attend(out=out)
    p.check(out)
    assert api.pd_get_device_status() == 0
