"""Bounded waits of the paged attention and of the row-prefetching norms that run out: a code is recorded, the kernel drains and
returns, and the next call is right.

The producers are switched off (pd_debug_withhold_loads) and the limit is cut to one millisecond, so that every warp that
waits for a key tile or a row gives up.  Nothing faults or hangs: no copy is in flight when the waits give up."""
import ctypes
from contextlib import contextmanager

import pytest
import torch

from test_gpu_paged_attention import Paged

pytestmark = pytest.mark.gpu


@contextmanager
def withheld_loads():
    from paper_2511_03586_b200 import api
    api.pd_clear_device_status()
    api.pd_debug_set_wait_limit_ns(1_000_000)
    api.pd_debug_withhold_loads(True)
    try:
        yield
    finally:
        api.pd_debug_withhold_loads(False)
        api.pd_debug_set_wait_limit_ns(2_000_000_000)


def expired_code():
    from paper_2511_03586_b200 import api
    code = api.pd_get_device_status()                              # synchronises
    assert api._lib.pd_get_device_status(ctypes.byref(ctypes.c_int(0))) == 7   # PD_ERR_DEVICE_TIMEOUT
    api.pd_clear_device_status()
    return code


@pytest.mark.parametrize("lens,codes", [([(1, 100), (1, 70)], (302,)), ([(1, 3000), (2, 40), (0, 0)], (302,)),
                                        ([(100, 300), (40, 40)], (312, 313)), ([(40, 4000)], (312, 313))],
                         ids=["rows", "rows joined", "chunk", "chunk split"])
@pytest.mark.parametrize("d", [64, 128])
def test_attention_whose_keys_do_not_arrive(lens, codes, d):
    from paper_2511_03586_b200 import api
    p = Paged(lens, 8, 2, d, 16, pad=3)
    out = torch.full_like(p.q, 3.0)
    with withheld_loads():
        p.attend(out=out)
        assert expired_code() in codes
    assert bool((out[sum(n for n, _ in lens):] == 3.0).all())      # padding stays as it was
    p.attend(out=out)
    p.check(out)
    assert api.pd_get_device_status() == 0


@pytest.mark.parametrize("cols", [2048, 4096, 8192])
def test_norms_whose_rows_do_not_arrive(cols):
    from paper_2511_03586_b200 import api
    x = torch.randn(4000, cols, device="cuda").bfloat16()
    want = api.pd_norm_gate_residual_norm(x, x)
    h, n = torch.full_like(x, 3.0), torch.full_like(x, 3.0)
    with withheld_loads():
        api.pd_norm_gate_residual_norm(x, x, h=h, n=n)
        assert expired_code() == 321
    assert bool((h == 3.0).all()) and bool((n == 3.0).all())       # nothing is written
    api.pd_norm_gate_residual_norm(x, x, h=h, n=n)
    assert torch.equal(h, want[0]) and torch.equal(n, want[1])
    assert api.pd_get_device_status() == 0
