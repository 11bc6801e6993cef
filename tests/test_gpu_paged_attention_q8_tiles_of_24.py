"""Attention over an 8-bit cache in tiles of 24 rows, which 17 to 24 rows to a cache head take where a CTA's share of the keys is long:
max_kv_len alone says so, whatever the lengths are.  Against the definition, with the tolerance of the operator's own test."""
import pytest

from test_gpu_paged_attention_q8 import PagedQ8, both

pytestmark = pytest.mark.gpu
LONG = 1 << 22      # keys that shares are planned for


@both
@pytest.mark.parametrize("page,block", [(8, 1), (16, 16), (128, 32), (4096, 64)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("group,tokens", [(8, 3), (5, 4), (18, 1), (23, 1)])
@pytest.mark.parametrize("heads_kv", [1, 2, 3, 4, 8])
def test_heads_pages_and_blocks(heads_kv, group, tokens, d, page, block, dtype):
    lens = [(tokens, 77), (tokens, 500), (tokens, tokens), (1, 260), (0, 9)]
    p = PagedQ8(lens, group * heads_kv, heads_kv, d, page, block=block, seed=page + group, dtype=dtype, pad=2)
    p.check(p.attend(max_kv_len=LONG))


@both
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window,sinks", [(300, 4), (150, 150)])
def test_windows_and_scales(window, sinks, d, dtype):
    """A window bounds the keys that shares are planned for; a large batch makes them long all the same.  The first sequences are looked at."""
    lens = [(3, 77), (3, 900), (3, 3), (1, 260), (2, 500), (0, 5)] + [(1 + i % 3, 3 + i % 40) for i in range(506)]
    p = PagedQ8(lens, 48, 8, d, 16, block=8, seed=window, window=window, sinks=sinks, dtype=dtype, spread=1.0, q_gain=0.2)
    assert (window + sinks + 3) * 8 * len(lens) >= 32 * 128 * 2 * 148
    out = p.attend(max_kv_len=LONG)
    p.lens = lens[:20]
    p.check(out)


@both
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("heads_kv", [1, 4])
def test_scales(heads_kv, d, dtype):
    lens = [(4, 77), (3, 900), (4, 4), (1, 260)]
    p = PagedQ8(lens, 6 * heads_kv, heads_kv, d, 16, block=2, seed=7, dtype=dtype, spread=2.0, q_gain=0.05)
    p.check(p.attend(max_kv_len=LONG))
