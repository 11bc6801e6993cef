"""Attention over an 8-bit cache where the rows that a kernel computes together have little in common: a query that is infinite or not a
number, queries of very different magnitudes, values of very different magnitudes that only some of the rows see.  What a row gets follows
from its own query and from the keys in its own view.

The tolerance is that of the operator's own test (test_gpu_paged_attention_q8.py), with the largest value of the keys in the view of
each query in place of the largest of the sequence; in the kernel for chunks, where keys of several scales share 32 positions, of those 32."""
import math

import pytest
import torch

import decoder_reference as ref
from test_gpu_paged_attention_q8 import PagedQ8, both, quantised

pytestmark = pytest.mark.gpu

# new tokens and keys of the sequences, query heads, cache heads, head_dim: 4 to 64 rows to a cache head, and chunks
FORMS = [([(1, 300), (1, 77)], 8, 2, 128), ([(1, 900), (1, 77)], 8, 4, 64), ([(2, 300), (2, 77)], 16, 2, 128), ([(3, 700), (2, 77)], 8, 1, 64),
         ([(3, 700), (3, 77)], 32, 4, 64), ([(5, 700), (2, 77)], 24, 4, 128), ([(4, 300), (4, 77)], 16, 2, 64), ([(5, 400), (3, 90)], 20, 2, 128),
         ([(16, 300), (9, 77)], 8, 2, 128), ([(40, 300), (33, 77)], 8, 2, 128), ([(70, 300), (33, 77)], 8, 2, 64)]
forms = pytest.mark.parametrize("form", FORMS, ids=str)
row_forms = pytest.mark.parametrize("form", FORMS[:9], ids=str)


def rows_of(p):
    """Sequence, first row and new tokens."""
    at = 0
    for b, (n, kv) in enumerate(p.lens):
        yield b, at, n, kv
        at += n


def check(p, out, rows=None, around=1, each_key=True):
    """rows: of tokens and heads, the ones to look at.  around: aligned positions that share their largest key and value.  each_key: what a
    key may be off by below fp16's normal numbers counts for every key; else once, where the other keys' products are below it."""
    from paper_2511_03586_b200 import api
    assert api.pd_get_device_status() == 0
    for b, at, n, kv in rows_of(p):
        q, k, v = p.q[at:at + n], p.k_seq[b], p.v_seq[b]
        heads, d = q.shape[1:]
        group = heads // k.shape[1]
        scale = d ** -0.5
        want, mag = ref.attention(q, k, v, kv - n, window=p.window, sinks=p.sinks)
        pos, key = torch.arange(kv - n, kv, device="cuda")[:, None], torch.arange(kv, device="cuda")[None, :]
        seen = key <= pos
        if p.window:
            seen &= (key > pos - p.window) | (key < p.sinks)
        near = seen
        if around > 1:
            whole = torch.zeros(n, -(-kv // around) * around, dtype=torch.bool, device="cuda")
            whole[:, :kv] = seen
            near = whole.unflatten(1, (-1, around)).any(-1).repeat_interleave(around, 1)[:, :kv]
        # the largest value, and the largest key element by element, of what each query sees
        v_most = torch.where(near[:, :, None], v.abs().amax(2)[None], 0.0).amax(1).repeat_interleave(group, 1)[:, :, None]
        e = torch.zeros(n, heads, 1, dtype=torch.float64, device="cuda")
        for t in range(n):
            most = torch.where(near[t][:, None, None], k.abs(), 0.0).amax(0).repeat_interleave(group, 0)
            e[t] = 6 * 2 ** -11 / 3 ** 0.5 * (q[t].double() * most).pow(2).sum(-1, keepdim=True).sqrt() * scale
        count = (seen.sum(1).double() + 1)[:, None, None] if each_key else 1.0
        bound = (2 * 2 ** -11 + 2 ** -10) * mag + 2 ** -8 * want.abs() + e * (mag + want.abs()) + 2 ** -30 * count * v_most + 1e-30
        off = (out[at:at + n].double() - want).abs() / bound
        if rows is not None:
            off = off[rows[at:at + n]]
        assert bool((off <= 1.0).all()), (b, n, kv, off.nan_to_num(math.inf).max().item())


@both
@forms
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan, 3e38], ids=str)
def test_a_query_that_is_not_finite_harms_its_own_row_only(value, form, dtype):
    """Bit for bit: nothing that the others' results are made of may know of it.  (3e38: finite, its scores are not.)"""
    lens, *heads = form
    p = PagedQ8(lens, *heads, 16, seed=31, dtype=dtype)
    want = p.attend()
    p.check(want)
    bad = torch.zeros(p.q.shape[:2], dtype=torch.bool, device="cuda")
    bad[0, 1] = True
    if len(p.q) > 2:
        bad[-1, 0] = bad[len(p.q) // 2, -1] = True
    p.q[bad] = torch.where(torch.arange(heads[2], device="cuda") % 7 == 3, value, p.q[bad].float()).bfloat16()
    got = p.attend()
    assert torch.equal(got[~bad], want[~bad])


@both
@forms
@pytest.mark.parametrize("power", [28, 40, 100])
def test_queries_of_different_magnitudes(power, form, dtype):
    """One row 2^power times as large as the others, and one as much smaller.  (The large one's scores are beyond what the operator takes: nothing is
    asked of its own result.)"""
    lens, *heads = form
    p = PagedQ8(lens, *heads, 16, seed=32, dtype=dtype)
    large = torch.zeros(p.q.shape[:2], dtype=torch.bool, device="cuda")
    large[0, 0] = True
    p.q[0, 0] *= 2.0 ** power
    p.q[-1, -1] *= 2.0 ** -power
    check(p, p.attend(), ~large)


@both
@forms
def test_queries_of_zero_beside_others(form, dtype):
    lens, *heads = form
    p = PagedQ8(lens, *heads, 16, seed=33, dtype=dtype)
    p.q[0, 0] = 0
    p.q[-1, 1:] = 0
    check(p, p.attend())


@both
@forms
@pytest.mark.parametrize("factor", [2.0 ** -60, 2.0 ** 60])
def test_scales_of_keys_far_from_one(factor, form, dtype):
    lens, *heads = form
    for block in (4, 16):
        p = PagedQ8(lens, *heads, 16, block=block, seed=38, dtype=dtype, q_gain=1 / factor)
        p.k_scale *= factor
        p.k_seq = [k * factor for k in p.k_seq]
        check(p, p.attend())


def scale_values(p, b, first, last, factor):
    """The values of the blocks of sequence b that lie in [first, last) times `factor`."""
    for blk in range(first // p.block, -(-last // p.block)):
        page, in_page = int(p.table[b, blk * p.block // p.page]), blk % (p.page // p.block)
        p.v_scale[page, :, in_page] *= factor
        p.v_seq[b][blk * p.block:(blk + 1) * p.block] *= factor


def later_values(form, block, dtype):
    """The last token's values are 2^30 times the others': no token in front of it sees them."""
    lens, *heads = form
    p = PagedQ8(lens, *heads, 32, block=block, seed=34, dtype=dtype)
    for b, _, n, kv in rows_of(p):
        scale_values(p, b, kv - 1, kv, 2.0 ** 30)
    return p


def earlier_values(form, block, window, sinks, factor, dtype):
    """Values `factor` times the others' that the first new tokens see and that have left the window of the last ones."""
    lens, *heads = form
    p = PagedQ8(lens, *heads, 32, block=block, seed=35, window=window, sinks=sinks, dtype=dtype)
    for b, _, n, kv in rows_of(p):
        first = max(kv - n - window + 1, 0)     # of the first new token's window
        last = max(kv - window + 1, 0)          # of the last one's
        if last - first > block:
            scale_values(p, b, first, first + (last - first) // 2, factor)
        elif last > first and block == 1:
            scale_values(p, b, first, first + 1, factor)
    return p


blocks = pytest.mark.parametrize("block", [1, 16, 32])
windows = pytest.mark.parametrize("block,window,sinks", [(1, 64, 0), (1, 40, 3), (16, 100, 0), (32, 64, 5), (32, 200, 0)])
factors = pytest.mark.parametrize("factor", [2.0 ** 30, 2.0 ** 90])


@both
@row_forms
@blocks
def test_values_that_later_tokens_bring(block, form, dtype):
    p = later_values(form, block, dtype)
    check(p, p.attend())


@both
@row_forms
@windows
@factors
def test_values_in_front_of_later_tokens_windows(factor, block, window, sinks, form, dtype):
    p = earlier_values(form, block, window, sinks, factor, dtype)
    check(p, p.attend())


chunk_forms = pytest.mark.parametrize("form", FORMS[9:] + [([(200, 1000), (70, 99)], 8, 1, 128), ([(300, 700), (129, 129), (1, 40)], 4, 4, 64)], ids=str)


@both
@chunk_forms
@blocks
def test_values_that_later_tokens_of_a_chunk_bring(block, form, dtype):
    p = later_values(form, block, dtype)
    check(p, p.attend(), around=32 if block < 32 else 1)


@both
@chunk_forms
@windows
@factors
def test_values_in_front_of_the_windows_of_a_chunks_last_tokens(factor, block, window, sinks, form, dtype):
    p = earlier_values(form, block, window, sinks, factor, dtype)
    check(p, p.attend(), around=32 if block < 32 else 1)


@both
@forms
@pytest.mark.parametrize("block", [8, 16])
def test_weights_on_the_smaller_scales_of_32_keys(block, form, dtype):
    """Every other block's values are 2^24 times smaller, and its keys get all of the weight: their scores are at least 32 and the others' at
    most -32, so that these, 2^24 times as large and e^-64 < 2^-92 times as heavy, add less than 2^-68 of the result.  What fp16 loses is then
    that of a few keys of weight one, not of every key."""
    lens, *heads = form
    p = PagedQ8(lens, *heads, 32, block=block, seed=36, dtype=dtype)
    g = torch.Generator(device="cuda").manual_seed(37)
    d, hk = heads[2], heads[1]
    for b, _, n, kv in rows_of(p):
        small = (torch.arange(kv, device="cuda") // block % 2 == 0)[:, None, None]    # (every query sees the first block)
        keys = torch.where(small, 1.0, -1.0) * (torch.rand(kv, hk, d, generator=g, device="cuda") * 0.5 + 0.75)
        values = torch.where(small, 2.0 ** -24, 1.0) * torch.randn(kv, hk, d, generator=g, device="cuda")
        for x, seq, cache, scales in ((keys, p.k_seq, p.k_cache, p.k_scale), (values, p.v_seq, p.v_cache, p.v_scale)):
            y, scale, seq[b] = quantised(x, block, dtype)
            for i in range(-(-kv // p.page)):
                lo, hi, pg = i * p.page, min(kv, (i + 1) * p.page), int(p.table[b, i])
                cache[pg, :hi - lo] = y[lo:hi]
                blocks = scale[lo // block:-(-hi // block)]
                scales[pg, :, :len(blocks)] = blocks.T
    # scores at most -32 and at least 32: |q k| = sum of d products of at least 0.75 x, divided by sqrt(d)
    p.q = (torch.rand(p.q.shape, generator=g, device="cuda") * 0.5 + 1.0).bfloat16() * (32 / (0.7 * d ** 0.5))
    check(p, p.attend(), each_key=False)
