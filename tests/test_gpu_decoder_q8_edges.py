"""Edges of the operators around an 8-bit cache, through the binding: every form of the kernel for few rows, empty batches, cut-off and
padded ones, caches beyond 32-bit offsets, shared pages, odd strides.  Bounds are those of the operators' own tests."""
import pytest
import torch

import decoder_q8_reference as ref8
from test_gpu_paged_attention_q8 import E4, I8, PagedQ8, both
from test_gpu_rope_append import Append

pytestmark = pytest.mark.gpu
I32, F32 = torch.int32, torch.float32


def test_empty_batches():
    from paper_2511_03586_b200 import api
    e = lambda *s, t=torch.bfloat16: torch.empty(*s, dtype=t, device="cuda")  # noqa: E731
    freq = torch.ones(32, device="cuda")
    for dtype in (I8, E4):
        cache = torch.full((4, 16, 2, 64), 7.0, device="cuda").to(dtype)
        scale = torch.full((4, 2, 2), 0.5, device="cuda")
        for batch in (0, 2):                                  # no sequences; sequences without new tokens
            table, lens = torch.zeros(batch, 3, dtype=I32, device="cuda"), torch.full((batch,), 5, dtype=I32, device="cuda")
            cu = torch.zeros(batch + 1, dtype=I32, device="cuda")
            got = api.pd_rope_kv_cache_append(e(0, 2, 64), e(0, 2, 64), cache, cache, table, cu, lens, q=e(0, 4, 64), inv_freq=freq,
                                              k_scale=scale, v_scale=scale)
            assert got.shape == (0, 4, 64)
            out = api.pd_attention_paged_q8_fwd(e(0, 4, 64), cache, cache, scale, scale, table, cu, lens, max_q_len=0, max_kv_len=48)
            assert out.shape == (0, 4, 64)
        assert bool((cache.float() == 7.0).all()) and bool((scale == 0.5).all())
    assert api.pd_penalize_logits(e(0, 100, t=F32), history=e(0, 3, t=I32), repetition=e(0, t=F32)).shape == (0, 100)
    assert torch.equal(api.pd_penalize_logits(torch.ones(2, 5, device="cuda"), history=e(2, 0, t=I32)), torch.ones(2, 5, device="cuda"))


@both
@pytest.mark.parametrize("page,block", [(8, 1), (16, 16), (128, 32), (4096, 64)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("group,tokens", [(4, 1), (4, 3), (8, 3), (8, 4), (11, 4), (16, 4)])      # 4, 12, 24, 32, 44, 64 rows
@pytest.mark.parametrize("heads_kv", [1, 2, 3, 4])
def test_forms_for_few_rows(heads_kv, group, tokens, d, page, block, dtype):
    """Cache heads side by side, warps that share keys, or rows; tiles of 32, 64 and 128 keys over pages smaller and larger."""
    lens = [(tokens, 77), (tokens, 500), (tokens, tokens), (1, 260)]
    p = PagedQ8(lens, group * heads_kv, heads_kv, d, page, block=block, seed=page + group, dtype=dtype)
    p.check(p.attend())


@both
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens", [[(3, 300), (0, 10), (5, 5), (1, 190)], [(130, 3000)], [(40, 2500), (0, 10), (33, 33), (1, 1900), (0, 0)]], ids=["few", "one", "some"])
@pytest.mark.parametrize("pad", [0, 2, 3000])
def test_padded_and_cut_off_batches(lens, pad, d, dtype):
    p = PagedQ8(lens, 8, 2, d, 16, seed=pad + d, pad=pad, dtype=dtype)
    out = torch.full_like(p.q, 3.0)
    for _ in range(2):
        p.attend(out=out)
        p.check(out)
        assert bool((out[sum(n for n, _ in lens):] == 3.0).all())
    cut = max(n for n, _ in lens) - 2                      # new tokens beyond max_q_len are not computed
    short = torch.full_like(p.q, 3.0)
    p.attend(out=short, max_q_len=cut)
    at, kept = 0, short.clone()
    for n, _ in lens:
        assert bool((short[at + min(n, cut):at + n] == 3.0).all())
        kept[at + min(n, cut):at + n] = out[at + min(n, cut):at + n]
        at += n
    p.check(kept)


@both
@pytest.mark.parametrize("lens", [[(1, 300), (1, 45)], [(60, 300), (33, 45)]], ids=["rows", "chunk"])
def test_pages_that_sequences_share(lens, dtype):
    p = PagedQ8(lens, 8, 2, 128, 16, seed=8, dtype=dtype)
    p.table[1] = p.table[0]
    p.k_seq[1], p.v_seq[1] = p.k_seq[0][:45], p.v_seq[0][:45]
    p.check(p.attend())


@both
def test_caches_beyond_32_bit_offsets(dtype):
    """Pages behind the first 2^32 bytes, and elements, of each cache."""
    lens, heads_kv, d, page = [(1, 300), (1, 45)], 8, 128, 64
    pages = (1 << 32) // (page * heads_kv * d) + 64
    for seed, lens in enumerate([[(1, 300), (1, 45)], [(60, 300), (33, 45)]]):
        p = PagedQ8(lens, 2 * heads_kv, heads_kv, d, page, block=32, seed=seed, dtype=dtype)
        last = pages - len(p.k_cache)
        for name in ("k_cache", "v_cache", "k_scale", "v_scale"):
            small = getattr(p, name)
            large = torch.empty((pages, *small.shape[1:]), dtype=small.dtype, device="cuda")
            large[last:] = small
            setattr(p, name, large)
        p.table += last
        p.check(p.attend())
        del p, large
    a = Append(lens, 2 * heads_kv, heads_kv, d, page, block=32, dtype=dtype)
    b = Append(lens, 2 * heads_kv, heads_kv, d, page, block=32, dtype=dtype)
    small = len(a.k_cache)
    for name in ("k_cache", "v_cache", "k_scale", "v_scale"):
        large = torch.empty((pages, *getattr(a, name).shape[1:]), dtype=getattr(a, name).dtype, device="cuda")
        large[-small:] = getattr(a, name)
        setattr(a, name, large)
    a.table = torch.where(a.table >= 0, a.table + pages - small, a.table)
    from paper_2511_03586_b200 import api
    args, named = a.args()
    api.pd_rope_kv_cache_append(*args, q=a.q, **named)
    b.run()
    for name in ("k_cache", "v_cache", "k_scale", "v_scale"):
        assert torch.equal(getattr(a, name)[-small:].view(torch.uint8), getattr(b, name).view(torch.uint8)), name


@pytest.mark.parametrize("dtype", [torch.bfloat16, I8, E4], ids=["bf16", "int8", "e4m3"])
@pytest.mark.parametrize("heads_kv", [1, 3, 9])
def test_append_for_many_sequences_with_long_blocks(heads_kv, dtype):
    Append([(1 + i % 3, 3 + 41 * i % 500) for i in range(150)], 2 * heads_kv, heads_kv, 128, 64, dtype=dtype, block=64, pad=1).run()
    Append([(200, 333)] + [(0, 3)] * 130 + [(70, 70)], heads_kv, heads_kv, 96, 128, dtype=dtype, block=128, rotary=32).run()


def test_one_call_after_the_other_on_another_stream():
    """The operators of a step on a stream of its own, in order, through one workspace that both attention calls use."""
    from paper_2511_03586_b200 import api
    for dtype in (I8, E4):
        a = PagedQ8([(1, 900), (1, 333)], 8, 2, 128, 16, seed=21, dtype=dtype)
        b = PagedQ8([(3, 500), (2, 70)], 8, 2, 128, 16, seed=22, dtype=dtype)
        ws = torch.full((64 << 20,), 255, dtype=torch.uint8, device="cuda")
        want = a.attend(), b.attend()
        torch.cuda.synchronize()
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            got = a.attend(workspace=ws), b.attend(workspace=ws), a.attend(workspace=ws)
        stream.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.equal(got[2], want[0])
    assert api.pd_get_device_status() == 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("vocab", [100, 4099, 33000])
@pytest.mark.parametrize("offset", [0, 1, 4])
def test_penalties_in_place_in_a_wider_tensor(vocab, offset, dtype):
    from paper_2511_03586_b200 import api
    g = torch.Generator(device="cuda").manual_seed(vocab)
    wide = (torch.randn(5, vocab + 12, generator=g, device="cuda") * 3).to(dtype)
    before = wide.clone()
    z = wide[:, offset:offset + vocab]
    history = torch.randint(-2, vocab + 2, (5, 300), generator=g, device="cuda", dtype=I32)
    r, f, s = (torch.full((5,), v, device="cuda") for v in (1.3, 0.25, 0.5))
    assert api.pd_penalize_logits(z, history=history, repetition=r, frequency=f, presence=s, out=z) is z
    for i in range(5):
        want = ref8.penalise_row(before[i, offset:offset + vocab].cpu(), history[i].tolist(), 0, float(r[i]), 0.25, 0.5, [], None)
        # a reciprocal and a product, one fused multiplication and a difference in fp32, of values below 32 + 300; then one rounding
        bound = 5 * 2 ** -24 * (want.abs() + 300 * 0.25 + 0.5) + (2 ** -8 * want.abs() if dtype == torch.bfloat16 else 0)
        assert bool(((z[i].cpu().double() - want).abs() <= bound).all())
    assert torch.equal(wide[:, :offset], before[:, :offset]) and torch.equal(wide[:, offset + vocab:], before[:, offset + vocab:])


@both
@pytest.mark.parametrize("heads,group,tokens,d", [(4, 4, 1, 128), (4, 8, 1, 64), (1, 8, 1, 128), (2, 5, 1, 128), (1, 16, 4, 64), (8, 4, 5, 128), (3, 8, 3, 128)])
def test_one_long_context(heads, group, tokens, d, dtype):
    """An item's keys over most of the CTAs, so that its join has hundreds of pieces; alone, and beside short ones."""
    for lens in ([(tokens, 20000)], [(1, 40), (tokens, 16400), (tokens, tokens)]):
        p = PagedQ8(lens, heads * group, heads, d, 16, seed=heads + d, dtype=dtype)
        p.check(p.attend())
