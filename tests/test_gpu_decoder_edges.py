"""Edges of the decoder operators, through the binding: empty batches, very long rows, padded batches, layouts and page sizes
beyond the ordinary ones."""
import ctypes

import pytest
import torch

import decoder_reference as ref

pytestmark = pytest.mark.gpu
BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32


def test_empty_batches():
    from paper_2511_03586_b200 import api
    e = lambda *s, t=BF16: torch.empty(*s, dtype=t, device="cuda")  # noqa: E731
    x = e(0, 64)
    h, n = api.pd_norm_gate_residual_norm(x, x, gate=e(0, 64), post_gamma=torch.ones(64, device="cuda"))
    assert h.shape == n.shape == (0, 64)
    api.pd_norm_gate_residual_norm(x, x, h=x, n=x)
    tokens, probs = api.pd_sample(e(0, 100, t=F32), e(0, t=F32), top_k=e(0, t=I32))
    assert tokens.shape == probs.shape == (0,)
    cache = torch.full((4, 16, 2, 64), 7.0, dtype=BF16, device="cuda")
    for batch in (0, 2):                                  # no sequences; sequences without new tokens
        table, lens = torch.zeros(batch, 3, dtype=I32, device="cuda"), torch.full((batch,), 5, dtype=I32, device="cuda")
        cu = torch.zeros(batch + 1, dtype=I32, device="cuda")
        api.pd_kv_cache_append(e(0, 2, 64), e(0, 2, 64), cache, cache, table, cu, lens)
        out = api.pd_attention_paged_fwd(e(0, 4, 64), cache, cache, table, cu, lens, max_q_len=0, max_kv_len=48)
        assert out.shape == (0, 4, 64)
    assert bool((cache == 7.0).all())


def test_norms_of_the_longest_row():
    """2^31 - 1 columns: the last step of a thread that walks them lies beyond 32 bits."""
    from paper_2511_03586_b200 import api
    cols = 2 ** 31 - 1
    ramp = (torch.arange(1 << 20, device="cuda") % 241 - 120).to(BF16)
    x = ramp.repeat(2048)[:cols].view(1, cols)
    y = torch.full((1, cols), 0.5, dtype=BF16, device="cuda")
    h = torch.zeros_like(x)
    d = api.NormGateResidualDesc(1, cols, 1, api.PD_BF16, api.PD_BF16, 0, 0, 1.0, 1e-5)
    stream = torch.cuda.current_stream().cuda_stream
    assert api._lib.pd_norm_gate_residual_norm(ctypes.byref(d), y.data_ptr(), x.data_ptr(), *(None,) * 5, h.data_ptr(), None, stream) == 0
    h.sub_(0.5)                                            # (exact: |x| <= 120, halves)
    step = 1 << 28
    assert all(torch.equal(h[:, i:i + step], x[:, i:i + step]) for i in range(0, cols, step))


@pytest.mark.parametrize("norms", [("rms", "rms"), ("layer", "rms")], ids=str)
@pytest.mark.parametrize("cols", [(1 << 18) + 8, (1 << 22) + 1])
def test_norms_of_long_rows(cols, norms):
    """Sums of millions of terms, of one size and sign (where roundings do not cancel) or two: 1e-5 of the value, or of the
    row's RMS where that is larger, as for rows of any length."""
    from paper_2511_03586_b200 import api
    y = torch.full((2, cols), 1.1, device="cuda")
    if norms[0] == "layer":
        y[:, ::2] = -0.3
    x = torch.full((2, cols), 0.7, device="cuda")
    got = api.pd_norm_gate_residual_norm(y, x, post_norm=norms[0], pre_norm=norms[1])
    want = ref.norm_gate_residual_norm(y, x, None, 1, 1.0, 1e-5, norms[0], None, None, norms[1], None, None)
    for g, w in zip(got, want):
        bound = 1e-5 * torch.maximum(w.abs(), w.pow(2).mean(-1, keepdim=True).sqrt())
        assert ((g.double() - w).abs() <= bound).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens", [[(130, 3000)], [(40, 2500), (0, 10), (33, 33), (1, 1900), (0, 0)]], ids=["one", "some"])
@pytest.mark.parametrize("pad", [0, 2, 3000])
def test_padded_batches_with_split_keys(lens, pad, d):
    """Few rows over many keys, which the chunk kernels share out, in token tensors of a fixed size."""
    from test_gpu_paged_attention import Paged
    p = Paged(lens, 8, 2, d, 16, seed=pad + d, pad=pad)
    out = torch.full_like(p.q, 3.0)
    for _ in range(2):
        p.attend(out=out)
        p.check(out)
        assert bool((out[sum(n for n, _ in lens):] == 3.0).all())
    cut = max(n for n, _ in lens) - 5                      # new tokens beyond max_q_len are not computed
    short = torch.full_like(p.q, 3.0)
    p.attend(out=short, max_q_len=cut)
    start = 0
    for b, (n, kv) in enumerate(lens):
        m = min(n, cut)
        want, mag = ref.attention(p.q[start:start + m], p.k_seq[b], p.v_seq[b], kv - n)
        bound = (2 ** -8 + 2 ** -10) * mag + 2 ** -8 * want.abs() + 1e-30   # as in test_gpu_paged_attention
        assert ((short[start:start + m].double() - want).abs() <= bound).all()
        assert bool((short[start + m:start + n] == 3.0).all())
        start += n


@pytest.mark.parametrize("page", [512, 1024, 4096])
@pytest.mark.parametrize("layout", ["slots", "heads"])
@pytest.mark.parametrize("d", [64, 128])
def test_attention_over_large_pages(page, layout, d):
    from test_gpu_paged_attention import Paged
    lens = [(1, 3), (1, page - 1), (1, page), (1, page + 1), (3, 2 * page + 130)]
    for window, sinks in ((0, 0), (70, 5)):
        p = Paged(lens, 8, 2, d, page, layout=layout, seed=page, window=window, sinks=sinks)
        p.check(p.attend())
        p = Paged([(100, page + 40), (30, 30)], 8, 2, d, page, layout=layout, seed=page + 1, window=window, sinks=sinks)
        p.check(p.attend())


@pytest.mark.parametrize("page", [1, 16, 48, 512, 4096])
@pytest.mark.parametrize("heads,d", [(2, 64), (8, 128), (1, 128), (3, 8)], ids=str)
def test_append_to_caches_whose_heads_lie_outside_their_slots(heads, d, page):
    """[pages, heads, slots, d], a block of a larger cache: page, slot and head strides that are not those of dense rows."""
    from paper_2511_03586_b200 import api
    lens = [(5, 5), (1, page), (7, 2 * page + 3), (0, 4)]
    need = [-(-kv // page) for _, kv in lens]
    whole = torch.full((2, sum(need) + 2, heads + 1, page, d), 7.0, dtype=BF16, device="cuda")
    k_cache, v_cache = whole[0, :, 1:].transpose(1, 2), whole[1, :, 1:].transpose(1, 2)
    tokens = sum(n for n, _ in lens)
    packed = torch.randn(tokens + 2, (4 + 2 * heads) * d, device="cuda").bfloat16()
    k = packed[:, 4 * d:(4 + heads) * d].unflatten(1, (heads, d))
    v = packed[:, (4 + heads) * d:].unflatten(1, (heads, d))
    table = torch.full((len(lens), max(need)), -1, dtype=I32)
    pages = torch.randperm(sum(need) + 2, generator=torch.Generator().manual_seed(page)).tolist()
    cu, want, at = [0], whole.clone(), 0
    for b, (n, kv) in enumerate(lens):
        table[b, :need[b]] = torch.tensor(pages[at:at + need[b]], dtype=I32)
        at += need[b]
        for i in range(n):
            pos = kv - n + i
            if pos < 0:
                continue                                   # a new token in front of the sequence is dropped
            want[0, table[b, pos // page], 1:, pos % page] = k[cu[-1] + i]
            want[1, table[b, pos // page], 1:, pos % page] = v[cu[-1] + i]
        cu.append(cu[-1] + n)
    api.pd_kv_cache_append(k, v, k_cache, v_cache, table.cuda(), torch.tensor(cu, dtype=I32, device="cuda"),
                           torch.tensor([kv for _, kv in lens], dtype=I32, device="cuda"))
    assert torch.equal(whole, want)


@pytest.mark.parametrize("cols", [1, 64, 65, 1000, 1001, 4096, 4097, 32768, 40001])
@pytest.mark.parametrize("post", ["none", "rms", "layer"])
@pytest.mark.parametrize("gate", [None, 0.7])
def test_layernorm_of_rows_of_one_value(cols, post, gate):
    """h does not vary within a row, whatever its rounding, so that LayerNorm leaves beta: a mean that is off by 5e-6 of the value
    is put right by the mean of the deviations, to 3e-11 of it, of which 1 / sqrt(eps) makes 1e-8.  1e-5, as for other rows."""
    from paper_2511_03586_b200 import api
    g = torch.Generator(device="cuda").manual_seed(cols)
    y, x = ((torch.randn(50, 1, generator=g, device="cuda") * 3).expand(50, cols).contiguous() for _ in range(2))
    beta = torch.randn(cols, generator=g, device="cuda").abs() + 0.5
    gates = None if gate is None else torch.full((1, cols), gate, device="cuda")
    _, n = api.pd_norm_gate_residual_norm(y, x, gate=gates, alpha=1.3, post_norm=post, pre_norm="layer", pre_beta=beta)
    assert ((n - beta).abs() <= 1e-5 * beta).all()
