"""The paged key/value cache and the attention over it, against the definition in 64 bits.

Tolerance of the attention, element by element.  The kernel rounds the exponentials to bf16 for the second product (half
a step: 2^-8 relative, each) while their sum stays fp32, so the numerator is off by at most 2^-8 sum_j p_j |v_j|; the
output is rounded to bf16 once (2^-8 of its own size).  The fp32 parts are far below: a score of D products is off by at
most D 2^-24 sum |q_i k_i| scale < 128 * 2^-24 * 32 = 2.4e-4 for the inputs here (scores up to 32 in absolute sum), which
moves numerator and denominator by that much, relative, at worst; 2^-10 covers both twice over."""
import pytest
import torch

import decoder_reference as ref

pytestmark = pytest.mark.gpu


class Paged:
    """Caches poisoned with NaN, pages dealt out in random order, and random new tokens for every sequence."""

    def __init__(self, lens, heads, heads_kv, d, page, *, seed=0, layout="slots", window=0, sinks=0, pad=0, spare=2, q_gain=1.0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.lens, self.window, self.sinks = lens, window, sinks
        self.page = page
        need = [-(-max(kv, 0) // page) for _, kv in lens]
        width = max(max(need), 1)
        num = sum(need) + spare
        order = torch.randperm(num, generator=g, device="cuda").tolist()
        shape = (num, page, heads_kv, d) if layout == "slots" else (num, heads_kv, page, d)
        self.k_cache = torch.full(shape, float("nan"), device="cuda").bfloat16()
        self.v_cache = torch.full(shape, float("nan"), device="cuda").bfloat16()
        if layout == "heads":
            self.k_cache, self.v_cache = self.k_cache.transpose(1, 2), self.v_cache.transpose(1, 2)
        table = torch.full((len(lens), width), -1, dtype=torch.int32)
        self.k_seq, self.v_seq = [], []
        at = 0
        for b, (n, kv) in enumerate(lens):
            k = torch.randn(kv, heads_kv, d, generator=g, device="cuda").bfloat16()
            v = torch.randn(kv, heads_kv, d, generator=g, device="cuda").bfloat16()
            self.k_seq.append(k), self.v_seq.append(v)
            first = kv - n
            for i in range(need[b]):
                lo, hi = i * page, min(kv, (i + 1) * page)
                in_view = not window or hi > first - window + 1 or lo < sinks
                if not in_view:
                    table[b, i] = -1 if i % 2 else num + 7   # evicted: the entry means nothing
                    continue
                pg = order[at + i]
                table[b, i] = pg
                self.k_cache[pg, :hi - lo] = k[lo:hi]
                self.v_cache[pg, :hi - lo] = v[lo:hi]
                if window:   # slots of a kept page in front of every window hold anything
                    for j in range(lo, hi):
                        if j <= first - window and j >= sinks:
                            self.k_cache[pg, j - lo] = float("nan")
                            self.v_cache[pg, j - lo] = float("nan")
            at += need[b]
        self.table = table.cuda()
        counts = [n for n, _ in lens]
        self.cu = torch.tensor([sum(counts[:i]) for i in range(len(lens) + 1)], dtype=torch.int32, device="cuda")
        self.kv = torch.tensor([kv for _, kv in lens], dtype=torch.int32, device="cuda")
        tokens = sum(counts) + pad
        packed = torch.randn(tokens, (heads + 2 * heads_kv) * d, generator=g, device="cuda") * q_gain
        self.q = packed.bfloat16()[:, :heads * d].unflatten(1, (heads, d))
        if pad:
            self.q[sum(counts):] = float("nan")
        self.max_q, self.max_kv = max(max(counts), 0), max(kv for _, kv in lens)

    def attend(self, **kw):
        from paper_2511_03586_b200 import api
        args = dict(max_q_len=self.max_q, max_kv_len=self.max_kv, window=self.window, sinks=self.sinks)
        args.update(kw)
        return api.pd_attention_paged_fwd(self.q, self.k_cache, self.v_cache, self.table, self.cu, self.kv, **args)

    def check(self, out, scale=None):
        start = 0
        for b, (n, kv) in enumerate(self.lens):
            if n == 0:
                continue
            want, mag = ref.attention(self.q[start:start + n], self.k_seq[b], self.v_seq[b], kv - n, window=self.window,
                                      sinks=self.sinks, scale=scale)
            got = out[start:start + n].double()
            bound = (2 ** -8 + 2 ** -10) * mag + 2 ** -8 * want.abs() + 1e-30
            worst = ((got - want).abs() / bound).max().item()
            assert worst <= 1.0, (b, n, kv, worst)
            start += n


LENS = {
    "single": [(1, 1), (1, 2), (1, 63), (1, 64), (1, 65), (1, 127), (1, 129), (1, 1000)],
    "empty": [(1, 5), (0, 0), (0, 40), (2, 2), (1, 300), (0, 0)],
    "few": [(3, 3), (5, 70), (2, 64), (7, 200), (1, 513)],
    "chunk": [(100, 100), (33, 200), (129, 129), (1, 7), (128, 640)],
    "long chunk": [(300, 300), (257, 700)],
    "one long": [(1, 5000)],
    "one short": [(1, 1)],
}
HEADS = [(8, 2, 64), (8, 2, 128), (4, 4, 64), (6, 2, 128), (10, 2, 64), (5, 1, 128), (16, 1, 128), (40, 1, 64), (64, 1, 128)]


@pytest.mark.parametrize("heads", HEADS, ids=str)
@pytest.mark.parametrize("lens", LENS, ids=str)
def test_attention(lens, heads):
    p = Paged(LENS[lens], *heads, page=16, seed=len(lens))
    p.check(p.attend())


@pytest.mark.parametrize("page", [8, 16, 32, 64, 128, 256])
@pytest.mark.parametrize("layout", ["slots", "heads"])
@pytest.mark.parametrize("d", [64, 128])
def test_page_sizes_and_layouts(page, layout, d):
    p = Paged([(1, 77), (1, 500), (1, 1), (3, 260)], 8, 2, d, page, layout=layout, seed=page)
    p.check(p.attend())
    p = Paged([(70, 77), (190, 500), (1, 1)], 8, 2, d, page, layout=layout, seed=page)
    p.check(p.attend())


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 4), (64, 0), (65, 64), (100, 37), (128, 130), (1000, 4), (300, 1000)])
@pytest.mark.parametrize("lens", ["single", "few", "chunk", "long chunk", "one long"])
@pytest.mark.parametrize("d", [64, 128])
def test_window_and_sinks(lens, window, sinks, d):
    p = Paged(LENS[lens], 8, 2, d, 16, seed=window, window=window, sinks=sinks)
    p.check(p.attend())


@pytest.mark.parametrize("gain", [0.0, 4.0])
@pytest.mark.parametrize("lens", ["single", "chunk"])
def test_flat_and_peaked_scores(lens, gain):
    p = Paged(LENS[lens], 8, 2, 64, 16, seed=3, q_gain=gain)
    # (gain 4 quadruples the fp32 part of the tolerance's derivation, which the factor of two and more in it covers)
    p.check(p.attend())


def test_growing_scores():
    """Scores that grow along the keys by hundreds: the reference of every row has to move again and again."""
    p = Paged([(1, 700), (60, 700)], 4, 2, 64, 16, seed=5)
    for k, kv in zip(p.k_seq, (700, 700)):
        k.copy_((torch.arange(kv, device="cuda")[:, None, None] * 0.03 - 10).expand_as(k))
    for b, k in enumerate(p.k_seq):
        for i in range(-(-700 // 16)):
            pg = int(p.table[b, i])
            m = min(700, 16 * i + 16) - 16 * i
            p.k_cache[pg, :m] = k[16 * i:16 * i + m]
    p.q.copy_(torch.ones_like(p.q))
    p.check(p.attend())


@pytest.mark.parametrize("lens", ["single", "chunk", "long chunk"])
def test_scale_and_hints(lens):
    p = Paged(LENS[lens], 8, 2, 64, 16, seed=9)
    want = p.attend(scale=0.05)
    p.check(want, scale=0.05)
    # max_kv_len only sizes the launch: far too small or too large gives the same rows
    for hint in (0, 1, 64, 100000):
        p.check(p.attend(scale=0.05, max_kv_len=hint), scale=0.05)


def test_positions_in_front_of_zero_see_nothing():
    from paper_2511_03586_b200 import api
    for n, kv in ((5, 3), (200, 130)):
        p = Paged([(n, n)], 8, 2, 64, 16, seed=1)
        p.kv.fill_(kv)                     # the cache is short: the first n - kv tokens have negative positions
        out = api.pd_attention_paged_fwd(p.q, p.k_cache, p.v_cache, p.table, p.cu, p.kv, max_q_len=n, max_kv_len=kv)
        assert (out[:n - kv] == 0).all()
        q = p.q
        p.q, p.lens = q[n - kv:], [(kv, kv)]
        p.check(out[n - kv:])


@pytest.mark.parametrize("lens", ["single", "chunk"])
def test_padding_rows_stay_and_out_strides(lens):
    p = Paged(LENS[lens], 8, 2, 64, 16, seed=2, pad=9)
    tokens = p.q.shape[0]
    wide = torch.full((tokens, 8 * 64 + 72), 3.0, device="cuda").bfloat16()
    out = wide[:, 8:8 + 512].unflatten(1, (8, 64))
    p.attend(out=out)
    p.check(out)
    assert (out[tokens - 9:] == 3.0).all() and (wide[:, :8] == 3.0).all() and (wide[:, 520:] == 3.0).all()


def test_max_q_len_cuts_off():
    for n, limit in ((40, 7), (300, 170)):
        p = Paged([(n, n + 30)], 8, 2, 64, 16, seed=2)
        out = torch.full(p.q.shape, 5.0, device="cuda").bfloat16()
        p.attend(out=out, max_q_len=limit)
        assert (out[limit:] == 5.0).all()
        want, mag = ref.attention(p.q, p.k_seq[0], p.v_seq[0], 30)
        bound = (2 ** -8 + 2 ** -10) * mag + 2 ** -8 * want.abs()
        assert ((out[:limit].double() - want[:limit]).abs() <= bound[:limit]).all()


def test_bad_table_entries_are_not_followed():
    """Entries outside the cache count as pages of zeros, wherever they are."""
    for lens in ([(1, 200)], [(150, 200)]):
        p = Paged(lens, 8, 2, 64, 16, seed=4)
        p.table[0, 3], p.table[0, 7] = 10 ** 9, -5
        for i in (3, 7):
            p.k_seq[0][16 * i:16 * i + 16] = 0
            p.v_seq[0][16 * i:16 * i + 16] = 0
        p.check(p.attend())
        p.kv.fill_(10 ** 6)                # longer than the table: keys end with the table
        p.attend()
        torch.cuda.synchronize()


def test_shared_prefix_and_repeatability():
    p = Paged([(1, 300), (1, 300), (40, 300)], 8, 2, 128, 32, seed=6)
    p.table[1, :8] = p.table[0, :8]
    p.k_seq[1][:256], p.v_seq[1][:256] = p.k_seq[0][:256], p.v_seq[0][:256]
    first = p.attend()
    p.check(first)
    for _ in range(3):
        assert torch.equal(p.attend(), first)


@pytest.mark.parametrize("lens", ["single", "long chunk"])
def test_other_stream_and_graph_replay(lens):
    p = Paged(LENS[lens], 8, 2, 128, 16, seed=7)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    out = torch.empty_like(p.q)
    p.attend(out=out, stream=s)
    s.synchronize()
    p.check(out)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        replayed = p.attend()
    replayed.zero_()
    g.replay()
    assert torch.equal(replayed, out)
    # the same graph with other lengths: shorter contexts, one sequence without a context at all
    shorter = [(n, max(n, kv // 2)) for n, kv in p.lens]
    p.kv.copy_(torch.tensor([kv for _, kv in shorter], dtype=torch.int32))
    p.lens = shorter
    p.k_seq = [k[:kv] for k, (_, kv) in zip(p.k_seq, shorter)]
    p.v_seq = [v[:kv] for v, (_, kv) in zip(p.v_seq, shorter)]
    g.replay()
    p.check(replayed)


def test_offsets_beyond_32_bits():
    """A cache of more than 2^32 elements; the pages in use are its last ones."""
    from paper_2511_03586_b200 import api
    pages, page, hk, d = 35000, 64, 16, 128       # 4.6e9 elements
    cache = torch.empty(pages, page, hk, d, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(0)
    for n, kv in ((1, 300), (130, 300)):
        k = torch.randn(kv, hk, d, generator=g, device="cuda").bfloat16()
        q = torch.randn(n, hk, d, generator=g, device="cuda").bfloat16()
        table = torch.arange(pages - 5, pages, dtype=torch.int32, device="cuda")[None].contiguous()
        cu = torch.tensor([0, kv], dtype=torch.int32, device="cuda")
        lens = torch.tensor([kv], dtype=torch.int32, device="cuda")
        api.pd_kv_cache_append(k, k, cache, cache, table, cu, lens)
        assert torch.equal(cache[pages - 5:].flatten(0, 1)[:kv], k)
        out = api.pd_attention_paged_fwd(q, cache, cache, table, torch.tensor([0, n], dtype=torch.int32, device="cuda"),
                                         lens, max_q_len=n, max_kv_len=kv)
        want, mag = ref.attention(q, k, k, kv - n)
        assert ((out.double() - want).abs() <= (2 ** -8 + 2 ** -10) * mag + 2 ** -8 * want.abs()).all()


@pytest.mark.parametrize("d,heads_kv", [(64, 2), (128, 8), (128, 1), (256, 7), (8, 3), (1024, 2)])
@pytest.mark.parametrize("page", [1, 16, 48])
def test_append(d, heads_kv, page):
    from paper_2511_03586_b200 import api
    g = torch.Generator(device="cuda").manual_seed(d + page)
    counts, kv = [1, 0, 5, 70, 1, 33], [1, 9, 105, 70, 300, 20]     # the last: 13 tokens in front of position 0
    batch, width = len(counts), -(-300 // page)
    pages = batch * width + 3
    table = torch.randperm(pages, generator=g, device="cuda")[:batch * width].reshape(batch, width).to(torch.int32)
    table[3, 0] = -1                                                # dropped
    table[2, -1] = pages                                            # (not reached)
    packed = torch.randn(sum(counts) + 4, 3 * heads_kv * d, generator=g, device="cuda").bfloat16()
    k, v = (packed[:, i * heads_kv * d:(i + 1) * heads_kv * d].unflatten(1, (heads_kv, d)) for i in (1, 2))
    k_cache = torch.randn(pages, page, heads_kv, d, generator=g, device="cuda").bfloat16()
    v_cache = torch.randn(pages, heads_kv, page, d, generator=g, device="cuda").bfloat16().transpose(1, 2).contiguous()
    want_k, want_v = k_cache.clone(), v_cache.clone()
    t = 0
    for b in range(batch):
        for i in range(counts[b]):
            pos = kv[b] - counts[b] + i
            pg = int(table[b, pos // page]) if pos >= 0 else -1
            if 0 <= pg < pages:
                want_k[pg, pos % page], want_v[pg, pos % page] = k[t], v[t]
            t += 1
    cu = torch.tensor([sum(counts[:i]) for i in range(batch + 1)], dtype=torch.int32, device="cuda")
    lens = torch.tensor(kv, dtype=torch.int32, device="cuda")
    api.pd_kv_cache_append(k, v, k_cache, v_cache, table, cu, lens)
    assert torch.equal(k_cache, want_k) and torch.equal(v_cache, want_v)


def test_append_finds_sequences_in_large_batches():
    from paper_2511_03586_b200 import api
    for batch in (31, 32, 33, 1023, 1025, 5000):
        g = torch.Generator().manual_seed(batch)
        counts = torch.randint(0, 4, (batch,), generator=g)
        cu = torch.cat([torch.zeros(1, dtype=torch.long), counts.cumsum(0)]).to(torch.int32).cuda()
        tokens = int(counts.sum())
        k = torch.randn(tokens, 1, 8).bfloat16().cuda()
        cache = torch.zeros(batch, 4, 1, 8, dtype=torch.bfloat16, device="cuda")
        other = torch.zeros_like(cache)
        table = torch.arange(batch, dtype=torch.int32, device="cuda")[:, None].contiguous()
        api.pd_kv_cache_append(k, k, cache, other, table, cu, counts.to(torch.int32).cuda())
        got = torch.cat([cache[b, :int(counts[b])] for b in range(batch)])
        assert torch.equal(got, k) and torch.equal(cache, other)


def test_binding_refusals():
    from paper_2511_03586_b200 import api
    p = Paged([(1, 20)], 8, 2, 64, 16)
    with pytest.raises(TypeError):
        api.pd_attention_paged_fwd(p.q.float(), p.k_cache, p.v_cache, p.table, p.cu, p.kv, max_q_len=1, max_kv_len=20)
    with pytest.raises(TypeError):
        api.pd_attention_paged_fwd(p.q, p.k_cache, p.v_cache, p.table.long(), p.cu, p.kv, max_q_len=1, max_kv_len=20)
    with pytest.raises(TypeError):
        api.pd_attention_paged_fwd(p.q, p.k_cache.cpu(), p.v_cache, p.table, p.cu, p.kv, max_q_len=1, max_kv_len=20)
    with pytest.raises(ValueError):
        api.pd_attention_paged_fwd(p.q, p.k_cache, p.v_cache, p.table, p.cu[:1], p.kv, max_q_len=1, max_kv_len=20)
    with pytest.raises(ValueError):
        api.pd_attention_paged_fwd(p.q.transpose(1, 2), p.k_cache, p.v_cache, p.table, p.cu, p.kv, max_q_len=1, max_kv_len=20)
    with pytest.raises(api.PdError):
        api.pd_attention_paged_fwd(p.q, p.k_cache, p.v_cache, p.table, p.cu, p.kv, max_q_len=1, max_kv_len=20, scale=-1.0)
    with pytest.raises(ValueError):
        api.pd_kv_cache_append(p.q, p.q, p.k_cache, p.v_cache, p.table, p.cu, p.kv)


def test_no_wait_ran_out():
    from paper_2511_03586_b200 import api
    assert api.pd_get_device_status() == 0


def test_stream_argument_keeps_memory():
    """Calls on a stream that is behind: the tensors made for them, and dropped at once, are not handed out meanwhile."""
    p = Paged([(1, 3000), (1, 2000)], 8, 2, 128, 16, seed=11)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)          # some ten milliseconds
    outs = [p.attend(stream=s) for _ in range(4)]
    scribble = [torch.full((1 << 20,), float("nan"), device="cuda") for _ in range(64)]
    s.synchronize()
    del scribble
    for o in outs:
        p.check(o)


@pytest.mark.parametrize("batch", [33, 200])
def test_large_batches(batch):
    """More sequences than a warp has lanes, and than a block has threads, with empty and absent ones among them."""
    lens = [(0 if i % 7 == 3 else 1, (i * 37) % 300 + 1) for i in range(batch)]
    lens = [(n, kv if n else 0) for n, kv in lens]
    p = Paged(lens, 4, 2, 64, 16, seed=batch)
    p.check(p.attend())
    p = Paged([(2 if n else 0, max(kv, 2) if n else 0) for n, kv in lens], 8, 1, 64, 16, seed=batch, window=40, sinks=3)
    p.check(p.attend())


def test_values_beyond_32_bits_are_refused():
    """The descriptor's fields would drop the upper half: a window of 2^32 + 5 keys must not become one of 5."""
    from paper_2511_03586_b200 import api
    case = dict(max_q_len=1, max_kv_len=64)
    q, cache = torch.zeros(1, 2, 64, device="cuda", dtype=torch.bfloat16), torch.zeros(4, 16, 2, 64, device="cuda", dtype=torch.bfloat16)
    table = torch.arange(4, dtype=torch.int32, device="cuda").view(1, 4)
    cu, lens = (torch.tensor(v, dtype=torch.int32, device="cuda") for v in ([0, 1], [64]))
    for name in ("max_q_len", "max_kv_len", "window", "sinks"):
        for v in (2 ** 31, 2 ** 32 + 5, -2 ** 31 - 1):
            with pytest.raises(ValueError):
                api.pd_attention_paged_fwd(q, cache, cache, table, cu, lens, **{**case, name: v})


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens", [[(60, 700), (300, 300)], [(40, 4000)]], ids=["whole", "split"])
def test_growing_scores_of_chunks(lens, d):
    """As test_growing_scores, for either kernel of chunks: rescaling while products are in flight, in pages of 8."""
    p = Paged(lens, 4, 2, d, 8, seed=5)
    for k, (_, kv) in zip(p.k_seq, lens):
        k.copy_((torch.arange(kv, device="cuda")[:, None, None] * (21.0 / kv) - 10).expand_as(k))
    for b, (k, (_, kv)) in enumerate(zip(p.k_seq, lens)):
        for i in range(-(-kv // 8)):
            m = min(kv, 8 * i + 8) - 8 * i
            p.k_cache[int(p.table[b, i]), :m] = k[8 * i:8 * i + m]
    p.q.copy_(torch.ones_like(p.q))
    p.check(p.attend())


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window,sinks", [(0, 0), (700, 5), (9000, 0)])
def test_chunks_over_long_caches(d, window, sinks):
    """Few rows of the chunk kernels over many keys: shares of the keys, joined; more sequences than fill the SMs, not shared."""
    p = Paged([(40, 20011), (17, 300), (0, 64), (33, 9000)], 8, 2, d, 32, seed=d, window=window, sinks=sinks)
    out = p.attend()
    p.check(out)
    assert torch.equal(p.attend(), out)
    p.check(p.attend(max_kv_len=1))            # not shared out: one walk per row tile
    many = Paged([(33, 100 + 13 * i) for i in range(40)], 8, 2, d, 16, seed=1, window=window, sinks=sinks)
    many.check(many.attend())


@pytest.mark.parametrize("lens", ["single", "chunk"])
@pytest.mark.parametrize("d", [64, 128])
def test_extreme_window_sinks_and_lengths(lens, d):
    """The largest window and sinks see everything; lengths in front of 0 leave nothing to see."""
    p = Paged(LENS[lens], 8, 2, d, 16, seed=13)
    for window, sinks in ((2 ** 31 - 1, 0), (1, 2 ** 31 - 1), (2 ** 31 - 1, 2 ** 31 - 1)):
        p.check(p.attend(window=window, sinks=sinks))
    for kv in (0, -1, -2 ** 31):
        p.kv.fill_(kv)
        out = p.attend()
        assert (out[:int(p.cu[-1])] == 0).all()
