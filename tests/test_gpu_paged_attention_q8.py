"""Attention over an 8-bit paged cache, against the definition in 64 bits.

Tolerance, element by element.  Exponentials times the scales of values are rounded to fp16 for the second product (half a step:
2^-11 relative) while their sum stays fp32: 2^-11 sum_j p_j |v_j|; the result is rounded to bf16 once, 2^-8 of itself; the fp32
parts are held by 2^-10 sum_j p_j |v_j| as in the test of the bf16 cache.  Stored values are exact in fp16, but where keys of several
scales share a group they are multiplied by their scales and rounded to fp16: another 2^-11 sum_j p_j |v_j| for the values, and
for a score 2^-11 sum_i |q_i k_i| scale at the very worst; D independent roundings do not conspire, and their sum is less than six
times its root mean square 2^-11 / sqrt(3) sqrt(sum_i (q_i k_i)^2) scale.  The weights move by that much, relative, and the result by
at most sum_j p_j e_j |v_j - out| <= e_max (sum_j p_j |v_j| + |out|).

Below its smallest normal number fp16 is off by half of its smallest one, 2^-25.  Exponentials with scales are in units of at most
4 F / 2^7 (F: the largest scale of a value in view; the kernel for few rows: 2 F / 2^11), the sum that they are divided by is at
least 1, and a stored value times F is at most the largest value of the head, V, since the largest value of a block takes up the
type's range: 2^-25 2^-7 4 V = 2^-30 V for every key.  Values that were multiplied by their scales are in units of F at most: 2^-25 F,
less than 2^-30 V once more."""
import pytest
import torch

import decoder_reference as ref

pytestmark = pytest.mark.gpu

I8, E4 = torch.int8, torch.float8_e4m3fn
TOP = {I8: 127.0, E4: 448.0}


def quantised(x, block, dtype):
    """x [n, heads, d] -> stored values, scales [ceil(n / block), heads], and what they stand for (fp64)."""
    n, heads, d = x.shape
    padded = torch.zeros(-(-n // block) * block, heads, d, device=x.device)
    padded[:n] = x
    padded = padded.unflatten(0, (-1, block))
    scale = padded.abs().amax((1, 3)) / TOP[dtype]
    y = padded / scale.clamp(min=1e-30)[:, None, :, None]
    y = (y.round() if dtype == I8 else y).clamp(-TOP[dtype], TOP[dtype]).to(dtype).flatten(0, 1)[:n]
    return y, scale, y.double() * scale.double().repeat_interleave(block, 0)[:n, :, None]


class PagedQ8:
    """8-bit caches whose unused slots and scales hold NaN (or what comes next to it), pages dealt out in random order."""

    def __init__(self, lens, heads, heads_kv, d, page, *, dtype=I8, block=None, seed=0, layout="slots", window=0, sinks=0, pad=0, q_gain=1.0,
                 spread=0.0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.lens, self.window, self.sinks, self.page, self.dtype = lens, window, sinks, page, dtype
        self.block = block = block or page
        need = [-(-max(kv, 0) // page) for _, kv in lens]
        num, width = sum(need) + 2, max(max(need), 1)
        order = torch.randperm(num, generator=g, device="cuda").tolist()
        shape = (num, page, heads_kv, d) if layout == "slots" else (num, heads_kv, page, d)
        poison = 0x7F if dtype == E4 else 0x80     # e4m3: NaN
        empty = lambda: torch.full(shape, poison, dtype=torch.uint8, device="cuda").view(dtype)  # noqa: E731
        self.k_cache, self.v_cache = empty(), empty()
        if layout == "heads":
            self.k_cache, self.v_cache = self.k_cache.transpose(1, 2), self.v_cache.transpose(1, 2)
        nan = lambda: torch.full((num, heads_kv, page // block), float("nan"), device="cuda")  # noqa: E731
        self.k_scale, self.v_scale = nan(), nan()
        table, at = torch.full((len(lens), width), -1, dtype=torch.int32), 0
        self.k_seq, self.v_seq = [], []
        for b, (n, kv) in enumerate(lens):
            first = kv - n
            for seq, cache, scales in ((self.k_seq, self.k_cache, self.k_scale), (self.v_seq, self.v_cache, self.v_scale)):
                x = torch.randn(kv, heads_kv, d, generator=g, device="cuda")
                if spread:   # blocks of very different magnitudes
                    x *= torch.exp(spread * torch.randn(-(-kv // block), 1, 1, generator=g, device="cuda")).repeat_interleave(block, 0)[:kv]
                y, scale, exact = quantised(x, block, dtype)
                seq.append(exact)
                for i in range(need[b]):
                    lo, hi = i * page, min(kv, (i + 1) * page)
                    if window and not (hi > first - window + 1 or lo < sinks):
                        table[b, i] = -1 if i % 2 else num + 7
                        continue
                    pg = table[b, i] = order[at + i]
                    cache[pg, :hi - lo] = y[lo:hi]
                    blocks = scale[lo // block:-(-hi // block)]
                    scales[pg, :, :len(blocks)] = blocks.T
                    if window:
                        for j in range(lo, hi):
                            if j <= first - window and j >= sinks:
                                cache.view(torch.uint8)[pg, j - lo] = poison
                            if j % block == 0 and j + block - 1 <= first - window and j >= sinks:
                                scales[pg, :, (j - lo) // block] = float("inf")
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
        return api.pd_attention_paged_q8_fwd(self.q, self.k_cache, self.v_cache, self.k_scale, self.v_scale, self.table, self.cu, self.kv, **args)

    def check(self, out, scale=None, alike=False):
        """alike: all elements of a key are the same, and so are their roundings; their errors add up."""
        from paper_2511_03586_b200 import api
        assert api.pd_get_device_status() == 0
        start = 0
        for b, (n, kv) in enumerate(self.lens):
            if n == 0:
                continue
            q = self.q[start:start + n]
            want, mag = ref.attention(q, self.k_seq[b], self.v_seq[b], kv - n, window=self.window, sinks=self.sinks, scale=scale)
            got = out[start:start + n].double()
            group = q.shape[1] // self.k_seq[b].shape[1]
            # the largest root of sum_i (q_i k_i)^2 of a head's keys, bounded through the keys' elementwise maxima
            most = self.k_seq[b].abs().amax(0).repeat_interleave(group, 0) if kv else torch.zeros_like(q[0]).double()
            e = 6 * 2 ** -11 / 3 ** 0.5 * (q.double() * most).pow(2).sum(-1, keepdim=True).sqrt() * (scale or q.shape[2] ** -0.5)
            if alike:
                e = 2 ** -11 * (q.double().abs() * most).sum(-1, keepdim=True) * (scale or q.shape[2] ** -0.5)
            v_most = self.v_seq[b].abs().amax((0, 2)).repeat_interleave(group)[:, None] if kv else 0.0
            bound = (2 * 2 ** -11 + 2 ** -10) * mag + 2 ** -8 * want.abs() + e * (mag + want.abs()) + 2 ** -30 * (kv + 1) * v_most + 1e-30
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
both = pytest.mark.parametrize("dtype", [I8, E4], ids=["int8", "e4m3"])


@both
@pytest.mark.parametrize("heads", HEADS, ids=str)
@pytest.mark.parametrize("lens", LENS, ids=str)
def test_attention(lens, heads, dtype):
    p = PagedQ8(LENS[lens], *heads, 16, seed=len(lens), dtype=dtype)
    p.check(p.attend())


@both
@pytest.mark.parametrize("page,block", [(8, 8), (8, 1), (16, 4), (32, 32), (64, 16), (128, 2), (128, 128), (256, 128), (1024, 1024)])
@pytest.mark.parametrize("layout", ["slots", "heads"])
@pytest.mark.parametrize("d", [64, 128])
def test_pages_blocks_and_layouts(page, block, layout, d, dtype):
    p = PagedQ8([(1, 77), (1, 500), (1, 1), (3, 260)], 8, 2, d, page, block=block, layout=layout, seed=page, dtype=dtype)
    p.check(p.attend())
    p = PagedQ8([(70, 77), (190, 500), (1, 1)], 8, 2, d, page, block=block, layout=layout, seed=page, dtype=dtype)
    p.check(p.attend())


@both
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 4), (64, 0), (65, 64), (100, 37), (128, 130), (1000, 4), (300, 1000)])
@pytest.mark.parametrize("lens", ["single", "few", "chunk", "long chunk", "one long"])
@pytest.mark.parametrize("d", [64, 128])
def test_window_and_sinks(lens, window, sinks, d, dtype):
    p = PagedQ8(LENS[lens], 8, 2, d, 16, block=8, seed=window, window=window, sinks=sinks, dtype=dtype)
    p.check(p.attend())


@both
@pytest.mark.parametrize("gain", [0.0, 4.0])
@pytest.mark.parametrize("lens", ["single", "chunk"])
@pytest.mark.parametrize("d", [64, 128])
def test_flat_and_peaked_scores(lens, gain, d, dtype):
    p = PagedQ8(LENS[lens], 8, 2, d, 16, seed=3, q_gain=gain, dtype=dtype)
    p.check(p.attend())


@both
@pytest.mark.parametrize("lens", ["single", "few", "chunk", "one long"])
@pytest.mark.parametrize("d", [64, 128])
def test_blocks_of_different_magnitudes(lens, d, dtype):
    """Scales that differ by factors of e^8 and more from block to block; keys of all magnitudes, so scores of 0 and of hundreds."""
    p = PagedQ8(LENS[lens], 8, 2, d, 16, block=4, seed=11, spread=2.0, q_gain=0.05, dtype=dtype)
    p.check(p.attend())


@both
@pytest.mark.parametrize("q_len", [1, 40])
@pytest.mark.parametrize("factor", [1e-30, 1e25])
def test_scales_far_from_one(q_len, factor, dtype):
    p = PagedQ8([(q_len, 300), (q_len, 77)], 8, 2, 128, 16, seed=12, dtype=dtype)
    p.v_scale *= factor
    p.v_seq = [v * float(torch.tensor(factor)) for v in p.v_seq]
    p.check(p.attend())


@both
def test_blocks_of_zeros(dtype):
    """Scales of zero: keys that score nothing, values that add nothing."""
    for lens in ([(1, 300), (2, 40)], [(60, 300), (33, 40)]):
        p = PagedQ8(lens, 8, 2, 128, 16, seed=13, dtype=dtype)
        for b, (_, kv) in enumerate(lens):
            for i in range(0, -(-kv // 16), 2):
                pg = int(p.table[b, i])
                p.k_scale[pg], p.v_scale[pg] = 0, 0
                p.k_seq[b][16 * i:16 * i + 16] = 0
                p.v_seq[b][16 * i:16 * i + 16] = 0
        p.check(p.attend())
        p.v_scale.nan_to_num_(0).zero_()
        p.v_seq = [v * 0 for v in p.v_seq]
        assert not p.attend().any()


@both
@pytest.mark.parametrize("lens", [[(1, 700), (1, 700)], [(60, 700)]], ids=["rows", "chunk"])
def test_growing_scores(lens, dtype):
    """Scores that grow along the keys by hundreds: the reference of every row has to move again and again."""
    p = PagedQ8(lens, 4, 2, 64, 16, seed=5, dtype=dtype)
    for b, (_, kv) in enumerate(lens):
        ramp = (torch.arange(kv, device="cuda")[:, None, None] * 0.03 - 10).expand(kv, 2, 64)
        y, scale, exact = quantised(ramp, 16, dtype)
        p.k_seq[b] = exact
        for i in range(-(-kv // 16)):
            pg, m = int(p.table[b, i]), min(kv, 16 * i + 16) - 16 * i
            p.k_cache[pg, :m] = y[16 * i:16 * i + m]
            p.k_scale[pg, :, 0] = scale[i]
    p.q = (torch.rand_like(p.q.float()) * 4).bfloat16()
    # A key's 64 elements are one integer y times one scale, so fp16 rounds all of them by the same d, |d| <= 2^-11 of them, and with
    # q >= 0 the score moves by d sum_i q_i k_i: nothing cancels, and six times the root of the squares' sum, sqrt(12) 2^-11
    # sqrt(sum_i (q_i k_i)^2) = sqrt(12) 2^-11 sqrt(4/3) sum_i q_i k_i / 8 = 0.5 2^-11 sum_i q_i k_i for q uniform in [0, 4], is half of what it can be.
    # (Keys rounded that way, everything else in 64 bits: 0.98 of that bound in the median of 200 draws of q, 1.05 at most.)
    p.check(p.attend(), alike=True)


@both
@pytest.mark.parametrize("lens", [[(1, 300), (1, 5)], [(40, 300), (33, 50)]], ids=["rows", "chunk"])
def test_padding_and_short_lengths(lens, dtype):
    p = PagedQ8(lens, 8, 2, 64, 16, pad=5, dtype=dtype)
    out = torch.full_like(p.q, 3.0)
    p.attend(out=out)
    p.check(out)
    assert bool((out[sum(n for n, _ in lens):] == 3.0).all())
    # kv_len short of the new tokens: those in front of position 0 see nothing
    p.kv[1] = lens[1][0] - 1
    first = lens[0][0]
    assert not p.attend(out=out)[first].any()


@both
def test_lengths_beyond_the_hints(dtype):
    """max_kv_len shapes the launch only."""
    p = PagedQ8([(1, 900), (1, 30)], 8, 2, 128, 16, dtype=dtype)
    p.check(p.attend(max_kv_len=1))
    p.check(p.attend(max_kv_len=1 << 20))


@both
def test_pages_outside_the_cache(dtype):
    """A table entry outside the cache counts as keys and values of zero."""
    for lens in ([(1, 100)], [(50, 100)]):
        p = PagedQ8(lens, 8, 2, 128, 16, dtype=dtype)
        p.table[0, 2], p.table[0, 4] = -1, 1 << 30
        for i in (2, 4):
            p.k_seq[0][16 * i:16 * i + 16] = 0
            p.v_seq[0][16 * i:16 * i + 16] = 0
        p.check(p.attend())
