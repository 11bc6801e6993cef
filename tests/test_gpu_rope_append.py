"""Rotation by positions with the append to a bf16 or 8-bit paged cache, against the definition in 64 bits.

Tolerances.  An angle's turns are exact to 2^-52 of themselves; what is left of them (at most half a turn) is rounded to fp32,
off by 2^-26 turns = 9.4e-8 radians, and sincospif is off by less than 2 units in the last place, 2^-23: cos and sin are off by
less than 2^-22 together.  The amplitude, two products and their sum add at most four roundings of 2^-24: a rotated element is
off by less than 2^-21 of the sum of its terms' magnitudes, |a| + |b| (ROT).  bf16 results are rounded once (2^-8 of their value).
8-bit values: x / scale is formed with a reciprocal and a product (2 roundings), the scale with a division: 2^-21 of x / scale
holds them twice over.  So a stored value is within half a step plus 2^-21 of x / scale plus ROT / scale of the exact quotient."""
import pytest
import torch

import decoder_q8_reference as ref

pytestmark = pytest.mark.gpu

ROT = 2.0 ** -21
I8, E4 = torch.int8, torch.float8_e4m3fn


class Append:
    """Caches of random contents and a random page table; `lens`: (new tokens, cached tokens with them) of each sequence."""

    def __init__(self, lens, heads, heads_kv, d, page, *, dtype=torch.bfloat16, block=None, rotary=None, interleaved=False, amplitude=1.0,
                 seed=0, layout="slots", pad=0, gain=1.0, holes=False, theta=10000.0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.lens, self.page, self.block, self.dtype, self.d = lens, page, block or page, dtype, d
        self.heads, self.heads_kv, self.interleaved, self.amplitude = heads, heads_kv, interleaved, amplitude
        rotary = d if rotary is None else rotary
        self.inv_freq = (theta ** (-torch.arange(0, rotary, 2, dtype=torch.float64) / rotary)).float().cuda() if rotary else None
        # pages only where new tokens go
        first = [max(kv - n, 0) // page for n, kv in lens]
        need = [-(-kv // page) for _, kv in lens]
        num = sum(n - f for n, f in zip(need, first)) + 3
        order = torch.randperm(num, generator=g, device="cuda").tolist()
        table, at = torch.full((len(lens), max(max(need), 1)), -1, dtype=torch.int32), 0
        for b, (f, n) in enumerate(zip(first, need)):
            for i in range(f, n):
                table[b, i] = order[at]
                at += 1
                if holes and i % 3 == 1:
                    table[b, i] = (-1, num, num + 5)[b % 3]
        self.table = table.cuda()
        shape = (num, page, heads_kv, d) if layout == "slots" else (num, heads_kv, page, d)
        def cache():
            if dtype == torch.bfloat16:
                c = torch.randn(shape, generator=g, device="cuda").bfloat16()
            elif dtype == I8:
                c = torch.randint(-127, 128, shape, generator=g, device="cuda", dtype=torch.int32).to(I8)
            else:
                c = (torch.randn(shape, generator=g, device="cuda") * 100).clamp(-448, 448).to(E4)
            return c if layout == "slots" else c.transpose(1, 2)
        self.k_cache, self.v_cache = cache(), cache()
        self.k_scale = self.v_scale = None
        if dtype != torch.bfloat16:
            scale = lambda: (torch.rand(num, heads_kv, page // self.block, generator=g, device="cuda") + 0.3) * 3 / ref.TOP[dtype]  # noqa: E731
            self.k_scale, self.v_scale = scale(), scale()
        counts = [n for n, _ in lens]
        self.cu = torch.tensor([sum(counts[:i]) for i in range(len(lens) + 1)], dtype=torch.int32, device="cuda")
        self.kv = torch.tensor([kv for _, kv in lens], dtype=torch.int32, device="cuda")
        tokens = sum(counts) + pad
        packed = (torch.randn(tokens, (heads + 2 * heads_kv) * d, generator=g, device="cuda") * gain).bfloat16()
        self.q = packed[:, :heads * d].unflatten(1, (heads, d))
        self.k = packed[:, heads * d:(heads + heads_kv) * d].unflatten(1, (heads_kv, d))
        self.v = packed[:, (heads + heads_kv) * d:].unflatten(1, (heads_kv, d))

    def args(self):
        return (self.k, self.v, self.k_cache, self.v_cache, self.table, self.cu, self.kv), dict(
            inv_freq=self.inv_freq, interleaved=self.interleaved, amplitude=self.amplitude, k_scale=self.k_scale, v_scale=self.v_scale)

    def run(self, **kw):
        """Calls, and checks everything that the call may have written."""
        from paper_2511_03586_b200 import api
        before = [None if t is None else t.clone() for t in (self.k_cache, self.v_cache, self.k_scale, self.v_scale)]
        q = self.q.clone()
        args, named = self.args()
        q_out = kw.pop("q_out", torch.full((self.q.shape), 7.0, device="cuda").bfloat16())
        untouched = q_out.clone()
        got = api.pd_rope_kv_cache_append(*args, q=self.q, q_out=q_out, **{**named, **kw})
        assert got is q_out
        self.check(before, q, q_out, untouched)
        return q_out

    def check(self, before, q, q_out, untouched):
        at = 0
        want = [t if t is None else t.clone().double() for t in before[:2]]
        slack = [torch.zeros_like(w) for w in want]
        scales = [None if t is None else t.clone().double() for t in before[2:]]
        for b, (n, kv) in enumerate(self.lens):
            pos = torch.arange(kv - n, kv, device="cuda")
            rows = torch.arange(at, at + n, device="cuda")[pos >= 0]
            pos = pos[pos >= 0]
            at += n
            if len(pos) == 0:
                continue
            exact, mag = ref.rotate(q[rows], pos, self.inv_freq, self.interleaved, self.amplitude)
            err = (q_out[rows].double() - exact).abs()
            assert bool((err <= 2 ** -8 * exact.abs() + ROT * mag + 1e-38).all())
            untouched[rows] = q_out[rows]
            k, k_mag = ref.rotate(self.k[rows], pos, self.inv_freq, self.interleaved, self.amplitude)
            v, v_mag = self.v[rows].double(), self.v[rows].double().abs()
            for c, (x, m) in enumerate(((k, k_mag), (v, v_mag))):
                for blk in range(int(pos[0]) // self.block, int(pos[-1]) // self.block + 1):
                    lo, hi = max(int(pos[0]), blk * self.block), min(int(pos[-1]) + 1, (blk + 1) * self.block)
                    pg = int(self.table[b, lo // self.page])
                    if not 0 <= pg < self.k_cache.shape[0]:
                        continue
                    mine = slice(lo - int(pos[0]), hi - int(pos[0]))
                    slots = slice(lo % self.page, lo % self.page + hi - lo)
                    if self.dtype == torch.bfloat16:
                        want[c][pg, slots] = x[mine]
                        slack[c][pg, slots] = 2 ** -8 * x[mine].abs() + (ROT * m[mine] if c == 0 else 0)
                        continue
                    older = slice(blk * self.block % self.page, lo % self.page)
                    in_page = blk % (self.page // self.block)
                    old_scale = scales[c][pg, :, in_page].clone()
                    scale, kept = ref.append_block(x[mine], before[c][pg, older].double(), old_scale, self.dtype)
                    grew = (scale > old_scale)[:, None]
                    scales[c][pg, :, in_page] = scale
                    want[c][pg, older] = kept
                    slack[c][pg, older] = torch.where(grew, ref.half_step(kept, self.dtype) + 2 ** -19 * kept.abs(), 0.0)
                    quotient = x[mine] / scale.clamp(min=1e-300)[:, None]
                    want[c][pg, slots] = quotient
                    slack[c][pg, slots] = ref.half_step(quotient, self.dtype) * (1 + 1e-6) + 2 ** -20 * quotient.abs() + ROT * m[mine] / scale.clamp(min=1e-300)[:, None]
        assert torch.equal(q_out, untouched), "rows of padding or without a position were written"
        for c, (got, name) in enumerate(((self.k_cache, "k"), (self.v_cache, "v"))):
            off = (got.double() - want[c]).abs()
            assert bool((off <= slack[c]).all()), (name, (off - slack[c]).max().item())
            if self.dtype != torch.bfloat16:
                got_scale = (self.k_scale, self.v_scale)[c].double()
                assert bool(((got_scale - scales[c]).abs() <= 2 ** -19 * scales[c]).all()), name


LENS = {
    "single": [(1, 1), (1, 2), (1, 16), (1, 17), (1, 500), (1, 33)],
    "empty": [(1, 5), (0, 0), (0, 40), (2, 2), (1, 300), (0, 0)],
    "few": [(3, 3), (5, 70), (2, 64), (7, 200), (1, 513)],
    "chunk": [(100, 100), (33, 200), (129, 129), (1, 7), (128, 640)],
    "far": [(2, 1_000_001), (1, 99_999)],
    "short": [(5, 3), (4, 0), (3, 3)],      # tokens in front of position 0
}


@pytest.mark.parametrize("dtype", [torch.bfloat16, I8, E4], ids=["bf16", "int8", "e4m3"])
@pytest.mark.parametrize("lens", LENS, ids=str)
@pytest.mark.parametrize("heads", [(8, 2, 64), (4, 4, 128), (10, 1, 128), (20, 10, 64)], ids=str)
def test_append(lens, heads, dtype):
    Append(LENS[lens], *heads, 16, dtype=dtype, seed=len(lens), pad=3).run()


@pytest.mark.parametrize("dtype", [torch.bfloat16, I8, E4], ids=["bf16", "int8", "e4m3"])
@pytest.mark.parametrize("rotary,interleaved", [(0, False), (8, False), (24, False), (24, True), (64, True), (96, False), (96, True)])
def test_rotated_part(rotary, interleaved, dtype):
    Append([(3, 50), (1, 9), (40, 77)], 6, 3, 96, 16, dtype=dtype, rotary=rotary, interleaved=interleaved, amplitude=1.25).run()


@pytest.mark.parametrize("d", [8, 16, 40, 64, 128, 256])
@pytest.mark.parametrize("dtype", [torch.bfloat16, I8, E4], ids=["bf16", "int8", "e4m3"])
def test_head_dims(d, dtype):
    layout = "heads" if dtype == torch.bfloat16 or d % 16 == 0 else None
    if layout is None:   # strides of an 8-bit cache are multiples of 16
        from paper_2511_03586_b200.api import PdError
        with pytest.raises(PdError):
            Append([(1, 1)], 2, 1, d, 16, dtype=dtype).run()
        return
    Append([(3, 50), (1, 9), (70, 90)], 6, 2, d, 32, dtype=dtype, layout=layout).run()


@pytest.mark.parametrize("page,block", [(8, 1), (16, 2), (32, 8), (64, 64), (128, 16), (256, 256), (1024, 512), (48, 16), (96, 32)])
@pytest.mark.parametrize("layout", ["slots", "heads"])
@pytest.mark.parametrize("dtype", [I8, E4], ids=["int8", "e4m3"])
def test_blocks(page, block, layout, dtype):
    Append([(1, 77), (3, 300), (1, 1), (200, 700), (520, 530)], 4, 2, 128, page, block=block, layout=layout, dtype=dtype, seed=page).run()


@pytest.mark.parametrize("dtype", [torch.bfloat16, I8, E4], ids=["bf16", "int8", "e4m3"])
def test_pages_that_are_not_there(dtype):
    Append([(60, 100), (1, 20), (40, 41), (33, 90)], 4, 2, 64, 16, dtype=dtype, holes=True).run()


@pytest.mark.parametrize("dtype", [I8, E4], ids=["int8", "e4m3"])
@pytest.mark.parametrize("gain", [0.0, 1e-38, 1e-30, 0.01, 100.0, 1e30])
def test_magnitudes(gain, dtype):
    """Blocks whose scale stays, grows a lot, is zero, or falls below the normal range."""
    a = Append([(1, 9), (3, 50), (40, 77), (16, 32)], 4, 2, 64, 16, dtype=dtype, gain=gain)
    a.run()
    if gain == 0.0:
        a.k_scale.zero_(), a.v_scale.zero_()     # nothing but zeros so far
        a.run()


@pytest.mark.parametrize("dtype", [I8, E4], ids=["int8", "e4m3"])
def test_token_by_token(dtype):
    """A block filled one token after the other, each step against the state before it; then its values against the tokens."""
    n, d, hk = 40, 64, 2
    g = torch.Generator(device="cuda").manual_seed(5)
    all_k = torch.randn(n, hk, d, generator=g, device="cuda") * torch.linspace(0.2, 3.0, n, device="cuda")[:, None, None]
    a = Append([(1, 1)], 2, hk, d, 64, block=16, dtype=dtype, rotary=0)
    grown = torch.zeros(4, hk, device="cuda")
    for i in range(n):
        a.lens, a.kv[0] = [(1, i + 1)], i + 1
        a.k[0], a.v[0] = all_k[i].bfloat16(), all_k[i].flip(0).bfloat16()
        old = a.k_scale[a.table[0, 0].item()].clone()
        a.run()
        grown += (a.k_scale[a.table[0, 0].item()] > old).T if i % 16 else 0
    page = a.table[0, 0].item()
    for i in range(n):
        scale = a.k_scale[page, :, i // 16].double()[:, None]
        err = (a.k_cache[page, i].double() * scale - all_k[i].bfloat16().double()).abs()
        steps = (1 + grown[i // 16].double())[:, None]
        most = ref.TOP[dtype]
        # half a step for the first rounding and for every time that the scale grew behind it
        bound = steps * scale * 0.5 if dtype == I8 else steps * (2 ** -4 * all_k[i].bfloat16().double().abs() * 1.1 + scale * 2 ** -10)
        assert bool((err <= bound * (1 + 1e-5) + scale * most * 1e-6).all())


def test_keys_and_values_only_and_in_place():
    from paper_2511_03586_b200 import api
    a, b = (Append([(3, 50), (40, 77)], 4, 2, 64, 16, seed=4) for _ in range(2))
    args, named = a.args()
    assert api.pd_rope_kv_cache_append(*args, **named) is None
    want = b.run()
    assert torch.equal(a.k_cache, b.k_cache) and torch.equal(a.v_cache, b.v_cache)
    args, named = a.args()
    q = a.q
    assert api.pd_rope_kv_cache_append(*args, q=q, q_out=q, **named) is q
    assert torch.equal(q, want)


def test_unrotated_append_is_the_copying_one():
    from paper_2511_03586_b200 import api
    a = Append([(3, 50), (40, 77), (1, 4)], 4, 2, 64, 16, rotary=0, seed=6)
    k, v = a.k_cache.clone(), a.v_cache.clone()
    api.pd_kv_cache_append(a.k, a.v, k, v, a.table, a.cu, a.kv)
    a.run()
    assert torch.equal(a.k_cache, k) and torch.equal(a.v_cache, v)


def test_many_sequences_and_long_chunks():
    Append([(1, 1 + 37 * i % 900) for i in range(300)], 8, 2, 64, 16, dtype=I8, block=8).run()
    Append([(0, 3)] * 70 + [(1, 5)] + [(0, 0)] * 70 + [(30, 31)], 8, 2, 64, 16, dtype=E4).run()
    Append([(3000, 5000), (1, 8)], 8, 2, 128, 64, dtype=I8, block=32).run()
