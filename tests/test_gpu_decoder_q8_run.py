"""The operators around an 8-bit paged cache together, as a program that generates text runs them: a two-layer decoder with rotated
queries and keys over an int8 or e4m3 cache with scales for blocks of tokens, its logits penalised, biased and masked before a token
is drawn; prompts in chunks, then tokens one by one, also from a captured graph and on two streams at once.

Each step is compared with the 64-bit forms of the next operator on what the library's own operators have handed to it, so that no
error of an operator before hides one behind it: the cache with what the append must have left (tests of the append), the context with
attention over the values that the cache stands for, the logits with the history.  Tolerances are those of the operators' own tests;
for the context, whose keys and values are read back from the cache, 2^-8 of its value and 2^-8 of the weighted magnitudes hold both
kernels' parts (2^-10 for exponentials and values in fp16, 2^-10 for the fp32 parts), with room for scores below 32 in size whose keys
were rounded to fp16 (six times 2^-11 / sqrt(3) of them at most 2^-7 of the weighted magnitudes, added)."""
import math

import pytest
import torch

import decoder_q8_reference as ref8
import decoder_reference as ref

pytestmark = pytest.mark.gpu

HIDDEN, HEADS, KV, D, VOCAB, LAYERS, PAGE, BLOCK = 512, 8, 2, 64, 1000, 2, 16, 8
WINDOW, SINKS = (0, 48), (0, 4)
EPS = 1e-5


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


class Decoder:
    def __init__(self, batch, max_len, dtype, seed=0):
        from paper_2511_03586_b200 import api
        self.api = api
        g = torch.Generator(device="cuda").manual_seed(seed)
        mat = lambda i, o: (torch.randn(i, o, generator=g, device="cuda") / i ** 0.5).bfloat16()  # noqa: E731
        vec = lambda: torch.rand(HIDDEN, generator=g, device="cuda") + 0.5  # noqa: E731
        self.embed = torch.randn(VOCAB, HIDDEN, generator=g, device="cuda").bfloat16()
        self.head = mat(HIDDEN, VOCAB)
        self.layers = [dict(qkv=mat(HIDDEN, (HEADS + 2 * KV) * D), o=mat(HEADS * D, HIDDEN), pre=vec(), post=vec()) for _ in range(LAYERS)]
        self.last = vec()
        width = -(-max_len // PAGE)
        pages = batch * width + 2
        self.table = torch.randperm(pages, generator=g, device="cuda")[:batch * width].reshape(batch, -1).to(torch.int32)
        self.inv_freq = (10000.0 ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)).float().cuda()
        byte = lambda: torch.full((pages, PAGE, KV, D), 0x7F, dtype=torch.uint8, device="cuda").view(dtype)  # noqa: E731
        nan = lambda: torch.full((pages, KV, PAGE // BLOCK), math.nan, device="cuda")  # noqa: E731
        self.cache = [(byte(), byte(), nan(), nan()) for _ in range(LAYERS)]
        self.max_len = max_len
        self.seen = []

    def stands_for(self, layer, b, n):
        """Keys and values [n, KV, D] of sequence b, as the cache has them."""
        kc, vc, ks, vs = self.cache[layer]
        pos = torch.arange(n, device="cuda")
        page, slot = self.table[b].long()[pos // PAGE], pos % PAGE
        scaled = lambda c, s: c[page, slot].double() * s[page, :, slot // BLOCK].double()[..., None]  # noqa: E731
        return scaled(kc, ks), scaled(vc, vs)

    def forward(self, tokens, cu, lens, max_q, keep=False):
        api = self.api
        x = self.embed[tokens.long()]
        zero = torch.zeros_like(x)
        x, n = api.pd_norm_gate_residual_norm(zero, x, eps=EPS, post_norm="none", pre_gamma=self.layers[0]["pre"])
        for i, w in enumerate(self.layers):
            qkv = api.pd_gemm_bf16(n, w["qkv"])
            q, k, v = (t.unflatten(1, (-1, D)) for t in qkv.split([HEADS * D, KV * D, KV * D], 1))
            kc, vc, ks, vs = self.cache[i]
            turned = api.pd_rope_kv_cache_append(k, v, kc, vc, self.table, cu, lens, q=q, inv_freq=self.inv_freq, k_scale=ks, v_scale=vs)
            ctx = api.pd_attention_paged_q8_fwd(turned, kc, vc, ks, vs, self.table, cu, lens, max_q_len=max_q, max_kv_len=self.max_len,
                                                window=WINDOW[i], sinks=SINKS[i])
            if keep:
                self.seen.append((i, q, k, v, turned, ctx))
            y = api.pd_gemm_bf16(ctx.flatten(1), w["o"])
            x, n = api.pd_norm_gate_residual_norm(y, x, eps=EPS, post_gamma=w["post"],
                                                  pre_gamma=self.layers[i + 1]["pre"] if i + 1 < LAYERS else self.last)
        return api.pd_gemm_bf16(n, self.head, c_dtype=torch.float32)

    def check(self, take, lens):
        """What the last forward of `take` new tokens left behind, and what it read."""
        for i, q, k, v, turned, ctx in self.seen:
            at = 0
            for b, (n, kv) in enumerate(zip(take, lens)):
                if n == 0:
                    continue
                rows, pos = slice(at, at + n), torch.arange(kv - n, kv, device="cuda")
                at += n
                exact, mag = ref8.rotate(q[rows], pos, self.inv_freq, False)
                assert bool(((turned[rows].double() - exact).abs() <= 2 ** -8 * exact.abs() + 2 ** -21 * mag).all())
                keys, values = self.stands_for(i, b, kv)
                for got, (want, m), scales in ((keys, ref8.rotate(k[rows], pos, self.inv_freq, False), self.cache[i][2]),
                                               (values, (v[rows].double(), v[rows].double().abs()), self.cache[i][3])):
                    step = scales[self.table[b].long()[pos // PAGE], :, pos % PAGE // BLOCK].double()[..., None]
                    half = ref8.half_step(want / step, self.cache[i][0].dtype) * step
                    assert bool(((got[pos] - want).abs() <= half * (1 + 1e-6) + 2 ** -20 * m).all())
                out, mag = ref.attention(turned[rows], keys, values, kv - n, window=WINDOW[i], sinks=SINKS[i])
                assert bool(((ctx[rows].double() - out).abs() <= 2 ** -8 * out.abs() + (2 ** -8 + 2 ** -7) * mag + 1e-9).all())
        self.seen = []


dtypes = pytest.mark.parametrize("dtype", [torch.int8, torch.float8_e4m3fn], ids=["int8", "e4m3"])


@dtypes
def test_prompts_in_chunks_then_tokens(dtype):
    lens = [150, 1, 77, 33]
    m = Decoder(len(lens), 200, dtype)
    g = torch.Generator(device="cuda").manual_seed(1)
    seqs = [torch.randint(VOCAB, (n,), generator=g, device="cuda") for n in lens]
    history = torch.full((len(lens), 200), -1, dtype=torch.int32, device="cuda")
    for i, s in enumerate(seqs):
        history[i, :len(s)] = s.int()
    prompt = ints(lens)
    done, last = [0] * len(lens), [None] * len(lens)
    while any(d < n for d, n in zip(done, lens)):
        take = [min(64, n - d) for d, n in zip(done, lens)]
        packed = torch.cat([s[d:d + t] for s, d, t in zip(seqs, done, take)] + [torch.zeros(3, dtype=torch.long, device="cuda")])
        done = [d + t for d, t in zip(done, take)]
        out = m.forward(packed, ints([sum(take[:i]) for i in range(len(take) + 1)]), ints(done), max(take), keep=True)
        m.check(take, done)
        for i, t in enumerate(take):
            if t:
                last[i] = out[sum(take[:i + 1]) - 1]
    logits = torch.stack(last)
    mask = torch.randint(-2 ** 31, 2 ** 31, (2, (VOCAB + 31) // 32), generator=g, device="cuda").to(torch.int32)
    mask_row = ints([0, -1, 1, -1])
    settings = dict(repetition=torch.full((4,), 1.3, device="cuda"), frequency=torch.full((4,), 0.2, device="cuda"),
                    presence=torch.full((4,), 0.1, device="cuda"))
    one = ints(list(range(len(lens) + 1)))
    for _ in range(3):
        z = m.api.pd_penalize_logits(logits, history=history, history_len=ints(lens), prompt_len=prompt, mask=mask, mask_row=mask_row, **settings)
        u = torch.rand(len(lens), generator=g, device="cuda")
        tokens, _ = m.api.pd_sample(z, u)
        for i, n in enumerate(lens):
            allowed = None
            if mask_row[i] >= 0:
                t = torch.arange(VOCAB)
                allowed = ((mask[mask_row[i]].cpu()[t // 32] >> (t % 32)) & 1).bool()
            want = ref8.penalise_row(logits[i].cpu(), history[i, :n].tolist(), int(prompt[i]), 1.3, 0.2, 0.1, [], allowed)
            got = z[i].cpu().double()
            assert bool(((got == want) | ((got - want).abs() <= 2 ** -20 * (want.abs() + 1))).all())
            assert tokens[i].item() == ref.sample_row(z[i].cpu(), u[i].item())[0]
            assert allowed is None or bool(allowed[tokens[i].item()])
            history[i, n] = tokens[i]
        lens = [n + 1 for n in lens]
        logits = m.forward(tokens, one, ints(lens), 1, keep=True)
        m.check([1] * len(lens), lens)
    assert m.api.pd_get_device_status() == 0


@dtypes
def test_captured_decode_steps(dtype):
    """A step captured once and replayed with other lengths and tokens gives what the same calls give one by one."""
    lens = [20, 90]
    runs = []
    for captured in (False, True):
        m = Decoder(2, 128, dtype, seed=3)
        g = torch.Generator(device="cuda").manual_seed(2)
        packed = torch.randint(VOCAB, (110,), generator=g, device="cuda")
        m.forward(packed, ints([0, 20, 110]), ints(lens), 90)
        tokens, length, one = ints([5, 7]), ints(lens), ints([0, 1, 2])
        history, u = torch.zeros(2, 128, dtype=torch.int32, device="cuda"), torch.rand(2, generator=g, device="cuda")
        ones = torch.full((2,), 0.4, device="cuda")

        def step():
            length.add_(1)
            history.scatter_(1, (length - 1).long()[:, None], tokens[:, None])
            logits = m.forward(tokens, one, length, 1)
            z = m.api.pd_penalize_logits(logits, history=history, history_len=length, frequency=ones, out=logits)
            drawn, _ = m.api.pd_sample(z, u)
            tokens.copy_(drawn)
            return z

        if captured:
            state = [t.clone() for c in m.cache for t in c] + [tokens.clone(), length.clone(), history.clone()]
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                step()
            torch.cuda.current_stream().wait_stream(side)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                z = step()
            for t, was in zip([t for c in m.cache for t in c] + [tokens, length, history], state):
                t.copy_(was)
        out = []
        for _ in range(20):
            if captured:
                graph.replay()
                out.append((z.clone(), tokens.clone()))
            else:
                out.append((step().clone(), tokens.clone()))
        runs.append(out)
        assert m.api.pd_get_device_status() == 0
    for (za, ta), (zb, tb) in zip(*runs):
        assert torch.equal(za, zb) and torch.equal(ta, tb)


def test_two_streams_at_once():
    """Two models' steps on two streams, interleaved, again and again: the same results every time."""
    models = [Decoder(3, 300, torch.int8, seed=5), Decoder(2, 100, torch.float8_e4m3fn, seed=6)]
    g = torch.Generator(device="cuda").manual_seed(4)
    runs = []
    for m, lens in zip(models, ([290, 4, 100], [60, 99])):
        cu = ints([sum(lens[:i]) for i in range(len(lens) + 1)])
        runs.append((m, torch.randint(VOCAB, (sum(lens),), generator=g, device="cuda"), cu, ints(lens), max(lens), torch.cuda.Stream()))
    torch.cuda.synchronize()
    outs = [[], []]
    for _ in range(5):
        for i, (m, tokens, cu, lens, n, stream) in enumerate(runs):
            with torch.cuda.stream(stream):
                outs[i].append(m.forward(tokens, cu, lens, n))
    torch.cuda.synchronize()
    for o in outs:
        assert torch.isfinite(o[0]).all()
        for other in o[1:]:
            assert torch.equal(other, o[0])


def test_explicit_stream_takes_no_memory_that_the_current_one_still_writes():
    from paper_2511_03586_b200 import api
    g = torch.Generator(device="cuda").manual_seed(9)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    q, k = rand(2, 8, 64), rand(2, 2, 64)
    cache = [torch.zeros(40, 16, 2, 64, dtype=torch.int8, device="cuda") for _ in range(2)]
    scale = [torch.ones(40, 2, 1, device="cuda") for _ in range(2)]
    table, cu, lens = torch.arange(40, dtype=torch.int32, device="cuda").view(2, 20), ints([0, 1, 2]), ints([300, 40])
    logits, history = rand(8, 4000), torch.randint(4000, (8, 50), dtype=torch.int32, device="cuda")
    half = torch.full((8,), 0.5, device="cuda")
    calls = (lambda s: api.pd_rope_kv_cache_append(k, k, *cache, table, cu, lens, q=q, k_scale=scale[0], v_scale=scale[1], stream=s),
             lambda s: api.pd_attention_paged_q8_fwd(q, *cache, *scale, table, cu, lens, max_q_len=1, max_kv_len=320, stream=s),
             lambda s: api.pd_penalize_logits(logits, history=history, frequency=half, stream=s))
    side = torch.cuda.Stream()
    for call in calls:
        want = call(None).clone()
        torch.cuda.synchronize()
        torch.cuda._sleep(100_000_000)                 # the fills below happen after the call on the other stream
        held = [torch.empty_like(want) for _ in range(4)]
        for t in held:
            t.fill_(1)
        del held, t
        got = call(side)
        side.synchronize()
        torch.cuda.synchronize()
        assert torch.equal(got, want)
