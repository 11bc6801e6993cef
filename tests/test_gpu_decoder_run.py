"""The decoder operators together, as a program that generates text runs them: a two-layer decoder (norms before and
after each block, grouped heads, one windowed layer with sink tokens, SwiGLU) over a paged cache, built from the library's
entry points; prompts in chunks, then tokens one by one, also from a captured graph.

Tolerance: every tensor between operators is rounded to bf16, which is off by 2^-8 / sqrt(3) = 0.23 % of its value in the
mean square at worst (half a step, uniformly distributed); a logit has some 22 such roundings behind it (2 layers of qkv, probabilities, context,
projection, two sums and norms, gate and up product, down projection, and the last norm and product), which add up in the mean
square to 0.23 % sqrt(22) = 1.1 %.  2 % of the logits' RMS holds that with the amplification of the residual branches."""
import pytest
import torch

import decoder_reference as ref

pytestmark = pytest.mark.gpu

HIDDEN, HEADS, KV, D, FFN, VOCAB, LAYERS, PAGE = 512, 8, 2, 64, 1024, 1000, 2, 16
WINDOW, SINKS = (0, 48), (0, 4)
EPS = 1e-5


class Decoder:
    def __init__(self, batch, max_len, seed=0):
        from paper_2511_03586_b200 import api
        self.api = api
        g = torch.Generator(device="cuda").manual_seed(seed)
        mat = lambda i, o: (torch.randn(i, o, generator=g, device="cuda") / i ** 0.5).bfloat16()  # noqa: E731
        vec = lambda: torch.rand(HIDDEN, generator=g, device="cuda") + 0.5  # noqa: E731
        self.embed = torch.randn(VOCAB, HIDDEN, generator=g, device="cuda").bfloat16()
        self.head = mat(HIDDEN, VOCAB)
        self.layers = [dict(qkv=mat(HIDDEN, (HEADS + 2 * KV) * D), o=mat(HEADS * D, HIDDEN), gate=mat(HIDDEN, FFN),
                            up=mat(HIDDEN, FFN), down=mat(FFN, HIDDEN), pre1=vec(), post1=vec(), pre2=vec(), post2=vec())
                       for _ in range(LAYERS)]
        self.last = vec()
        pages = batch * -(-max_len // PAGE) + 2
        self.table = torch.randperm(pages, generator=g, device="cuda")[:batch * -(-max_len // PAGE)].reshape(batch, -1).to(torch.int32)
        nan = lambda: torch.full((pages, PAGE, KV, D), float("nan"), device="cuda").bfloat16()  # noqa: E731
        self.cache = [(nan(), nan()) for _ in range(LAYERS)]
        self.max_len = max_len
        zero = torch.zeros(1, HIDDEN, dtype=torch.bfloat16, device="cuda")
        self.zeros = lambda n: zero.expand(n, -1).contiguous()

    def forward(self, tokens, cu, lens, max_q):
        """Logits (fp32) of every token; the cache is extended by them."""
        api = self.api
        x = self.embed[tokens.long()]
        norms = lambda y, x, post, pre, kind="rms": api.pd_norm_gate_residual_norm(  # noqa: E731
            y, x, eps=EPS, post_norm=kind, post_gamma=post, pre_norm="rms", pre_gamma=pre)
        x, n = norms(self.zeros(x.shape[0]), x, None, self.layers[0]["pre1"], "none")
        for i, w in enumerate(self.layers):
            qkv = api.pd_gemm_bf16(n, w["qkv"])
            q, k, v = qkv.split([HEADS * D, KV * D, KV * D], 1)
            kc, vc = self.cache[i]
            api.pd_kv_cache_append(k.unflatten(1, (KV, D)), v.unflatten(1, (KV, D)), kc, vc, self.table, cu, lens)
            ctx = api.pd_attention_paged_fwd(q.unflatten(1, (HEADS, D)), kc, vc, self.table, cu, lens, max_q_len=max_q,
                                             max_kv_len=self.max_len, window=WINDOW[i], sinks=SINKS[i])
            x, n = norms(api.pd_gemm_bf16(ctx.flatten(1), w["o"]), x, w["post1"], w["pre2"])
            y = api.pd_gemm_bf16(api.pd_swiglu_gemm(n, w["gate"], w["up"]), w["down"])
            x, n = norms(y, x, w["post2"], self.layers[i + 1]["pre1"] if i + 1 < LAYERS else self.last)
        return api.pd_gemm_bf16(n, self.head, c_dtype=torch.float32)

    def reference(self, tokens):
        """Logits of one whole sequence in 64 bits."""
        x = self.embed[tokens.long()].double()
        rms = lambda v, g: ref.norm("rms", v, g, None, EPS)  # noqa: E731
        for i, w in enumerate(self.layers):
            n = rms(x, w["pre1"])
            q, k, v = (n @ w["qkv"].double()).split([HEADS * D, KV * D, KV * D], 1)
            ctx, _ = ref.attention(q.unflatten(1, (HEADS, D)), k.unflatten(1, (KV, D)), v.unflatten(1, (KV, D)), 0,
                                   window=WINDOW[i], sinks=SINKS[i])
            x = x + rms(ctx.flatten(1) @ w["o"].double(), w["post1"])
            n = rms(x, w["pre2"])
            gate = n @ w["gate"].double()
            x = x + rms((gate * torch.sigmoid(gate) * (n @ w["up"].double())) @ w["down"].double(), w["post2"])
        return rms(x, self.last) @ self.head.double()


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def check(logits, want):
    err = (logits.double() - want).pow(2).mean().sqrt() / want.pow(2).mean().sqrt()
    assert err < 2e-2, err.item()


def test_prompts_in_chunks_then_tokens():
    lens = [150, 1, 77, 33]
    m = Decoder(len(lens), 200)
    g = torch.Generator(device="cuda").manual_seed(1)
    seqs = [torch.randint(VOCAB, (n,), generator=g, device="cuda") for n in lens]
    want = [m.reference(s) for s in seqs]
    # chunks of up to 64 tokens, with rows of padding behind the last sequence
    done = [0] * len(lens)
    logits = [[] for _ in lens]
    while any(d < n for d, n in zip(done, lens)):
        take = [min(64, n - d) for d, n in zip(done, lens)]
        packed = torch.cat([s[d:d + t] for s, d, t in zip(seqs, done, take)] + [torch.zeros(3, dtype=torch.long, device="cuda")])
        cu = ints([sum(take[:i]) for i in range(len(take) + 1)])
        done = [d + t for d, t in zip(done, take)]
        out = m.forward(packed, cu, ints(done), max(take))
        at = 0
        for i, t in enumerate(take):
            logits[i].append(out[at:at + t])
            at += t
    for got, w in zip(logits, want):
        check(torch.cat(got), w)
    # tokens one by one: drawn, appended, compared with the whole sequence in 64 bits
    last = torch.stack([torch.cat(l)[-1] for l in logits])
    one = ints(list(range(len(lens) + 1)))
    for step in range(3):
        u = torch.rand(len(lens), generator=g, device="cuda")
        k, p = ints([40] * len(lens)), torch.full((len(lens),), 0.9, device="cuda")
        tokens, probs = m.api.pd_sample(last, u, top_k=k, top_p=p)
        for i in range(len(lens)):
            token, prob = ref.sample_row(last[i].cpu(), u[i].item(), 1.0, 40, p[i].item())
            assert tokens[i].item() == token and abs(probs[i].item() - prob) < 1e-6
            seqs[i] = torch.cat([seqs[i], tokens[i:i + 1].long()])
        lens = [n + 1 for n in lens]
        last = m.forward(tokens, one, ints(lens), 1)
        check(last, torch.stack([m.reference(s)[-1] for s in seqs]))
    assert m.api.pd_get_device_status() == 0


def test_captured_decode_steps():
    """A decode step captured once and replayed: token, lengths and random numbers live in the graph's buffers."""
    lens = [20, 90]
    m = Decoder(2, 128, seed=3)
    g = torch.Generator(device="cuda").manual_seed(2)
    seqs = [torch.randint(VOCAB, (n,), generator=g, device="cuda") for n in lens]
    m.forward(torch.cat(seqs), ints([0, 20, 110]), ints(lens), 90)
    tokens, length, one = ints([5, 7]), ints(lens), ints([0, 1, 2])
    u = torch.rand(4, 2, generator=g, device="cuda")
    u_now = u[0].clone()

    def step():
        length.add_(1)
        logits = m.forward(tokens, one, length, 1)
        drawn, probs = m.api.pd_sample(logits, u_now)
        return logits, drawn, probs

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):                  # warm-up as captures want it, then the state is put back
        step()
    torch.cuda.current_stream().wait_stream(side)
    length.copy_(ints(lens))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        logits, drawn, probs = step()
    for i in range(4):
        u_now.copy_(u[i])
        seqs = [torch.cat([s, tokens[j:j + 1].long()]) for j, s in enumerate(seqs)]
        graph.replay()
        check(logits, torch.stack([m.reference(s)[-1] for s in seqs]))
        for j in range(2):
            token, prob = ref.sample_row(logits[j].cpu(), u[i, j].item())
            assert drawn[j].item() == token and abs(probs[j].item() - prob) < 1e-6
        tokens.copy_(drawn)
    assert m.api.pd_get_device_status() == 0


def test_two_streams_at_once():
    """Two models' steps on two streams, interleaved: each call has a workspace of its own."""
    a, b = Decoder(3, 300, seed=5), Decoder(2, 100, seed=6)
    g = torch.Generator(device="cuda").manual_seed(4)
    runs = []
    for m, lens in ((a, [290, 4, 100]), (b, [60, 99])):
        seqs = [torch.randint(VOCAB, (n,), generator=g, device="cuda") for n in lens]
        cu = ints([sum(lens[:i]) for i in range(len(lens) + 1)])
        runs.append((m, torch.cat(seqs), cu, ints(lens), max(lens), torch.cat([m.reference(s) for s in seqs]), torch.cuda.Stream()))
    torch.cuda.synchronize()
    outs = [[], []]
    for _ in range(5):
        for i, (m, tokens, cu, lens, n, _, stream) in enumerate(runs):
            with torch.cuda.stream(stream):
                outs[i].append(m.forward(tokens, cu, lens, n))
    torch.cuda.synchronize()
    for i, run in enumerate(runs):
        check(outs[i][0], run[5])
        for o in outs[i][1:]:
            assert torch.equal(o, outs[i][0])


def test_explicit_stream_takes_no_memory_that_the_current_one_still_writes():
    """What is allocated for a call on another stream must not be what the current stream has freed but not finished with."""
    from paper_2511_03586_b200 import api
    g = torch.Generator(device="cuda").manual_seed(9)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    y, x, logits, u = rand(64, 512), rand(64, 512), rand(8, 4000), torch.rand(8, generator=g, device="cuda")
    q, cache = rand(2, 8, 64), rand(40, 16, 2, 64)
    table, cu, lens = torch.arange(40, dtype=torch.int32, device="cuda").view(2, 20), ints([0, 1, 2]), ints([300, 40])
    calls = (lambda s: api.pd_norm_gate_residual_norm(y, x, stream=s),
             lambda s: api.pd_sample(logits, u, stream=s),
             lambda s: (api.pd_attention_paged_fwd(q, cache, cache, table, cu, lens, max_q_len=1, max_kv_len=320, stream=s),))
    side = torch.cuda.Stream()
    for call in calls:
        want = [t.clone() for t in call(None)]
        torch.cuda.synchronize()
        torch.cuda._sleep(100_000_000)                 # the fills below happen after the call on the other stream
        held = [[torch.empty_like(t) for t in want] for _ in range(4)]
        for t in (t for ts in held for t in ts):
            t.fill_(1)
        del held, t
        got = call(side)
        side.synchronize()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)
