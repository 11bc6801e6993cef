"""Sampling from logits, token by token against the definition in 64 bits.

Tokens have to be equal.  The kernel sums weights in units of 2^-44 of the largest, so a running sum of n weights is off
by at most n 2^-45 relative to it: for the random inputs here a decision lies that close to its border with a
probability below 1e-6 (ties and exact fractions, where borders are hit exactly, are representable in both).
Probabilities: fp32, one rounding (2^-24) of a quotient whose parts are exact to n 2^-45 / total: 2^-22 covers it for
weights that are not tiny, and 2^-45 absolute those."""
import math

import pytest
import torch

import decoder_reference as ref

pytestmark = pytest.mark.gpu


def check(logits, u, temperature=None, top_k=None, top_p=None, min_p=None):
    from paper_2511_03586_b200 import api
    rows = logits.shape[0]
    dev = lambda v, t: None if v is None else torch.tensor(v if isinstance(v, list) else [v] * rows, dtype=t, device="cuda")  # noqa: E731
    u_dev = dev(u, torch.float32)
    t, k, p, m = dev(temperature, torch.float32), dev(top_k, torch.int32), dev(top_p, torch.float32), dev(min_p, torch.float32)
    tokens, probs = api.pd_sample(logits, u_dev, temperature=t, top_k=k, top_p=p, min_p=m)
    cpu = logits.float().cpu()
    at = lambda v, i, none: none if v is None else v[i].item()  # noqa: E731
    for i in range(rows):
        want, prob = ref.sample_row(cpu[i], u_dev[i].item(), at(t, i, 1.0), at(k, i, 0), at(p, i, 1.0), at(m, i, 0.0))
        assert tokens[i].item() == want, (i, tokens[i].item(), want)
        assert abs(probs[i].item() - prob) <= 2 ** -22 * prob + 2 ** -45, (i, probs[i].item(), prob)
    return tokens


def logits_of(rows, vocab, dtype=torch.float32, spread=2.5, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(rows, vocab, generator=g, device="cuda") * spread).to(dtype), torch.rand(rows, generator=g, device="cuda").tolist()


SETTINGS = [dict(), dict(top_k=1), dict(top_k=50), dict(top_k=1000), dict(top_p=0.9), dict(top_p=0.05), dict(min_p=0.05),
            dict(top_k=40, top_p=0.8), dict(top_p=0.95, min_p=0.02, temperature=1.3), dict(top_k=300, top_p=0.99, min_p=0.001),
            dict(temperature=0.3), dict(temperature=0.0, top_p=0.5), dict(temperature=3.0, top_p=0.999)]


@pytest.mark.parametrize("vocab", [1, 2, 7, 511, 2049, 5000, 16385, 32000, 50257, 131073])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
def test_settings(vocab, dtype):
    x, u = logits_of(4, vocab, dtype, seed=vocab)
    for s in SETTINGS:
        check(x, u, **s)


@pytest.mark.parametrize("vocab", [200001, 327680])
def test_largest_vocabularies(vocab):
    x, u = logits_of(3, vocab, seed=vocab)
    for s in SETTINGS[3:9]:
        check(x, u, **s)


@pytest.mark.parametrize("rows", [1, 18, 19, 37, 74, 75, 148, 300])
def test_row_counts(rows):
    """Cluster sizes go by rows and vocabulary."""
    for vocab in (1500, 9000, 20000):
        x, u = logits_of(rows, vocab, torch.bfloat16, seed=rows)
        check(x, u, top_k=20, top_p=0.9)


@pytest.mark.parametrize("vocab", [1000, 40000])
def test_ties(vocab):
    """Few distinct values, equal ones by the thousand: cuts fall inside groups of equal logits."""
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randint(-3, 4, (8, vocab), generator=g, device="cuda").float()
    u = torch.rand(8, generator=g, device="cuda").tolist()
    for s in SETTINGS:
        check(x, u, **s)
    same = torch.zeros(4, vocab, device="cuda")        # all equal: running sums are whole numbers
    for s in (dict(), dict(top_k=vocab // 3), dict(top_p=0.5), dict(top_p=0.25, top_k=vocab // 2)):
        check(same, [0.0, 0.25, 0.5, 0.999], **s)
    signed = torch.zeros(4, vocab, device="cuda")      # -0 and +0 are equal
    signed[:, ::2] = -0.0
    check(signed, [0.1, 0.3, 0.6, 0.9], top_k=7)


def test_settings_differ_by_row():
    x, u = logits_of(8, 30000, seed=3)
    check(x, u, temperature=[1.0, 0.0, 0.7, 2.0, float("nan"), -1.0, 1e-6, 1e6], top_k=[0, 5, -1, 100, 0, 9, 3, 30000],
          top_p=[0.9, 1.0, 2.0, 0.0, 0.5, -1.0, float("nan"), 0.7], min_p=[0.0, 0.1, -1.0, float("nan"), 2.0, 0.5, 0.0, 0.0])


def test_random_numbers_at_their_ends():
    x, _ = logits_of(6, 10000, seed=4)
    below_one = 1.0 - 2.0 ** -24
    t = check(x, [0.0, below_one, 1.0, 5.0, -1.0, float("nan")], top_k=100)
    x1 = x[:1].expand(6, -1).contiguous()
    t = check(x1, [0.0, below_one, 1.0, 5.0, -1.0, float("nan")], top_k=100).tolist()
    assert t[0] == t[4] == t[5] and t[1] == t[2] == t[3]


@pytest.mark.parametrize("vocab", [600, 30000])
def test_masked_and_odd_logits(vocab):
    inf, nan = math.inf, math.nan
    x, u = logits_of(8, vocab, seed=5)
    x[0, :] = -inf                      # nothing to draw
    x[1, :] = nan
    x[2, ::2] = -inf
    x[3, ::3] = nan
    x[4, 17] = inf                      # takes all
    x[5, 100:110] = inf                 # share it
    x[6, :] = -inf
    x[6, vocab - 1] = -5.0
    x[7, :] = torch.finfo(torch.float32).min   # a mask of the type's lowest value
    x[7, 77] = 1.0
    for s in SETTINGS:
        t = check(x, u, **s).tolist()
        assert t[0] == t[1] == -1 and t[4] == 17 and t[6] == vocab - 1 and t[7] == 77
    low = torch.full((2, vocab), torch.finfo(torch.float32).min, device="cuda")
    for s in SETTINGS[:9]:
        check(low, [0.3, 0.9], **s)


def test_wide_and_narrow_rows():
    """Logits that differ by one step of the type, and by more than any weight can show."""
    x = 5.0 + torch.arange(4000, device="cuda").float()[None] * 2.0 ** -21
    for s in SETTINGS:
        check(x.contiguous(), [0.37], **s)
    x = (torch.arange(4000, device="cuda").float()[None] - 2000) * 1e30
    for s in SETTINGS:
        check(x.contiguous(), [0.37], **s)


@pytest.mark.parametrize("spread", [0.01, 1.0, 6.0])
def test_top_p_towards_its_ends(spread):
    """The bins that may hold the cut are bounded in single precision: shares close to 0 and to 1, flat and peaked rows."""
    x, u = logits_of(6, 60000, seed=77)
    x = (x - x.mean()) * (spread / x.std())
    for top_p in (1e-30, 1e-6, 1e-3, 0.3, 0.5, 0.75, 0.999, 0.99999, 1.0 - 2.0 ** -24):
        check(x, u, top_p=top_p)
        check(x, u, top_p=top_p, min_p=1e-4)


@pytest.mark.parametrize("ld", [1003, 1024, 1500])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
def test_strided_rows(ld, dtype):
    x, u = logits_of(5, ld, dtype, seed=ld)
    check(x[:, 3:1003] if ld > 1003 else x[:, :1000], u, top_k=30, top_p=0.9)


def test_streams_and_graphs():
    from paper_2511_03586_b200 import api
    x, u = logits_of(16, 32000, seed=8)
    u = torch.tensor(u, device="cuda")
    p = torch.full((16,), 0.9, device="cuda")
    want = api.pd_sample(x, u, top_p=p)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = api.pd_sample(x, u, top_p=p)
    s.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = api.pd_sample(x, u, top_p=p)
    u.copy_(u.flip(0))
    x.copy_(x.flip(0))
    g.replay()
    assert torch.equal(got[0], want[0].flip(0)) and torch.equal(got[1], want[1].flip(0))


def test_frequencies():
    """Drawn with evenly spread random numbers, tokens come as often as their probabilities say, to within one draw each."""
    from paper_2511_03586_b200 import api
    x, _ = logits_of(1, 50, seed=9)
    n = 4096
    u = (torch.arange(n, device="cuda") + 0.5) / n
    tokens, _ = api.pd_sample(x.expand(n, -1).contiguous(), u)
    freq = torch.bincount(tokens.long(), minlength=50).double() / n
    assert ((freq - torch.softmax(x[0].double(), 0)).abs() <= 1.0 / n + 1e-9).all()


def test_binding_refusals():
    from paper_2511_03586_b200 import api
    x, u = logits_of(4, 100)
    u = torch.tensor(u, device="cuda")
    with pytest.raises(TypeError):
        api.pd_sample(x.half(), u)
    with pytest.raises(TypeError):
        api.pd_sample(x, u.cpu())
    with pytest.raises(ValueError):
        api.pd_sample(x, u[:3])
    with pytest.raises(TypeError):
        api.pd_sample(x, u, top_k=torch.ones(4, dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError):
        api.pd_sample(x.t(), u)
    with pytest.raises(api.PdError):
        api.pd_sample(torch.zeros(1, 327681, device="cuda"), u[:1])
