"""Penalties, biases and masks on logits, against the definition in 64 bits.

Tolerance: a quotient or product, two differences, a product and a sum, in fp32: six roundings of 2^-24 of what they act on, all
at most the largest of |z| r, f n, g, |bias| added up; then one rounding to the type of the result."""
import math
import random

import pytest
import torch

import decoder_q8_reference as ref

pytestmark = pytest.mark.gpu


def problem(rows, vocab, columns, *, seed=0, biases=0, mask=None, dtype=torch.float32):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = random.Random(seed)
    p = dict(logits=(torch.randn(rows, vocab, generator=g, device="cuda") * 3).to(dtype))
    if columns:
        spread = min(vocab, max(2, columns // 2))
        p["history"] = (torch.randint(0, spread, (rows, columns), generator=g, device="cuda") * (vocab // spread) + vocab % spread // 2).to(torch.int32)
        p["history"][torch.rand(rows, columns, generator=g, device="cuda") < 0.05] = -1
        p["history"][torch.rand(rows, columns, generator=g, device="cuda") < 0.05] = vocab
        p["history_len"] = torch.tensor([r.choice([0, 1, columns, columns + 5, r.randint(0, columns), -3]) for _ in range(rows)], dtype=torch.int32, device="cuda")
        p["prompt_len"] = torch.tensor([r.choice([0, 1, columns, r.randint(0, columns), -1]) for _ in range(rows)], dtype=torch.int32, device="cuda")
        p["repetition"] = torch.tensor([r.choice([1.0, 1.2, 0.8, 5.0]) for _ in range(rows)], device="cuda")
        p["frequency"] = torch.tensor([r.choice([0.0, 0.3, -0.2]) for _ in range(rows)], device="cuda")
        p["presence"] = torch.tensor([r.choice([0.0, 0.7, -0.4]) for _ in range(rows)], device="cuda")
    if biases:
        p["bias_tokens"] = torch.randint(-2, vocab + 2, (rows, biases), generator=g, device="cuda").to(torch.int32)
        p["bias_values"] = torch.randn(rows, biases, generator=g, device="cuda") * 5
        p["bias_values"][torch.rand(rows, biases, generator=g, device="cuda") < 0.1] = -math.inf
    if mask:
        p["mask"] = torch.randint(-2 ** 31, 2 ** 31, (mask, (vocab + 31) // 32), generator=g, device="cuda").to(torch.int32)
        p["mask_row"] = torch.tensor([r.randint(-1, mask) for _ in range(rows)], dtype=torch.int32, device="cuda")
    return p


def check(p, out=None, **kw):
    from paper_2511_03586_b200 import api
    logits = p["logits"]
    host = {k: v.cpu().clone() for k, v in p.items()}
    got = api.pd_penalize_logits(**p, out=out, **kw)
    rows, vocab = logits.shape
    assert got.shape == logits.shape
    eps = torch.finfo(got.dtype).eps / 2 if got.dtype == torch.bfloat16 else 2.0 ** -24
    got = got.cpu()
    for i in range(rows):
        n = 0
        if "history" in host:
            n = min(max(int(host["history_len"][i]), 0), host["history"].shape[1]) if "history_len" in host else host["history"].shape[1]
        history = host["history"][i, :n].tolist() if n else []
        value = lambda name, none: float(host[name][i]) if name in host else none  # noqa: E731
        rep, freq, pres = value("repetition", 1.0), value("frequency", 0.0), value("presence", 0.0)
        biases = list(zip(host["bias_tokens"][i].tolist(), host["bias_values"][i].tolist())) if "bias_tokens" in host else []
        allowed = None
        if "mask" in host:
            m = int(host["mask_row"][i]) if "mask_row" in host else i
            if 0 <= m < host["mask"].shape[0]:
                token = torch.arange(vocab)
                allowed = ((host["mask"][m][token // 32] >> (token % 32)) & 1).bool()
        want = ref.penalise_row(host["logits"][i], history, int(host["prompt_len"][i]) if "prompt_len" in host else 0, rep, freq, pres, biases, allowed)
        sizes = host["logits"][i].double().abs() * max(rep, 1 / rep if rep > 0 else 1, 1) + abs(freq) * len(history) + abs(pres)
        finite = {t: abs(v) for t, v in biases if math.isfinite(v)}
        sizes = sizes + max(finite.values(), default=0.0)
        g = got[i].double()
        # (3.5 / 1e-38 = 3.5e38 is beyond fp32's 3.4e38 and has no value there but infinity)
        same = (g == want.float().double()) | ((g - want).abs() <= 6 * 2.0 ** -24 * sizes + eps * want.abs() * 1.01) | (g.isnan() & want.isnan())
        assert bool(same.all()), (i, (~same).nonzero()[:5].tolist())
    return got


@pytest.mark.parametrize("rows,vocab", [(1, 1), (1, 31), (3, 33), (2, 100), (5, 2048), (4, 2049), (3, 8191), (2, 50257), (1, 128000), (40, 8200), (300, 9000)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_everything_at_once(rows, vocab, dtype):
    check(problem(rows, vocab, 60, seed=vocab, biases=7, mask=3, dtype=dtype))


@pytest.mark.parametrize("columns,biases,mask", [(0, 0, None), (1, 0, None), (0, 5, None), (0, 0, 2), (5000, 0, None), (7, 2047, 1)])
@pytest.mark.parametrize("rows,vocab", [(4, 1000), (2, 20000), (300, 16001)])
def test_parts(rows, vocab, columns, biases, mask):
    check(problem(rows, vocab, columns, seed=columns + biases, biases=biases, mask=mask))


def test_settings_left_out():
    p = problem(6, 3000, 50, seed=9)
    for name in ("history_len", "prompt_len", "repetition", "frequency", "presence"):
        check({k: v for k, v in p.items() if k != name})
    q = problem(3, 300, 0, mask=3)
    del q["mask_row"]
    check(q)


def test_types_strides_and_in_place():
    p = problem(5, 4099, 40, biases=3, mask=2, dtype=torch.bfloat16)
    check(p, out=torch.empty(5, 4099, device="cuda"))
    wide = torch.full((5, 5000), 9.0, device="cuda")
    check(p, out=wide[:, 3:4102])
    assert bool((wide[:, :3] == 9).all()) and bool((wide[:, 4102:] == 9).all())
    p = problem(5, 4096, 40, biases=3, mask=2)
    check(p, out=torch.empty(5, 4096, device="cuda", dtype=torch.bfloat16))
    p["history"] = torch.cat([p["history"], p["history"]], 1)[:, 3:43]
    p["mask"] = torch.cat([p["mask"], p["mask"]], 1)[:, 1:]
    check(p, out=p["logits"])


def test_settings_that_count_as_none():
    p = problem(6, 500, 30, seed=2)
    p["repetition"] = torch.tensor([0.0, -1.0, math.nan, math.inf, 1e-38, 1.0], device="cuda")
    host = p["repetition"].clone()
    got = check({**p, "repetition": torch.where((host > 0) & host.isfinite(), host, 1.0)})
    from paper_2511_03586_b200 import api
    assert torch.equal(api.pd_penalize_logits(**p).cpu(), got)


def test_infinite_and_nan_logits():
    p = problem(3, 700, 30, mask=2, seed=3)
    p["mask_row"] = torch.tensor([0, 1, -1], dtype=torch.int32, device="cuda")
    p["logits"][:, ::5], p["logits"][:, 1::5], p["logits"][:, 2::5] = -math.inf, math.inf, math.nan
    check(p)


def test_one_token_many_times():
    """Counts up to the limit of the history."""
    columns = (1 << 20) - 1
    p = dict(logits=torch.zeros(2, 4000, device="cuda"), history=torch.full((2, columns), 17, dtype=torch.int32, device="cuda"),
             prompt_len=torch.tensor([0, 5], dtype=torch.int32, device="cuda"), frequency=torch.tensor([0.5, 0.25], device="cuda"))
    from paper_2511_03586_b200 import api
    out = api.pd_penalize_logits(**p)
    assert out[0, 17].item() == -0.5 * columns and out[1, 17].item() == -0.25 * (columns - 5)
    out[:, 17] = 0
    assert not out.any()
