"""Penalties, biases and masks on logits in the form for many rows (slices of 16384 logits) where a row has several slices, at the border
between that form and the one for few rows, and over unaligned rows and in place; against the definition in 64 bits, with the tolerance of
the operator's own test."""
import math

import pytest
import torch

from test_gpu_penalize_logits import check, problem

pytestmark = pytest.mark.gpu

# rows * ceil(vocab / 16384) reaches 296: the form for many rows
WIDE = [(160, 33003), (60, 128001), (37, 131072), (99, 49151), (148, 32768), (296, 16384), (148, 16385)]
NARROW = [(147, 32768), (295, 16384), (147, 16385), (98, 49152)]


def few_rows(p, rows, keep):
    """The problem's rows `keep` as a problem of their own (what is done to a row does not depend on the others)."""
    return {k: v if k == "mask" else v[keep] for k, v in p.items()}


@pytest.mark.parametrize("rows,vocab", WIDE + NARROW)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_slices(rows, vocab, dtype):
    """A sample of rows against the definition, all of them against calls of the form for few rows."""
    from paper_2511_03586_b200 import api
    p = problem(rows, vocab, 900, seed=vocab + rows, biases=300, mask=3, dtype=dtype)
    got = api.pd_penalize_logits(**p)
    for at in range(0, rows, 4):
        keep = slice(at, min(at + 4, rows))
        few = few_rows(p, rows, keep)
        alone = check(few) if at in (0, rows // 8 * 4) else api.pd_penalize_logits(**few).cpu()
        part = got[keep].cpu()
        assert bool(((part == alone) | (part.isnan() & alone.isnan())).all()), at


@pytest.mark.parametrize("rows,vocab", [(160, 33003), (60, 128001), (296, 16384)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("offset", [0, 1, 4])
def test_slices_in_place_in_a_wider_tensor(rows, vocab, offset, dtype):
    from paper_2511_03586_b200 import api
    p = problem(rows, vocab, 60, seed=rows, biases=7, mask=3, dtype=dtype)
    want = api.pd_penalize_logits(**p)
    few = few_rows(p, rows, slice(rows - 2, rows))
    assert torch.equal(check(few).nan_to_num(7.0), want[rows - 2:].cpu().nan_to_num(7.0))
    wide = torch.full((rows, vocab + 12), 9.0, dtype=dtype, device="cuda")
    inside = wide[:, offset:offset + vocab]
    inside.copy_(p["logits"])
    assert api.pd_penalize_logits(**{**p, "logits": inside}, out=inside) is inside
    assert torch.equal(inside, want)
    assert bool((wide[:, :offset] == 9).all()) and bool((wide[:, offset + vocab:] == 9).all())


@pytest.mark.parametrize("rows,vocab", [(160, 33003), (60, 128001)])
def test_each_place_of_a_slice(rows, vocab):
    """Tokens at both ends of every slice, in the history and among the biases, and mask words next to them."""
    from paper_2511_03586_b200 import api
    ends = [t for s in range(0, vocab, 16384) for t in (s - 1, s, s + 1, s + 31, s + 32, s + 16383)] + [vocab - 2, vocab - 1]
    ends = sorted({t for t in ends if 0 <= t < vocab})
    history = torch.tensor(ends, dtype=torch.int32, device="cuda").repeat(rows, 1)
    logits = torch.ones(rows, vocab, device="cuda")
    presence = torch.full((rows,), 0.25, device="cuda")
    out = api.pd_penalize_logits(logits, history=history, presence=presence)
    want = torch.ones(vocab, device="cuda")
    want[ends] = 0.75
    assert bool((out == want).all())
    values = torch.arange(1, len(ends) + 1, device="cuda").float().repeat(rows, 1)
    out = api.pd_penalize_logits(logits, bias_tokens=history, bias_values=values)
    want = torch.ones(vocab, device="cuda")
    want[ends] += values[0]
    assert bool((out == want).all())
    bits = torch.zeros((vocab + 31) // 32 * 32, dtype=torch.int64)
    bits[ends] = 1
    words = (bits.view(-1, 32) << torch.arange(32)).sum(1)
    words = torch.where(words >= 2 ** 31, words - 2 ** 32, words).to(torch.int32).cuda()[None]
    out = api.pd_penalize_logits(logits, mask=words, mask_row=torch.zeros(rows, dtype=torch.int32, device="cuda"))
    want = torch.full((vocab,), -math.inf, device="cuda")
    want[ends] = 1
    assert bool((out == want).all())
