"""Plain 64-bit forms of the rotation, of the append to an 8-bit paged cache and of the changes to logits, for the tests of the
kernels.  Torch on whatever device the inputs are; no code of the package."""
import math

import torch

TOP = {torch.int8: 127.0, torch.float8_e4m3fn: 448.0}


def rotate(x, pos, inv_freq, interleaved, amplitude=1.0):
    """x [n, heads, d] at positions pos [n]; also the sum of the magnitudes of each element's two terms."""
    r = 0 if inv_freq is None else 2 * inv_freq.numel()
    x = x.double()
    if r == 0:
        return x, x.abs()
    angle = pos.double()[:, None, None] * inv_freq.double()
    c, s = amplitude * torch.cos(angle), amplitude * torch.sin(angle)
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if interleaved else (x[..., :r // 2], x[..., r // 2:r])
    first, second, mag = a * c - b * s, a * s + b * c, (a.abs() + b.abs()) * abs(amplitude)
    join = lambda u, v: torch.stack((u, v), -1).flatten(-2) if interleaved else torch.cat((u, v), -1)  # noqa: E731
    return torch.cat((join(first, second), x[..., r:]), -1), torch.cat((join(mag, mag), x[..., r:].abs()), -1)


def half_step(v, dtype):
    """Half the distance between the 8-bit values around v."""
    if dtype == torch.int8:
        return torch.full_like(v, 0.5)
    binade = torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6)))
    return 2.0 ** (binade.clamp(max=8) - 4)


def append_block(fresh, kept, before, dtype):
    """Scale of a block [heads] and its older values after the new ones `fresh` [n, heads, d] (64 bits) came to the older ones
    `kept` [m, heads, d] (stored values, unscaled) at scale `before` [heads]; the older ones not rounded."""
    need = fresh.abs().amax((0, 2)) / TOP[dtype]
    need = torch.where(need > 0, need.clamp(min=2.0 ** -126), need)
    scale = torch.maximum(before, need) if len(kept) else need
    ratio = torch.where(scale > before, before / scale.clamp(min=1e-300), torch.ones_like(scale))
    return scale, kept * ratio[:, None]


def penalise_row(z, history, prompt, repetition, frequency, presence, biases, allowed):
    """One row of logits; `biases`: (token, value) in order, `allowed`: a truth value per token, or None."""
    z = z.double().clone()
    vocab = len(z)
    inside = [t for t in history if 0 <= t < vocab]
    if repetition > 0 and math.isfinite(repetition):
        for t in set(inside):
            z[t] = z[t] / repetition if z[t] > 0 else z[t] * repetition
    count = {}
    for t in history[max(prompt, 0):]:
        if 0 <= t < vocab:
            count[t] = count.get(t, 0) + 1
    for t, n in count.items():
        z[t] = z[t] - frequency * n - presence
    for t, v in {t: v for t, v in biases if 0 <= t < vocab}.items():
        z[t] = z[t] + v
    if allowed is not None:
        z[~allowed] = -math.inf
    return z
