"""Plain 64-bit forms of the decoder operators, for the tests of the kernels.  Torch on whatever device the inputs are;
no code of the package."""
import math

import torch


def attention(q, k_seq, v_seq, pos0, *, window=0, sinks=0, scale=None):
    """q [n, heads, d] at positions pos0 ...; k_seq, v_seq [length, heads_kv, d].  Returns (out, weighted |v|), [n, heads, d],
    zeros where nothing is visible."""
    n, heads, d = q.shape
    length, heads_kv, _ = k_seq.shape
    group = heads // heads_kv
    out = torch.zeros(n, heads, d, dtype=torch.float64, device=q.device)
    mag = torch.zeros_like(out)
    scale = d ** -0.5 if scale is None else scale
    pos = pos0 + torch.arange(n, device=q.device)[:, None]
    key = torch.arange(length, device=q.device)[None, :]
    seen = key <= pos
    if window:
        seen = seen & ((key > pos - window) | (key < sinks))
    for h in range(heads):
        k, v = k_seq[:, h // group].double(), v_seq[:, h // group].double()
        z = (q[:, h].double() @ k.T) * scale
        z = torch.where(seen, z, torch.full_like(z, -math.inf))
        top = z.amax(-1, keepdim=True) if length else torch.full((n, 1), -math.inf, device=q.device, dtype=torch.float64)
        top = torch.where(top == -math.inf, torch.zeros_like(top), top)
        p = torch.where(seen, torch.exp(z - top), torch.zeros_like(z))
        total = p.sum(-1, keepdim=True)
        p = torch.where(total > 0, p / total.clamp_min(1e-300), torch.zeros_like(p))
        out[:, h] = p @ v
        mag[:, h] = p @ v.abs()
    return out, mag


def norm(kind, v, gamma, beta, eps):
    if kind == "none":
        return v
    if kind == "layer":
        v = v - v.mean(-1, keepdim=True)
    v = v / torch.sqrt((v * v).mean(-1, keepdim=True) + eps)
    if gamma is not None:
        v = v * gamma.double()
    return v + beta.double() if kind == "layer" and beta is not None else v


def norm_gate_residual_norm(y, x, gate, gate_rows, alpha, eps, post, post_gamma, post_beta, pre, pre_gamma, pre_beta):
    block = norm(post, y.double(), post_gamma, post_beta, eps)
    if gate is not None:
        gate = gate.reshape(-1, y.shape[1]).double()
        block = block * gate[torch.arange(y.shape[0], device=y.device) // gate_rows]
    h = alpha * x.double() + block
    return h, norm(pre, h, pre_gamma, pre_beta, eps)


def sample_row(x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """One row: (token, probability)."""
    x = torch.where(torch.isnan(x.double()), torch.full_like(x.double(), -math.inf), x.double())
    top = float(x.max())
    if top == -math.inf:
        return -1, 0.0
    if not temperature > 0:
        temperature, top_k = 1.0, 1
    w = torch.where(x == top, torch.ones_like(x), torch.exp((x - top) / temperature)) if math.isfinite(top) else (x == top).double()
    order = torch.sort(x, descending=True, stable=True).indices
    if 0 < top_k < len(x):
        order = order[:top_k]
    if top_p < 1.0:
        reach = torch.cumsum(w[order], 0)
        before = reach - w[order]
        keep = before < max(top_p, 0.0) * reach[-1]
        keep[0] = True
        order = order[keep]
    if min_p > 0:
        order = order[w[order] >= min(min_p, 1.0)]
    order = order.sort().values
    order = order[w[order] > 0]
    reach = torch.cumsum(w[order], 0)
    u = min(max(u, 0.0), 1.0 - 2.0 ** -24) if u == u else 0.0
    at = min(int((reach <= u * reach[-1]).sum()), len(order) - 1)
    return int(order[at]), float(w[order[at]] / reach[-1])
