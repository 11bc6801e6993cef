"""Cases of the operators around a decoder's 8-bit paged cache, for measuring: the rotation of queries and keys by their
positions with the append to a cache in bf16 or 8 bits, the attention over a cache held in 8 bits with a scale for each
block of tokens and head (whole prompts, chunks and single tokens), and the penalties, biases and grammar masks that are
put on logits before a token is drawn.

``listed()`` names the cases, ``draw(rng)`` makes more of the same ranges, ``prepare`` the inputs, ``run`` one pass:
in plain torch operations where ``own`` is false, through the package's entry points where it is true.  ``exact``
computes the same results in 64 bits, by other means than the plain form where there is a choice.
"""
import math

import numpy as np
import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "int8": torch.int8, "e4m3": torch.float8_e4m3fn}
_TOP = {"int8": 127.0, "e4m3": 448.0}  # the largest value of either 8-bit type that is used


# ---------------------------------------------------------------------------------------------------- the cases
def listed():
    return [
        # the new tokens of a decode batch, rotated, to a bf16 cache; far positions
        dict(name="rotate append 64 x 1", op="append", batch=64, q_max=1, q_ragged=False, kv_max=100000, kv_min=100,
             heads=32, kv_heads=8, dim=128, page=16, rotary=128, interleaved=False, cache="bf16", block=16),
        # prompts to a bf16 cache
        dict(name="rotate append 8 x 2048", op="append", batch=8, q_max=2048, q_ragged=True, kv_max=8192, kv_min=2048,
             heads=32, kv_heads=8, dim=128, page=64, rotary=128, interleaved=False, cache="bf16", block=64),
        # the same two for an 8-bit cache; half of each head rotated, pairs side by side
        dict(name="rotate quantise 64 x 1", op="append", batch=64, q_max=1, q_ragged=False, kv_max=8192, kv_min=100,
             heads=32, kv_heads=8, dim=128, page=32, rotary=64, interleaved=True, cache="e4m3", block=16),
        dict(name="rotate quantise 8 x 2048", op="append", batch=8, q_max=2048, q_ragged=True, kv_max=8192, kv_min=2048,
             heads=32, kv_heads=8, dim=128, page=64, rotary=128, interleaved=False, cache="e4m3", block=32),
        # one user, one token, a short context: what a decode step costs when nothing is large
        dict(name="attend 8-bit 1 x 1", op="attend", batch=1, q_max=1, q_ragged=False, kv_max=700, kv_min=700,
             heads=32, kv_heads=8, dim=128, page=16, window=0, sinks=0, cache="int8", block=16),
        # a decode batch of a server with ragged contexts
        dict(name="attend 8-bit 64 x 1", op="attend", batch=64, q_max=1, q_ragged=False, kv_max=8192, kv_min=200,
             heads=32, kv_heads=8, dim=128, page=16, window=0, sinks=0, cache="int8", block=16),
        # few long contexts, with a sliding window and sink tokens, the other 8-bit type
        dict(name="attend 8-bit 32 x 1 window", op="attend", batch=32, q_max=1, q_ragged=False, kv_max=32768, kv_min=1000,
             heads=32, kv_heads=4, dim=128, page=64, window=4096, sinks=4, cache="e4m3", block=64),
        # a few tokens for each sequence: drafts being verified
        dict(name="attend 8-bit 16 x 5", op="attend", batch=16, q_max=5, q_ragged=False, kv_max=8192, kv_min=100,
             heads=32, kv_heads=8, dim=128, page=32, window=0, sinks=0, cache="e4m3", block=32),
        # chunks of prompts over what earlier chunks left in the cache
        dict(name="attend 8-bit 4 x 2048 chunk", op="attend", batch=4, q_max=2048, q_ragged=True, kv_max=16384, kv_min=2048,
             heads=32, kv_heads=8, dim=128, page=64, window=0, sinks=0, cache="int8", block=32),
        # the library's own head layout (16 heads of 64, no sharing), prompts with a sliding window and sinks
        dict(name="attend 8-bit 8 x 2048 window", op="attend", batch=8, q_max=2048, q_ragged=True, kv_max=4096, kv_min=2048,
             heads=16, kv_heads=16, dim=64, page=32, window=1024, sinks=4, cache="e4m3", block=32),
        # a small batch of chats: repetition penalty, a few biases, no grammar
        dict(name="penalise 8 x 32000", op="penalise", rows=8, vocab=32000, dtype="bf16", history=1500, counted=True,
             biases=20, masked=0.0, repetition=1.1),
        # a large batch and vocabulary, long histories, a grammar for half of the rows
        dict(name="penalise 256 x 128000", op="penalise", rows=256, vocab=128000, dtype="f32", history=8000, counted=True,
             biases=300, masked=0.5, repetition=1.2),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attend", "attend", "attend", "append", "append", "penalise"])
    if op == "penalise":
        return dict(op=op, rows=_log_int(rng, 1, 128), vocab=_log_int(rng, 1000, 160000), dtype=rng.choice(["bf16", "f32"]),
                    history=_log_int(rng, 1, 16000), counted=rng.random() < 0.7, biases=rng.choice([0, 0, 1, 20, 300]),
                    masked=rng.choice([0.0, 0.0, 0.5, 1.0]), repetition=rng.choice([1.0, 0.9, 1.1, 1.5]))
    dim, page, kv_heads = rng.choice([64, 128]), rng.choice([16, 32, 64, 128]), rng.choice([1, 2, 4, 8])
    block = rng.choice([b for b in (1, 8, 16, 32, 64, 128) if b <= page])
    if rng.random() < 0.5:  # tokens one by one, or a few
        batch, q_max, kv_max = _log_int(rng, 1, 64), rng.choice([1, 1, 1, 2, 5, 9]), _log_int(rng, 64, 16384)
    else:  # chunks
        batch, q_max = _log_int(rng, 1, 4), _log_int(rng, 16, 2048)
        kv_max = q_max + rng.choice([0, _log_int(rng, 1, 4096)])
    kv_max = max(kv_max, q_max)
    case = dict(op=op, batch=batch, q_max=q_max, q_ragged=rng.random() < 0.5, kv_max=kv_max, kv_min=rng.randint(q_max, kv_max),
                heads=kv_heads * rng.choice([g for g in (1, 2, 4, 5, 8) if kv_heads * g <= 40]), kv_heads=kv_heads, dim=dim,
                page=page, block=block)
    if op == "append":
        return dict(case, cache=rng.choice(["bf16", "int8", "e4m3"]), rotary=rng.choice([dim, dim, dim // 2, 24]),
                    interleaved=rng.random() < 0.4)
    window = _log_int(rng, 16, 4096) if rng.random() < 0.4 else 0
    return dict(case, cache=rng.choice(["int8", "e4m3"]), window=window, sinks=rng.choice([0, 1, 4, 37]) if window else 0)


def _lengths(case):
    """New tokens and cached tokens (the new ones included) of each sequence: spread over the case's ranges."""
    b = case["batch"]
    q = [case["q_max"]] * b
    if case["q_ragged"]:
        q = [max(1, case["q_max"] - (i * 7919) % (case["q_max"] // 2 + 1)) for i in range(b)]
    lo = case["kv_min"]
    kv = [case["kv_max"] - int((case["kv_max"] - lo) * ((i * 0.6180339887) % 1.0)) for i in range(b)]
    return q, [max(k, n) for k, n in zip(kv, q)]


# --------------------------------------------------------------------------------------------------- the inputs
def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda")  # noqa: E731
    uniform = lambda *shape: torch.rand(*shape, generator=g, device="cuda")  # noqa: E731
    whole = lambda v: torch.tensor(np.asarray(v, dtype=np.int32)).cuda()  # noqa: E731
    s = dict(case=case)
    if case["op"] == "penalise":
        r, v = case["rows"], case["vocab"]
        s["logits"] = (normal(r, v) * 2.5).to(_DTYPES[case["dtype"]])
        # prompt and answer so far: tokens repeat as words do, a few of them often
        s["history"] = (uniform(r, case["history"]) ** 4 * v).to(torch.int32).clamp_(max=v - 1)
        s["history_len"] = (case["history"] * (0.25 + 0.75 * uniform(r))).to(torch.int32)
        s["prompt_len"] = (s["history_len"] * uniform(r)).to(torch.int32)
        s["repetition"] = torch.full((r,), case["repetition"], device="cuda") if case["repetition"] != 1.0 else None
        s["frequency"] = 0.5 * uniform(r) if case["counted"] else None
        s["presence"] = 0.5 * uniform(r) if case["counted"] else None
        s["bias_tokens"] = s["bias_values"] = s["mask"] = s["mask_row"] = None
        if case["biases"]:  # different tokens of a row, some of them forbidden outright
            step = max(1, v // case["biases"])
            n = min(case["biases"], v)
            s["bias_tokens"] = (torch.arange(n, device="cuda") * step + (uniform(r, 1) * step).long()).clamp_(max=v - 1).to(torch.int32)
            s["bias_values"] = normal(r, n) * 3
            s["bias_values"][:, ::7] = -math.inf
        if case["masked"]:  # a grammar's state allows some of the tokens; rows without one have no mask
            groups = max(1, int(r * case["masked"]))
            s["mask"] = torch.randint(-2 ** 31, 2 ** 31, (groups, (v + 31) // 32), generator=g, device="cuda").to(torch.int32)
            row = torch.arange(r, device="cuda")
            s["mask_row"] = torch.where(row < groups, row, -1).to(torch.int32)[torch.randperm(r, generator=g, device="cuda")].contiguous()
        return s
    q, kv = _lengths(case)
    tokens, page, block = sum(q), case["page"], case["block"]
    hq, hk, d = case["heads"], case["kv_heads"], case["dim"]
    # the projection's packed output: queries, keys and values of a token side by side
    s["qkv"] = normal(tokens, (hq + 2 * hk) * d).to(torch.bfloat16)
    s["q"] = s["qkv"][:, :hq * d].unflatten(1, (hq, d))
    s["k"] = s["qkv"][:, hq * d:(hq + hk) * d].unflatten(1, (hk, d))
    s["v"] = s["qkv"][:, (hq + hk) * d:].unflatten(1, (hk, d))
    # an append only touches the pages from the first new token's on: the others are left out of its cache
    first = [(n - m) // page if case["op"] == "append" else 0 for m, n in zip(q, kv)]
    need = [(n + page - 1) // page for n in kv]
    pages, width = sum(n - f for n, f in zip(need, first)) + 3, max(need)
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32).cpu()
    table, at = torch.full((len(q), width), -1, dtype=torch.int32), 0
    for i, (f, n) in enumerate(zip(first, need)):
        table[i, f:n] = order[at:at + n - f]
        at += n - f
    s["table"] = table.cuda()
    for c in ("k", "v"):
        x = normal(pages, page, hk, d)
        if case["cache"] == "bf16":
            s[c + "_cache"] = x.to(torch.bfloat16)
        else:
            x = x.unflatten(1, (page // block, block))
            scale = x.abs().amax((2, 4)) / _TOP[case["cache"]]                                       # [pages, blocks, hk]
            x = (x / scale[:, :, None, :, None]).flatten(1, 2)
            s[c + "_cache"] = (x.round() if case["cache"] == "int8" else x).clamp_(-_TOP[case["cache"]], _TOP[case["cache"]]).to(_DTYPES[case["cache"]])
            s[c + "_scale"] = scale.transpose(1, 2).contiguous()                                     # [pages, hk, blocks]
        del x
    s["q_len"], s["kv_len"] = q, kv
    s["cu_q"], s["kv_len_dev"] = whole(np.concatenate([[0], np.cumsum(q)])), whole(kv)
    # where each new token goes (sequence, place in it and position), and the tokens before them in blocks that get new ones
    s["seq_of"] = whole(np.repeat(np.arange(len(q)), q)).long()
    s["place_of"] = whole(np.concatenate([np.arange(n) for n in q])).long()
    s["pos_of"] = whole(np.concatenate([np.arange(k - n, k) for n, k in zip(q, kv)])).long()
    if case["op"] == "append":
        old = [np.arange((k - n) // block * block, k - n) for n, k in zip(q, kv)]
        s["old_seq"], s["old_pos"] = whole(np.repeat(np.arange(len(q)), [len(o) for o in old])).long(), whole(np.concatenate(old)).long()
        s["inv_freq"] = (500000.0 ** (-torch.arange(0, case["rotary"], 2, dtype=torch.float64) / case["rotary"])).float().cuda()
        s["q_out"] = torch.zeros(tokens, hq, d, dtype=torch.bfloat16, device="cuda")
    return s


# ------------------------------------------------------------------------------------------------------ one pass
def run(state):
    return (_own if own else _plain)[state["case"]["op"]](state)


def _plain_attend(s):
    c = s["case"]
    hk, group, d, block, n = c["kv_heads"], c["heads"] // c["kv_heads"], c["dim"], c["block"], c["q_max"]
    pages = s["table"].clamp(min=0).long()

    def sequences(name):  # [batch, hk, keys, d], the values that the cache stands for
        x = s[name + "_cache"][pages].float()
        scale = s[name + "_scale"].transpose(1, 2).repeat_interleave(block, 1)[pages]
        return (x * scale[..., None]).flatten(1, 2).transpose(1, 2)

    k, v = sequences("k"), sequences("v")
    batch, length = k.shape[0], k.shape[2]
    q = torch.zeros(batch, n, hk * group, d, device="cuda")
    q[s["seq_of"], s["place_of"]] = s["q"].float()
    q = q.unflatten(2, (hk, group)).permute(0, 2, 3, 1, 4).flatten(2, 3)                            # [batch, hk, group * n, d]
    scores = torch.matmul(q, k.transpose(2, 3)).unflatten(2, (group, n)) / math.sqrt(d)
    pos = (s["kv_len_dev"] - (s["cu_q"][1:] - s["cu_q"][:-1]))[:, None, None].long() + torch.arange(n, device="cuda")[:, None]
    key = torch.arange(length, device="cuda")
    seen = key <= pos
    if c["window"]:
        seen &= (key > pos - c["window"]) | (key < c["sinks"])
    scores.masked_fill_(~seen[:, None, None], -math.inf)
    p = scores.sub_(scores.amax(-1, keepdim=True)).exp_()
    out = torch.matmul(p.flatten(2, 3), v).unflatten(2, (group, n)) / p.sum(-1, keepdim=True)
    out = out.permute(0, 3, 1, 2, 4).flatten(2, 3)                                                  # [batch, n, heads, d]
    return out[s["seq_of"], s["place_of"]].to(torch.bfloat16)


def _rotated(x, s):
    """In 64 bits: the angles of far positions, and values next to a border between two 8-bit ones."""
    c = s["case"]
    half = c["rotary"] // 2
    angle = s["pos_of"].double()[:, None, None] * s["inv_freq"].double()
    cos, sin, x = torch.cos(angle), torch.sin(angle), x.double()
    part = x[..., :2 * half]
    a, b = (part[..., 0::2], part[..., 1::2]) if c["interleaved"] else (part[..., :half], part[..., half:])
    a, b = a * cos - b * sin, a * sin + b * cos
    part = torch.stack((a, b), -1).flatten(-2) if c["interleaved"] else torch.cat((a, b), -1)
    return torch.cat((part, x[..., 2 * half:]), -1)


def _plain_append(s):
    c = s["case"]
    page, block, kind = c["page"], c["block"], c["cache"]
    s["q_out"].copy_(_rotated(s["q"], s))
    where, slot = s["table"][s["seq_of"], s["pos_of"] // page].long(), s["pos_of"] % page
    if kind == "bf16":
        s["k_cache"][where, slot] = _rotated(s["k"], s).to(torch.bfloat16)
        s["v_cache"][where, slot] = s["v"]
        return s["q_out"], s["k_cache"], s["v_cache"]
    top, blocks = _TOP[kind], page // block
    old_where, old_slot = s["table"][s["old_seq"], s["old_pos"] // page].long(), s["old_pos"] % page
    at, old_at = where * blocks + slot // block, old_where * blocks + old_slot // block              # blocks of the whole cache

    def rounded(x):
        x = (x.round() if kind == "int8" else x.float()).clamp(-top, top)
        return x.to(torch.int8) if kind == "int8" else x.to(torch.float8_e4m3fn).view(torch.int8)

    for name, x in (("k", _rotated(s["k"], s)), ("v", s["v"].double())):
        cache = s[name + "_cache"]
        bits = cache.view(torch.int8)
        before = s[name + "_scale"].transpose(1, 2).flatten(0, 1)                                     # [pages * blocks, hk]
        most = x.abs().amax(-1)
        need = torch.zeros_like(before).index_reduce_(0, at, most.float() / top, "amax")
        keeps = torch.zeros(before.shape[0], 1, device="cuda").index_fill_(0, old_at, 1.0) > 0          # holds older tokens
        touched = torch.zeros(before.shape[0], 1, device="cuda").index_fill_(0, at, 1.0) > 0
        after = torch.where(touched, torch.where(keeps, torch.maximum(before, need), need), before)
        scale = after[old_at].double()[..., None]
        value = cache[old_where, old_slot].double() * (before[old_at].double()[..., None] / scale.clamp(min=1e-300))
        bits[old_where, old_slot] = torch.where(after[old_at][..., None] > before[old_at][..., None], rounded(value), bits[old_where, old_slot])
        bits[where, slot] = rounded(x / after[at].double()[..., None].clamp(min=1e-300))
        s[name + "_scale"].copy_(after.unflatten(0, (-1, blocks)).transpose(1, 2))
    return _cache_outputs(s)


def _cache_outputs(s):
    """The caches as the values that they stand for: the 8-bit floats with their scales, whole numbers times theirs."""
    if s["case"]["cache"] != "int8":
        return s["q_out"], s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"]
    values = lambda n: s[n + "_cache"] * s[n + "_scale"].transpose(1, 2).repeat_interleave(s["case"]["block"], 1)[..., None]  # noqa: E731
    return s["q_out"], values("k").to(torch.bfloat16), values("v").to(torch.bfloat16)


def _plain_penalise(s):
    z = s["logits"].float()
    rows, vocab = z.shape
    place = torch.arange(s["history"].shape[1], device="cuda")[None]
    there = place < s["history_len"][:, None]
    answer = (there & (place >= s["prompt_len"][:, None])).float()
    tokens = s["history"].long()
    seen = torch.zeros_like(z).scatter_add_(1, tokens, there.float()) > 0
    count = torch.zeros_like(z).scatter_add_(1, tokens, answer)
    if s["repetition"] is not None:
        r = s["repetition"][:, None]
        z = torch.where(seen, torch.where(z > 0, z / r, z * r), z)
    if s["frequency"] is not None:
        z = z - s["frequency"][:, None] * count - s["presence"][:, None] * (count > 0)
    if s["bias_tokens"] is not None:
        z = z.scatter_add(1, s["bias_tokens"].long(), s["bias_values"])
    if s["mask"] is not None:
        token = torch.arange(vocab, device="cuda")
        allowed = (s["mask"][:, token // 32] >> (token % 32)) & 1
        allowed = (allowed[s["mask_row"].clamp(min=0).long()] > 0) | (s["mask_row"] < 0)[:, None]
        z = z.masked_fill(~allowed, -math.inf)
    return z.to(s["logits"].dtype)


def _own_attend(s):
    from paper_2511_03586_b200 import api
    c = s["case"]
    return api.pd_attention_paged_q8_fwd(s["q"], s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"], s["table"], s["cu_q"],
                                         s["kv_len_dev"], max_q_len=c["q_max"], max_kv_len=c["kv_max"], window=c["window"],
                                         sinks=c["sinks"])


def _own_append(s):
    from paper_2511_03586_b200 import api
    c = s["case"]
    bf16 = c["cache"] == "bf16"
    api.pd_rope_kv_cache_append(s["k"], s["v"], s["k_cache"], s["v_cache"], s["table"], s["cu_q"], s["kv_len_dev"], q=s["q"],
                                q_out=s["q_out"], inv_freq=s["inv_freq"], interleaved=c["interleaved"],
                                k_scale=None if bf16 else s["k_scale"], v_scale=None if bf16 else s["v_scale"])
    return (s["q_out"], s["k_cache"], s["v_cache"]) if bf16 else _cache_outputs(s)


def _own_penalise(s):
    from paper_2511_03586_b200 import api
    return api.pd_penalize_logits(s["logits"], history=s["history"], history_len=s["history_len"], prompt_len=s["prompt_len"],
                                  repetition=s["repetition"], frequency=s["frequency"], presence=s["presence"],
                                  bias_tokens=s["bias_tokens"], bias_values=s["bias_values"], mask=s["mask"],
                                  mask_row=s["mask_row"])


_plain = {"attend": _plain_attend, "append": _plain_append, "penalise": _plain_penalise}
_own = {"attend": _own_attend, "append": _own_append, "penalise": _own_penalise}


# ------------------------------------------------------------------------------------------------ the least work
def _pairs(case, n, length):
    """Visible (query, key) pairs of one sequence, and the keys that some query sees."""
    first = length - n
    w, s = case["window"], case["sinks"]
    if w == 0:
        return n * first + n * (n + 1) // 2, length
    pos = np.arange(first, length, dtype=np.int64)
    low = np.maximum(pos - w + 1, 0)
    seen = int(low[0])
    return int(np.sum(pos - low + 1 + np.minimum(s, low))), length - seen + min(s, seen)


def work(case):
    if case["op"] == "penalise":
        r, v = case["rows"], case["vocab"]
        masks = (max(1, int(r * case["masked"])) if case["masked"] else 0) * ((v + 31) // 32) * 4
        return {"bytes": r * v * 2 * (2 if case["dtype"] == "bf16" else 4) + int(r * case["history"] * 0.625) * 4 + masks + r * case["biases"] * 8,
                "flops": 4 * r * v}
    q, kv = _lengths(case)
    hq, hk, d = case["heads"], case["kv_heads"], case["dim"]
    if case["op"] == "append":
        wide = 2 if case["cache"] == "bf16" else 1
        scales = 0 if wide == 2 else 2 * 4 * sum((n - 1) // case["block"] + 1 for n in q) * hk
        return {"bytes": sum(q) * (2 * 2 * hq * d + 2 * hk * d * (2 + wide)) + scales, "flops": 3 * sum(q) * (hq + hk) * case["rotary"]}
    pairs, keys = zip(*(_pairs(case, n, k) for n, k in zip(q, kv)))
    return {"bytes": 2 * 2 * sum(q) * hq * d + 2 * sum(keys) * hk * d + 2 * 4 * sum(keys) // case["block"] * hk + 4 * sum(keys) // case["page"],
            "flops": 4 * sum(pairs) * hq * d}


# ---------------------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"attend": _exact_attend, "append": _exact_append, "penalise": _exact_penalise}[case["op"]](case, s)


def _exact_attend(case, s):
    """One cache head and up to 512 queries at a time; every weight is taken relative to the log of the visible ones' sum."""
    hk, group, d, block = case["kv_heads"], case["heads"] // case["kv_heads"], case["dim"], case["block"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    start = 0
    for i, (n, length) in enumerate(zip(s["q_len"], s["kv_len"])):
        index = torch.arange(length, device="cuda")
        page, slot = s["table"][i].long()[index // case["page"]], index % case["page"]
        for h in range(hk):
            k = s["k_cache"][page, slot, h].double() * s["k_scale"][page, h, slot // block].double()[:, None]
            v = s["v_cache"][page, slot, h].double() * s["v_scale"][page, h, slot // block].double()[:, None]
            for a in range(0, n, 512):
                b = min(n, a + 512)
                pos = (length - n + torch.arange(a, b, device="cuda")).repeat_interleave(group)
                low = pos - case["window"] + 1 if case["window"] else torch.zeros_like(pos)
                hidden = (index[None] > pos[:, None]) | ((index[None] < low[:, None]) & (index[None] >= case["sinks"]))
                q = s["q"][start + a:start + b, h * group:(h + 1) * group].reshape(-1, d).double()
                z = (q @ k.T) * d ** -0.5
                z[hidden] = -math.inf
                weight = torch.exp(z - torch.logsumexp(z, -1, keepdim=True))
                out[start + a:start + b, h * group:(h + 1) * group] = (weight @ v).view(b - a, group, d)
        start += n
    return out


def _exact_append(case, s):
    """Pairs as complex numbers, turned by e^(i angle); sequence by sequence, block by block."""
    def turned(x, first):
        angle = (first + torch.arange(x.shape[0], device="cuda")).double()[:, None, None] * s["inv_freq"].double()
        z, half = x[..., :case["rotary"]].double(), case["rotary"] // 2
        z = z.unflatten(-1, (half, 2)) if case["interleaved"] else z.unflatten(-1, (2, half)).transpose(-1, -2)
        z = torch.view_as_real(torch.view_as_complex(z.contiguous()) * torch.polar(torch.ones_like(angle), angle))
        z = z.flatten(-2) if case["interleaved"] else z.transpose(-1, -2).flatten(-2)
        return torch.cat((z, x[..., case["rotary"]:].double()), -1)

    kind, page, block = case["cache"], case["page"], case["block"]
    top = _TOP.get(kind)
    rounded = lambda x: (torch.round(x) if kind == "int8" else x.float().to(torch.float8_e4m3fn).double()).clamp(-top, top)  # noqa: E731
    q_out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    caches = {n: s[n + "_cache"].double() for n in "kv"}
    scales = {n: s[n + "_scale"].double() for n in "kv" if kind != "bf16"}
    at = 0
    for i, (n, length) in enumerate(zip(s["q_len"], s["kv_len"])):
        first, mine = length - n, slice(at, at + n)
        q_out[mine] = turned(s["q"][mine], first)
        for name, x in (("k", turned(s["k"][mine], first)), ("v", s["v"][mine].double())):
            pos = torch.arange(first, length, device="cuda")
            where, slot = s["table"][i].long()[pos // page], pos % page
            if kind == "bf16":
                caches[name][where, slot] = x
                continue
            for b in range(first // block, (length - 1) // block + 1):
                lo, hi = max(first, b * block), min(length, (b + 1) * block)
                pg, at_block, from_slot = int(s["table"][i, lo // page]), b % (page // block), b * block % page
                fresh = x[lo - first:hi - first]                                                    # [tokens, hk, d]
                scale = fresh.abs().amax((0, 2)) / top
                if lo > b * block:
                    before = scales[name][pg, :, at_block].clone()
                    scale = torch.maximum(scale, before)
                    kept = caches[name][pg, from_slot:lo % page]
                    kept.copy_(torch.where((scale > before)[:, None], rounded(kept * (before / scale)[:, None]), kept))
                scales[name][pg, :, at_block] = scale
                caches[name][pg, lo % page:lo % page + hi - lo] = rounded(fresh / scale[:, None])
        at += n
    if kind == "bf16":
        return q_out, caches["k"], caches["v"]
    if kind == "e4m3":
        return q_out, caches["k"], caches["v"], scales["k"], scales["v"]
    return (q_out,) + tuple(caches[n] * scales[n].transpose(1, 2).repeat_interleave(block, 1)[..., None] for n in "kv")


def _exact_penalise(case, s):
    """Row by row on the host."""
    host = {k: v.cpu().numpy() for k, v in s.items() if isinstance(v, torch.Tensor) and v.dtype != torch.bfloat16}
    z = s["logits"].double().cpu().numpy()
    for i, row in enumerate(z):
        n, m = int(host["history_len"][i]), int(host["prompt_len"][i])
        if s["repetition"] is not None:
            seen = np.unique(host["history"][i, :n])
            r = float(host["repetition"][i])
            row[seen] = np.where(row[seen] > 0, row[seen] / r, row[seen] * r)
        if s["frequency"] is not None:
            answered, count = np.unique(host["history"][i, m:n], return_counts=True)
            row[answered] -= count * float(host["frequency"][i]) + float(host["presence"][i])
        if s["bias_tokens"] is not None:
            row[host["bias_tokens"][i]] += host["bias_values"][i].astype(np.float64)
        if s["mask"] is not None and host["mask_row"][i] >= 0:
            words = host["mask"][host["mask_row"][i]].view(np.uint32)
            bits = np.unpackbits(words.view(np.uint8), bitorder="little")[:case["vocab"]]
            row[bits == 0] = -math.inf
    return torch.from_numpy(z).cuda()
