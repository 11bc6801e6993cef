"""Cases of the paged-cache decoder operators, for measuring: the key/value cache and the attention that reads it
(whole prompts, chunks of new tokens and single tokens; with a sliding window and sink tokens), the norms, gate and
scaled residual between two blocks, and the sampling of a token from its logits.

``listed()`` names the cases, ``draw(rng)`` makes more of the same ranges, ``prepare`` the inputs, ``run`` one pass:
in plain torch operations where ``own`` is false, through the package's entry points where it is true.  ``exact``
computes the same results in 64 bits, by other means than the plain form where there is a choice.
"""
import math

import numpy as np
import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---------------------------------------------------------------------------------------------------- the cases
def listed():
    return [
        # one user, one token, a short context: what a decode step costs when nothing is large
        dict(name="attend 1 x 1 token", op="attend", batch=1, q_max=1, q_ragged=False, kv_max=700, kv_min=700,
             heads=32, kv_heads=8, dim=128, page=16, window=0, sinks=0),
        # a decode batch of a server with ragged contexts, small pages
        dict(name="attend 64 x 1 token", op="attend", batch=64, q_max=1, q_ragged=False, kv_max=8192, kv_min=200,
             heads=32, kv_heads=8, dim=128, page=16, window=0, sinks=0),
        # decode with a sliding window and sink tokens over long contexts
        dict(name="attend 32 x 1 window", op="attend", batch=32, q_max=1, q_ragged=False, kv_max=32768, kv_min=1000,
             heads=32, kv_heads=4, dim=128, page=64, window=4096, sinks=4),
        # a few tokens for each sequence: drafts being verified
        dict(name="attend 16 x 5 tokens", op="attend", batch=16, q_max=5, q_ragged=False, kv_max=4096, kv_min=100,
             heads=32, kv_heads=8, dim=128, page=32, window=0, sinks=0),
        # chunks of prompts over what earlier chunks left in the cache
        dict(name="attend 4 x 2048 chunk", op="attend", batch=4, q_max=2048, q_ragged=True, kv_max=16384, kv_min=2048,
             heads=32, kv_heads=8, dim=128, page=64, window=0, sinks=0),
        # the library's own head layout (16 heads of 64, no sharing), prompts with a sliding window and sinks
        dict(name="attend 8 x 4096 window", op="attend", batch=8, q_max=4096, q_ragged=True, kv_max=8192, kv_min=4096,
             heads=16, kv_heads=16, dim=64, page=32, window=1024, sinks=4),
        # the new keys and values of a decode batch, and of prompts, go to their pages
        dict(name="append 64 x 1 token", op="append", batch=64, q_max=1, q_ragged=False, kv_max=512, kv_min=1,
             heads=32, kv_heads=8, dim=128, page=16, window=0, sinks=0),
        dict(name="append 8 x 2048 tokens", op="append", batch=8, q_max=2048, q_ragged=True, kv_max=4096, kv_min=2048,
             heads=32, kv_heads=8, dim=128, page=64, window=0, sinks=0),
        # between two blocks of a decode step: RMSNorm after, RMSNorm before, bf16 stream
        dict(name="norms 64 x 4096", op="norms", rows=64, cols=4096, post="rms", pre="rms", gate_rows=0, alpha=1.0,
             stream="bf16", block="bf16"),
        # the same for prompts, with a gate for each sequence and an fp32 residual stream
        dict(name="norms 16384 x 4096", op="norms", rows=16384, cols=4096, post="rms", pre="layer", gate_rows=512,
             alpha=1.25, stream="f32", block="bf16"),
        # a small batch with the usual settings, half precision logits
        dict(name="sample 8 x 32000", op="sample", rows=8, vocab=32000, dtype="bf16", top_k=50, top_p=0.9, min_p=0.0,
             masked=0),
        # a large batch and vocabulary, nucleus and min-p without top-k, part of the vocabulary masked
        dict(name="sample 256 x 128000", op="sample", rows=256, vocab=128000, dtype="f32", top_k=0, top_p=0.95,
             min_p=0.02, masked=1),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attend", "attend", "attend", "attend", "append", "norms", "sample"])
    if op in ("attend", "append"):
        dim = rng.choice([64, 128])
        group = rng.choice([1, 2, 4, 5, 8])
        kv_heads = rng.choice([1, 2, 4, 8])
        page = rng.choice([16, 32, 64, 128])
        windowed = rng.random() < 0.4
        if rng.random() < 0.5:  # tokens one by one, or a few
            batch, q_max, kv_max = _log_int(rng, 1, 64), rng.choice([1, 1, 1, 2, 5, 9]), _log_int(rng, 64, 16384)
        else:  # chunks
            batch, q_max = _log_int(rng, 1, 4), _log_int(rng, 16, 2048)
            kv_max = q_max + rng.choice([0, _log_int(rng, 1, 8192)])
        kv_max = max(kv_max, q_max)
        window = _log_int(rng, 16, 4096) if windowed and op == "attend" else 0
        return dict(op=op, batch=batch, q_max=q_max, q_ragged=rng.random() < 0.5, kv_max=kv_max,
                    kv_min=rng.randint(q_max, kv_max), heads=kv_heads * group, kv_heads=kv_heads, dim=dim, page=page,
                    window=window, sinks=rng.choice([0, 1, 4, 37]) if window else 0)
    if op == "norms":
        rows, cols = _log_int(rng, 1, 8192), _log_int(rng, 64, 8192)
        if rng.random() < 0.8:
            cols = (cols + 7) // 8 * 8
        stream = rng.choice(["bf16", "f32"])
        return dict(op=op, rows=rows, cols=cols, post=rng.choice(["none", "rms", "layer"]),
                    pre=rng.choice(["rms", "layer"]), gate_rows=rng.choice([-1, 0, 1, max(1, rows // 3)]),
                    alpha=rng.choice([1.0, 0.7071, 1.5]), stream=stream, block=rng.choice(["bf16", stream]))
    return dict(op=op, rows=_log_int(rng, 1, 128), vocab=_log_int(rng, 1000, 160000), dtype=rng.choice(["bf16", "f32"]),
                top_k=rng.choice([0, 1, 20, 50, 1000]), top_p=rng.choice([1.0, 0.8, 0.9, 0.95]),
                min_p=rng.choice([0.0, 0.0, 0.02, 0.1]), masked=rng.choice([0, 1]))


def _lengths(case):
    """New tokens and cached tokens (the new ones included) of each sequence: spread over the case's ranges."""
    b = case["batch"]
    q = [case["q_max"]] * b
    if case["q_ragged"]:
        q = [max(1, case["q_max"] - (i * 7919) % (case["q_max"] // 2 + 1)) for i in range(b)]
    lo = case["kv_min"]
    kv = [case["kv_max"] - int((case["kv_max"] - lo) * ((i * 0.6180339887) % 1.0)) for i in range(b)]
    return q, [max(k, n) for k, n in zip(kv, q)]


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


# --------------------------------------------------------------------------------------------------- the inputs
def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda")  # noqa: E731
    uniform = lambda *shape: torch.rand(*shape, generator=g, device="cuda")  # noqa: E731
    s = dict(case=case)
    if case["op"] in ("attend", "append"):
        q, kv = _lengths(case)
        tokens, page = sum(q), case["page"]
        hq, hk, d = case["heads"], case["kv_heads"], case["dim"]
        # the projection's packed output: queries, keys and values of a token side by side
        s["qkv"] = normal(tokens, (hq + 2 * hk) * d).to(torch.bfloat16)
        s["q"] = s["qkv"][:, :hq * d].unflatten(1, (hq, d))
        s["k"] = s["qkv"][:, hq * d:(hq + hk) * d].unflatten(1, (hk, d))
        s["v"] = s["qkv"][:, (hq + hk) * d:].unflatten(1, (hk, d))
        need = [(n + page - 1) // page for n in kv]
        pages, width = sum(need) + 3, max(need)
        order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32).cpu()
        table, at = torch.full((len(q), width), -1, dtype=torch.int32), 0
        for i, n in enumerate(need):
            table[i, :n] = order[at:at + n]
            at += n
        s["table"] = table.cuda()
        s["k_cache"] = normal(pages, page, hk, d).to(torch.bfloat16)
        s["v_cache"] = normal(pages, page, hk, d).to(torch.bfloat16)
        s["q_len"], s["kv_len"] = q, kv
        s["cu_q"] = torch.tensor(np.concatenate([[0], np.cumsum(q)]), dtype=torch.int32).cuda()
        s["kv_len_dev"] = torch.tensor(kv, dtype=torch.int32).cuda()
        # where each new token goes: sequence and position
        s["seq_of"] = torch.tensor(np.repeat(np.arange(len(q)), q)).cuda()
        s["pos_of"] = torch.tensor(np.concatenate([np.arange(k - n, k) for n, k in zip(q, kv)])).cuda()
    elif case["op"] == "norms":
        r, c = case["rows"], case["cols"]
        s["x"] = (normal(r, c) * 2).to(_DTYPES[case["stream"]])
        s["y"] = (normal(r, c) + 0.25).to(_DTYPES[case["block"]])
        s["gate"] = None
        if case["gate_rows"] >= 0:  # 0: one gate for all rows; n: one for every n rows
            groups = 1 if case["gate_rows"] == 0 else (r + case["gate_rows"] - 1) // case["gate_rows"]
            s["gate"] = (normal(groups, c) * 0.5).to(_DTYPES[case["block"]])
        s["post_gamma"], s["post_beta"] = uniform(c) + 0.5, normal(c) * 0.1
        s["pre_gamma"], s["pre_beta"] = uniform(c) + 0.5, normal(c) * 0.1
    else:
        r, v = case["rows"], case["vocab"]
        z = normal(r, v) * 2.5
        z[torch.arange(r, device="cuda"), torch.randint(v, (r,), generator=g, device="cuda")] += 6.0
        if case["masked"]:  # a constraint forbids a third of the tokens
            z = z.masked_fill(uniform(v) < 0.33, -math.inf)
        s["logits"] = z.to(_DTYPES[case["dtype"]])
        s["u"] = uniform(r)
        s["temperature"] = 0.6 + 0.8 * uniform(r)
        s["top_k"] = torch.full((r,), case["top_k"], dtype=torch.int32, device="cuda") if case["top_k"] else None
        s["top_p"] = torch.full((r,), case["top_p"], device="cuda") if case["top_p"] < 1.0 else None
        s["min_p"] = torch.full((r,), case["min_p"], device="cuda") if case["min_p"] > 0.0 else None
    return s


# ------------------------------------------------------------------------------------------------------ one pass
def run(state):
    return (_own if own else _plain)[state["case"]["op"]](state)


def _plain_attend(s):
    c = s["case"]
    hk, group, d = c["kv_heads"], c["heads"] // c["kv_heads"], c["dim"]
    out = torch.empty(s["q"].shape, dtype=torch.bfloat16, device="cuda")
    at = 0
    for i, (n, length) in enumerate(zip(s["q_len"], s["kv_len"])):
        pages = s["table"][i, :(length + c["page"] - 1) // c["page"]].long()
        k = s["k_cache"][pages].flatten(0, 1)[:length].permute(1, 0, 2).float()             # [hk, length, d]
        v = s["v_cache"][pages].flatten(0, 1)[:length].permute(1, 0, 2).float()
        q = s["q"][at:at + n].unflatten(1, (hk, group)).permute(1, 2, 0, 3).float()         # [hk, group, n, d]
        scores = torch.matmul(q.flatten(1, 2), k.transpose(1, 2)).unflatten(1, (group, n)) / math.sqrt(d)
        pos = torch.arange(length - n, length, device="cuda")[:, None]
        key = torch.arange(length, device="cuda")[None, :]
        seen = key <= pos
        if c["window"]:
            seen &= (key > pos - c["window"]) | (key < c["sinks"])
        scores.masked_fill_(~seen, -math.inf)
        p = torch.exp(scores - scores.amax(-1, keepdim=True))
        del scores
        total = p.sum(-1, keepdim=True)
        o = torch.matmul(p.flatten(1, 2), v).unflatten(1, (group, n)) / total
        out[at:at + n] = o.permute(2, 0, 1, 3).flatten(1, 2).to(torch.bfloat16)
        at += n
    return out


def _plain_append(s):
    page = s["case"]["page"]
    where = s["table"][s["seq_of"], s["pos_of"] // page].long()
    s["k_cache"][where, s["pos_of"] % page] = s["k"]
    s["v_cache"][where, s["pos_of"] % page] = s["v"]
    return s["k_cache"], s["v_cache"]


_EPS = 1e-5


def _plain_norm(kind, x, gamma, beta):
    if kind == "none":
        return x
    if kind == "rms":
        return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + _EPS) * gamma
    x = x - x.mean(-1, keepdim=True)
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + _EPS) * gamma + beta


def _plain_norms(s):
    c = s["case"]
    y = _plain_norm(c["post"], s["y"].float(), s["post_gamma"], s["post_beta"])
    if s["gate"] is not None:
        every = c["gate_rows"] or c["rows"]
        y = y * s["gate"].float()[torch.arange(c["rows"], device="cuda") // every]
    h = c["alpha"] * s["x"].float() + y
    n = _plain_norm(c["pre"], h, s["pre_gamma"], s["pre_beta"])
    return h.to(s["x"].dtype), n.to(s["y"].dtype)


def _plain_sample(s):
    # in 64 bits: a token is kept or not, and drawn or not, by comparisons of long sums
    z = s["logits"].double() / s["temperature"].double()[:, None]
    vocab = z.shape[1]
    mass = torch.exp(z - z.amax(-1, keepdim=True))
    _, order = torch.sort(s["logits"].float(), dim=-1, descending=True, stable=True)
    ranked = mass.gather(-1, order)
    if s["top_k"] is not None:
        ranked = ranked * (torch.arange(vocab, device="cuda")[None, :] < s["top_k"][:, None])
    keep = ranked > 0
    if s["top_p"] is not None:
        total = ranked.sum(-1, keepdim=True)
        before = ranked.cumsum(-1) - ranked
        keep &= before < s["top_p"].double()[:, None] * total
        keep[:, 0] = True
    if s["min_p"] is not None:
        keep &= ranked >= s["min_p"].double()[:, None]
    kept = torch.zeros_like(mass).scatter_(-1, order, ranked * keep)
    cum = kept.cumsum(-1)
    total = cum[:, -1:]
    token = (cum <= s["u"].double()[:, None] * total).sum(-1, keepdim=True).clamp_(max=vocab - 1)
    prob = kept.gather(-1, token) / total
    return token[:, 0].to(torch.int32), prob[:, 0].float()


def _own_attend(s):
    from paper_2511_03586_b200 import api
    c = s["case"]
    return api.pd_attention_paged_fwd(s["q"], s["k_cache"], s["v_cache"], s["table"], s["cu_q"], s["kv_len_dev"],
                                      max_q_len=c["q_max"], max_kv_len=c["kv_max"], window=c["window"],
                                      sinks=c["sinks"])


def _own_append(s):
    from paper_2511_03586_b200 import api
    api.pd_kv_cache_append(s["k"], s["v"], s["k_cache"], s["v_cache"], s["table"], s["cu_q"], s["kv_len_dev"])
    return s["k_cache"], s["v_cache"]


def _own_norms(s):
    from paper_2511_03586_b200 import api
    c = s["case"]
    beta = lambda which: s[which + "_beta"] if c[which] == "layer" else None  # noqa: E731
    return api.pd_norm_gate_residual_norm(
        s["y"], s["x"], gate=s["gate"], gate_rows=c["gate_rows"] or c["rows"], alpha=c["alpha"], eps=_EPS,
        post_norm=c["post"], post_gamma=None if c["post"] == "none" else s["post_gamma"], post_beta=beta("post"),
        pre_norm=c["pre"], pre_gamma=s["pre_gamma"], pre_beta=beta("pre"))


def _own_sample(s):
    from paper_2511_03586_b200 import api
    return api.pd_sample(s["logits"], s["u"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"],
                         min_p=s["min_p"])


_plain = {"attend": _plain_attend, "append": _plain_append, "norms": _plain_norms, "sample": _plain_sample}
_own = {"attend": _own_attend, "append": _own_append, "norms": _own_norms, "sample": _own_sample}


# ------------------------------------------------------------------------------------------------ the least work
def work(case):
    if case["op"] in ("attend", "append"):
        q, kv = _lengths(case)
        hq, hk, d = case["heads"], case["kv_heads"], case["dim"]
        if case["op"] == "append":
            return {"bytes": 2 * 2 * 2 * sum(q) * hk * d + 4 * sum(q), "flops": 0}
        pairs, keys = zip(*(_pairs(case, n, k) for n, k in zip(q, kv)))
        return {"bytes": 2 * 2 * sum(q) * hq * d + 2 * 2 * sum(keys) * hk * d + 4 * sum(keys) // case["page"],
                "flops": 4 * sum(pairs) * hq * d}
    if case["op"] == "norms":
        r, c = case["rows"], case["cols"]
        wide = {"bf16": 2, "f32": 4}
        b, x = wide[case["block"]], wide[case["stream"]]
        gates = 0 if case["gate_rows"] < 0 else 1 if case["gate_rows"] == 0 else -(-r // case["gate_rows"])
        return {"bytes": r * c * (2 * b + 2 * x) + gates * c * b + 4 * 4 * c, "flops": 16 * r * c}
    return {"bytes": case["rows"] * case["vocab"] * (2 if case["dtype"] == "bf16" else 4) + 28 * case["rows"],
            "flops": 4 * case["rows"] * case["vocab"]}


# ---------------------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    if case["op"] == "append":
        return None  # copies: no computed numbers
    s = prepare(case, seed)
    if case["op"] == "attend":
        return _exact_attend(case, s)
    if case["op"] == "norms":
        return _exact_norms(case, s)
    return _exact_sample(case, s)


def _exact_attend(case, s):
    """One head and up to 512 queries at a time; a key outside a query's view is left out of its sums by a zero
    weight, and every weight is taken relative to the log of the visible ones' sum."""
    hk, group, d = case["kv_heads"], case["heads"] // case["kv_heads"], case["dim"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    start = 0
    for i, (n, length) in enumerate(zip(s["q_len"], s["kv_len"])):
        index = torch.arange(length, device="cuda")
        page, slot = s["table"][i].long()[index // case["page"]], index % case["page"]
        for h in range(hk):
            k, v = s["k_cache"][page, slot, h].double(), s["v_cache"][page, slot, h].double()
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


def _exact_norms(case, s):
    def normed(kind, t, gamma, beta):
        if kind == "none":
            return t
        if kind == "rms":
            return gamma.double() * t / torch.sqrt(torch.linalg.vector_norm(t, dim=-1, keepdim=True) ** 2 / t.shape[1] + _EPS)
        var, mean = torch.var_mean(t, dim=-1, correction=0, keepdim=True)
        return beta.double() + gamma.double() * (t - mean) / torch.sqrt(var + _EPS)
    block = normed(case["post"], s["y"].double(), s["post_gamma"], s["post_beta"])
    if s["gate"] is not None:
        every = case["gate_rows"] or case["rows"]
        block = block * s["gate"].double().repeat_interleave(every, 0)[:case["rows"]]
    h = block + s["x"].double() * case["alpha"]
    return h, normed(case["pre"], h, s["pre_gamma"], s["pre_beta"])


def _exact_sample(case, s):
    """Row by row on the host: tokens ranked by value and then by index, the filters taken one after the other."""
    logits, u = s["logits"].double().cpu().numpy(), s["u"].double().cpu().numpy()
    temperature = s["temperature"].double().cpu().numpy()
    column = lambda t, none: [none] * len(u) if t is None else t.double().cpu().tolist()  # noqa: E731
    ks, ps, ms = column(s["top_k"], 0), column(s["top_p"], 1.0), column(s["min_p"], 0.0)
    tokens, probs = [], []
    for row, (x, t) in enumerate(zip(logits, temperature)):
        z = x / t
        mass = np.exp(z - z.max())
        rank = np.argsort(-x, kind="stable")
        if ks[row]:
            rank = rank[:int(ks[row])]
        if ps[row] < 1.0:
            reach = np.cumsum(mass[rank])
            rank = rank[:1 + int(np.searchsorted(reach, ps[row] * mass[rank].sum(), side="left"))]
        rank = np.sort(rank[(mass[rank] >= ms[row]) & (mass[rank] > 0)])
        reach = np.cumsum(mass[rank])
        at = min(int(np.searchsorted(reach, u[row] * reach[-1], side="right")), len(rank) - 1)
        tokens.append(int(rank[at]))
        probs.append(mass[rank[at]] / reach[-1])
    return (torch.tensor(tokens, dtype=torch.int32, device="cuda"),
            torch.tensor(probs, dtype=torch.float64, device="cuda"))
