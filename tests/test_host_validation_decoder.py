"""Argument checking of the decoder entry points (paged cache, norms between blocks, sampling), without a GPU: what the
library turns away, or accepts as empty, before it looks at the device.  The pointers are made-up addresses; none of
these calls may reach a kernel."""
import ctypes

import pytest

from paper_2511_03586_b200 import build

build.build()  # the binding loads the library when it is imported

from paper_2511_03586_b200 import api  # noqa: E402
from paper_2511_03586_b200.api import NormGateResidualDesc, PagedAttentionDesc  # noqa: E402

OK, NULLP, SHAPE, UNSUP, ALIGN, WS_SMALL = 0, 1, 2, 3, 4, 5
P = 0x10000
lib = api._lib


def paged(**kw):
    d = dict(batch=2, tokens=2, heads_q=8, heads_kv=2, head_dim=64, num_pages=16, page_size=16, max_pages=8, max_q_len=1,
             max_kv_len=128, window=0, sinks=0, scale=0.125, ld_q=512, ld_out=512, page_stride=2048, slot_stride=128,
             head_stride=64)
    d.update(kw)
    return PagedAttentionDesc(**d)


def attend(q=P, k=P, v=P, table=P, cu=P, lens=P, out=P, ws=P, ws_bytes=1 << 40, **kw):
    return lib.pd_attention_paged_fwd(ctypes.byref(paged(**kw)), q, k, v, table, cu, lens, out, ws, ws_bytes, None)


def append(k=P, v=P, ld=128, kc=P, vc=P, table=P, cu=P, lens=P, **kw):
    return lib.pd_kv_cache_append(ctypes.byref(paged(**kw)), k, v, ld, kc, vc, table, cu, lens, None)


def test_attention_refusals():
    assert lib.pd_attention_paged_fwd(None, P, P, P, P, P, P, P, P, 0, None) == NULLP
    for name in ("q", "k", "v", "table", "cu", "lens", "out"):
        assert attend(**{name: None}) == NULLP
    for kw in (dict(batch=-1), dict(tokens=-1), dict(heads_q=0), dict(heads_kv=0), dict(heads_q=7), dict(head_dim=0),
               dict(num_pages=0), dict(page_size=0), dict(max_pages=0), dict(max_q_len=-1), dict(max_kv_len=-1),
               dict(window=-1), dict(sinks=-1), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")),
               dict(scale=float("inf")), dict(ld_q=504), dict(ld_out=504), dict(page_stride=0), dict(slot_stride=-8),
               dict(head_stride=0)):
        assert attend(**kw) == SHAPE, kw
    for kw in (dict(head_dim=32), dict(head_dim=96), dict(head_dim=256), dict(page_size=24), dict(page_size=4),
               dict(page_size=8192), dict(heads_q=130), dict(batch=65536), dict(max_pages=1 << 28)):
        kw.setdefault("ld_q", 1 << 20), kw.setdefault("ld_out", 1 << 20)
        assert attend(**kw) == UNSUP, kw
    for kw in (dict(q=P + 8), dict(k=P + 2), dict(v=P + 8), dict(out=P + 4), dict(table=P + 2), dict(cu=P + 1),
               dict(lens=P + 2), dict(ld_q=516), dict(ld_out=516), dict(page_stride=2052), dict(slot_stride=132),
               dict(head_stride=68)):
        assert attend(**kw) == ALIGN, kw
    for kw in (dict(batch=0), dict(tokens=0), dict(max_q_len=0)):
        assert attend(**kw) == OK, kw


def test_attention_workspace():
    long = dict(max_kv_len=8192, max_pages=512)
    need = lib.pd_attention_paged_workspace_bytes(ctypes.byref(paged(**long)))
    assert need > 0
    assert attend(ws=None, **long) == NULLP
    assert attend(ws_bytes=need - 1, **long) == WS_SMALL
    assert attend(ws=P + 128, **long) == ALIGN
    assert lib.pd_attention_paged_workspace_bytes(None) == 0
    assert lib.pd_attention_paged_workspace_bytes(ctypes.byref(paged(head_dim=32, **long))) == 0
    assert lib.pd_attention_paged_workspace_bytes(ctypes.byref(paged(heads_q=7, **long))) == 0
    assert lib.pd_attention_paged_workspace_bytes(ctypes.byref(paged(batch=0, **long))) == 0
    # a window bounds the keys a token reads, and with them the splits
    windowed = lib.pd_attention_paged_workspace_bytes(ctypes.byref(paged(window=64, **long)))
    assert windowed < need


def test_append_refusals():
    assert lib.pd_kv_cache_append(None, P, P, 128, P, P, P, P, P, None) == NULLP
    for name in ("k", "v", "kc", "vc", "table", "cu", "lens"):
        assert append(**{name: None}) == NULLP
    for kw in (dict(batch=-1), dict(tokens=-1), dict(heads_kv=0), dict(head_dim=0), dict(num_pages=0),
               dict(page_size=0), dict(max_pages=0), dict(ld=120), dict(page_stride=0), dict(slot_stride=0),
               dict(head_stride=0)):
        assert append(**kw) == SHAPE, kw
    assert append(head_dim=60) == UNSUP
    assert append(head_dim=1032, ld=1 << 20) == UNSUP
    for kw in (dict(k=P + 8), dict(v=P + 2), dict(kc=P + 8), dict(vc=P + 8), dict(table=P + 2), dict(cu=P + 2),
               dict(lens=P + 1), dict(ld=132), dict(page_stride=2052), dict(slot_stride=132), dict(head_stride=68)):
        assert append(**kw) == ALIGN, kw
    assert append(batch=0) == OK
    assert append(tokens=0) == OK


def norms(y=P, x=P, gate=P, vec=(P, P, P, P), h=P, n=P, **kw):
    d = dict(rows=4, cols=64, gate_rows=1, x_dtype=0, y_dtype=0, post_norm=1, pre_norm=2, alpha=1.0, eps=1e-5)
    d.update(kw)
    return lib.pd_norm_gate_residual_norm(ctypes.byref(NormGateResidualDesc(**d)), y, x, gate, *vec, h, n, None)


def test_norm_refusals():
    assert lib.pd_norm_gate_residual_norm(None, P, P, P, P, P, P, P, P, P, None) == NULLP
    assert norms(y=None) == NULLP
    assert norms(x=None) == NULLP
    assert norms(h=None, n=None) == NULLP
    for kw in (dict(rows=-1), dict(cols=0), dict(cols=1 << 31), dict(eps=-1.0), dict(eps=float("nan")),
               dict(alpha=float("nan")), dict(gate_rows=0), dict(x_dtype=2), dict(y_dtype=-1), dict(post_norm=3),
               dict(pre_norm=-1)):
        assert norms(**kw) == SHAPE, kw
    for kw in (dict(y=P + 1), dict(x=P + 2, x_dtype=1), dict(gate=P + 1), dict(h=P + 2, x_dtype=1), dict(n=P + 1),
               dict(vec=(P + 2, P, P, P)), dict(vec=(P, P, P, P + 1))):
        assert norms(**kw) == ALIGN, kw
    assert norms(rows=0) == OK
    assert norms(rows=0, gate=None, gate_rows=0, vec=(None,) * 4) == OK   # gate and vectors are optional


def sample(logits=P, dtype=1, rows=4, vocab=100, ld=100, t=P, k=P, p=P, m=P, u=P, tokens=P, probs=P):
    return lib.pd_sample(logits, dtype, rows, vocab, ld, t, k, p, m, u, tokens, probs, None)


def test_sample_refusals():
    for name in ("logits", "u", "tokens"):
        assert sample(**{name: None}) == NULLP
    for kw in (dict(rows=-1), dict(vocab=0, ld=8), dict(ld=99), dict(dtype=2)):
        assert sample(**kw) == SHAPE, kw
    assert sample(vocab=327681, ld=327681) == UNSUP
    assert sample(rows=1 << 30) == UNSUP
    for kw in (dict(logits=P + 2), dict(logits=P + 1, dtype=0), dict(t=P + 2), dict(k=P + 2), dict(p=P + 1),
               dict(m=P + 2), dict(u=P + 2), dict(tokens=P + 2), dict(probs=P + 2)):
        assert sample(**kw) == ALIGN, kw
    assert sample(rows=0) == OK


def test_binding_wants_cuda_tensors():
    import torch
    t = torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        api.pd_attention_paged_fwd(t, t, t, t, t, t, max_q_len=1, max_kv_len=1)
    with pytest.raises(TypeError):
        api.pd_kv_cache_append(t, t, t, t, t, t, t)
    with pytest.raises(TypeError):
        api.pd_norm_gate_residual_norm(t[0], t[0])
    with pytest.raises(TypeError):
        api.pd_sample(t[0], t[0])


def test_extents_beyond_the_kernels_index_types():
    many = dict(batch=1, tokens=(1 << 24), heads_kv=128, heads_q=128, head_dim=64, ld_q=1 << 20, ld_out=1 << 20)
    assert attend(**many) == UNSUP                       # tokens * heads_q = 2^31: the joining kernel's grid
    assert lib.pd_attention_paged_workspace_bytes(ctypes.byref(paged(**many))) == 0
    assert append(tokens=(1 << 30) + 1) == UNSUP
    assert append(batch=(1 << 30) + 1) == UNSUP
