"""Argument checking of the rotating append, the attention over 8-bit caches and the changes to logits, without a GPU: what the
library turns away, or accepts as empty, before it looks at the device.  The pointers are made-up addresses; none of these calls
may reach a kernel."""
import ctypes

import pytest

from paper_2511_03586_b200 import build

build.build()  # the binding loads the library when it is imported

from paper_2511_03586_b200 import api  # noqa: E402
from paper_2511_03586_b200.api import CacheScales, PenalizeDesc, RopeDesc  # noqa: E402
from test_host_validation_decoder import ALIGN, NULLP, OK, P, SHAPE, UNSUP, WS_SMALL, lib, paged  # noqa: E402

I8, E4 = api.PD_I8, api.PD_E4M3


def q8(dtype=I8, block=16, ks=P, vs=P):
    return ctypes.byref(CacheScales(dtype, block, ks, vs))


def rope(rotary=64, interleaved=0, amplitude=1.0, freq=P):
    return ctypes.byref(RopeDesc(rotary, interleaved, amplitude, freq))


def append(scales=None, r=None, q=P, q_out=P, k=P, v=P, ld=128, kc=P, vc=P, table=P, cu=P, lens=P, **kw):
    return lib.pd_rope_kv_cache_append(ctypes.byref(paged(**kw)), rope() if r is None else r, scales, q, q_out, k, v, ld, kc, vc, table, cu,
                                       lens, None)


@pytest.mark.parametrize("scales", [None, q8(), q8(E4, 8)], ids=["bf16", "int8", "e4m3"])
def test_append_refusals(scales):
    assert lib.pd_rope_kv_cache_append(None, rope(), scales, P, P, P, P, 128, P, P, P, P, P, None) == NULLP
    assert lib.pd_rope_kv_cache_append(ctypes.byref(paged()), None, scales, P, P, P, P, 128, P, P, P, P, P, None) == NULLP
    for name in ("q", "q_out", "k", "v", "kc", "vc", "table", "cu", "lens"):
        assert append(scales, **{name: None}) == NULLP, name
    assert append(scales, rope(freq=None)) == NULLP
    for kw in (dict(batch=-1), dict(tokens=-1), dict(heads_kv=0), dict(head_dim=0), dict(num_pages=0), dict(page_size=0),
               dict(max_pages=0), dict(heads_q=0), dict(ld=120), dict(ld_q=504), dict(ld_out=504), dict(page_stride=0),
               dict(slot_stride=-16), dict(head_stride=0)):
        assert append(scales, **kw) == SHAPE, kw
    for kw in (dict(rotary=-8), dict(rotary=72), dict(interleaved=2), dict(amplitude=float("nan")), dict(amplitude=float("inf"))):
        assert append(scales, rope(**kw)) == SHAPE, kw
    for kw in (dict(head_dim=68, ld=1 << 20, ld_q=1 << 20, ld_out=1 << 20), dict(head_dim=264, ld=1 << 20, ld_q=1 << 20, ld_out=1 << 20),
               dict(batch=65536), dict(tokens=(1 << 30) + 1), dict(heads_kv=65537, ld=1 << 30)):
        assert append(scales, **kw) == UNSUP, kw
    assert append(scales, rope(rotary=20)) == UNSUP
    for kw in (dict(q=P + 8), dict(q_out=P + 2), dict(k=P + 8), dict(v=P + 2), dict(kc=P + 8), dict(vc=P + 8), dict(table=P + 2),
               dict(cu=P + 2), dict(lens=P + 1), dict(ld=132), dict(ld_q=516), dict(ld_out=516), dict(page_stride=2052),
               dict(slot_stride=132), dict(head_stride=68)):
        assert append(scales, **kw) == ALIGN, kw
    assert append(scales, rope(freq=P + 2)) == ALIGN
    assert append(scales, batch=0) == OK
    assert append(scales, tokens=0) == OK


def test_append_refuses_scales():
    for dtype, block in ((0, 16), (1, 16), (4, 16), (I8, 0), (I8, -1), (I8, 3), (I8, 32), (E4, 12)):
        assert append(q8(dtype, block)) == SHAPE, (dtype, block)
    assert append(q8(ks=None)) == NULLP
    assert append(q8(vs=None)) == NULLP
    assert append(q8(ks=P + 2)) == ALIGN
    assert append(q8(vs=P + 1)) == ALIGN
    assert append(q8(), slot_stride=136) == ALIGN      # 8 elements are enough for a bf16 cache only
    assert append(q8(block=1), tokens=1 << 30, heads_kv=128, ld=1 << 20) == UNSUP   # more CTAs than a grid has


def attend(scales=None, q=P, k=P, v=P, table=P, cu=P, lens=P, out=P, ws=P, ws_bytes=1 << 40, **kw):
    return lib.pd_attention_paged_q8_fwd(ctypes.byref(paged(**kw)), scales or q8(), q, k, v, table, cu, lens, out, ws, ws_bytes, None)


def test_attention_refusals():
    assert lib.pd_attention_paged_q8_fwd(None, q8(), P, P, P, P, P, P, P, P, 0, None) == NULLP
    assert lib.pd_attention_paged_q8_fwd(ctypes.byref(paged()), None, P, P, P, P, P, P, P, P, 0, None) == NULLP
    for name in ("q", "k", "v", "table", "cu", "lens", "out"):
        assert attend(**{name: None}) == NULLP
    for kw in (dict(batch=-1), dict(tokens=-1), dict(heads_q=0), dict(heads_kv=0), dict(heads_q=7), dict(head_dim=0),
               dict(num_pages=0), dict(page_size=0), dict(max_pages=0), dict(max_q_len=-1), dict(max_kv_len=-1),
               dict(window=-1), dict(sinks=-1), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")),
               dict(scale=float("inf")), dict(ld_q=504), dict(ld_out=504), dict(page_stride=0), dict(slot_stride=-16),
               dict(head_stride=0)):
        assert attend(**kw) == SHAPE, kw
    for dtype, block in ((0, 16), (1, 16), (5, 16), (I8, 0), (I8, 5), (E4, 64)):
        assert attend(q8(dtype, block)) == SHAPE, (dtype, block)
    assert attend(q8(ks=None)) == NULLP
    assert attend(q8(vs=None)) == NULLP
    for kw in (dict(head_dim=32), dict(head_dim=96), dict(head_dim=256), dict(page_size=48), dict(page_size=8192, max_pages=1),
               dict(heads_q=130), dict(batch=65536), dict(max_pages=1 << 28)):
        kw.setdefault("ld_q", 1 << 20), kw.setdefault("ld_out", 1 << 20)
        assert attend(**kw) == UNSUP, kw
    assert attend(q8(block=4), page_size=4) == UNSUP
    for kw in (dict(q=P + 8), dict(k=P + 2), dict(v=P + 8), dict(out=P + 4), dict(table=P + 2), dict(cu=P + 1),
               dict(lens=P + 2), dict(ld_q=516), dict(ld_out=516), dict(page_stride=2056), dict(slot_stride=136),
               dict(head_stride=72)):
        assert attend(**kw) == ALIGN, kw
    assert attend(q8(ks=P + 2)) == ALIGN
    assert attend(q8(vs=P + 3)) == ALIGN
    for kw in (dict(batch=0), dict(tokens=0), dict(max_q_len=0)):
        assert attend(**kw) == OK, kw


def test_attention_workspace():
    need = lambda **kw: lib.pd_attention_paged_q8_workspace_bytes(ctypes.byref(paged(**kw)))  # noqa: E731
    long = dict(max_kv_len=8192, max_pages=512)
    if need(**long) > 0:
        assert attend(ws=None, **long) == NULLP
        assert attend(ws_bytes=need(**long) - 1, **long) == WS_SMALL
        assert attend(ws=P + 128, **long) == ALIGN
    assert lib.pd_attention_paged_q8_workspace_bytes(None) == 0
    for kw in (dict(head_dim=32), dict(heads_q=7), dict(batch=0), dict(tokens=0), dict(page_size=24)):
        assert need(**{**long, **kw}) == 0


def penalise(logits=P, out=P, history=P, hl=P, pl=P, r=P, f=P, g=P, bt=P, bv=P, mask=P, mr=P, **kw):
    d = dict(rows=4, vocab=100, ld_logits=100, ld_out=100, dtype=1, out_dtype=1, history_cols=10, ld_history=10, bias_cols=3, mask_rows=4, ld_mask=4)
    d.update(kw)
    return lib.pd_penalize_logits(ctypes.byref(PenalizeDesc(**d)), logits, out, history, hl, pl, r, f, g, bt, bv, mask, mr, None)


def test_penalise_refusals():
    assert lib.pd_penalize_logits(None, *[P] * 12, None) == NULLP
    for name in ("logits", "out", "bt", "bv"):
        assert penalise(**{name: None}) == NULLP, name
    for kw in (dict(rows=-1), dict(vocab=0), dict(ld_logits=99), dict(ld_out=99), dict(dtype=2), dict(out_dtype=3), dict(history_cols=-1),
               dict(bias_cols=-1), dict(mask_rows=-1), dict(ld_history=9), dict(ld_mask=3), dict(mr=None, mask_rows=3)):
        assert penalise(**kw) == SHAPE, kw
    for kw in (dict(vocab=(1 << 24) + 1, ld_logits=1 << 25, ld_out=1 << 25, ld_mask=1 << 20), dict(rows=1 << 31),
               dict(history_cols=1 << 20, ld_history=1 << 20), dict(bias_cols=2048)):
        assert penalise(**kw) == UNSUP, kw
    for kw in (dict(logits=P + 2), dict(out=P + 2), dict(logits=P + 1, dtype=0), dict(out=P + 1, out_dtype=0), dict(history=P + 2), dict(hl=P + 2),
               dict(pl=P + 1), dict(r=P + 2), dict(f=P + 2), dict(g=P + 2), dict(bt=P + 2), dict(bv=P + 2), dict(mask=P + 2), dict(mr=P + 2)):
        assert penalise(**kw) == ALIGN, kw
    assert penalise(rows=0) == OK


def test_binding_wants_cuda_tensors():
    import torch
    t, c = torch.zeros(2, 4, 64, dtype=torch.bfloat16), torch.zeros(2, 16, 4, 64, dtype=torch.int8)
    with pytest.raises(TypeError):
        api.pd_rope_kv_cache_append(t, t, t, t, t, t, t)
    with pytest.raises(TypeError):
        api.pd_attention_paged_q8_fwd(t, c, c, t, t, t, t, t, max_q_len=1, max_kv_len=1)
    with pytest.raises(TypeError):
        api.pd_penalize_logits(t[0])


@pytest.mark.parametrize("batch,max_pages,tiles,ok", [
    (64, 1 << 16, 1 << 26, True),
    (64, (1 << 16) + 1, (1 << 26) + 1024, True),      # 64 * 8 heads * 2 tiles of 32 keys a page more
    (1024, 1 << 16, 1 << 30, True),
    (1024, (1 << 16) + 1, (1 << 30) + 16384, False),
])
def test_extents_beyond_the_kernels_index_types(batch, max_pages, tiles, ok):
    kw = dict(batch=batch, heads_kv=8, max_pages=max_pages, page_size=64)
    assert batch * 8 * max_pages * 64 // 32 == tiles and (tiles <= 1 << 30) == ok
    assert (lib.pd_attention_paged_q8_workspace_bytes(ctypes.byref(paged(**kw))) > 0) == ok
    if not ok:
        assert attend(**kw) == UNSUP
