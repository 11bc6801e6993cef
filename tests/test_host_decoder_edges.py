"""Edges of the decoder entry points that need no GPU: empty batches as the binding hands them over, sizes that follow from a
desc.  The pointers are made-up addresses or null; none of these calls may reach a kernel."""
import ctypes

from paper_2511_03586_b200 import build

build.build()  # the binding loads the library when it is imported

from paper_2511_03586_b200 import api  # noqa: E402
from paper_2511_03586_b200.api import NormGateResidualDesc, PagedAttentionDesc  # noqa: E402

OK, NULLP, SHAPE, UNSUP, ALIGN, WS_SMALL = 0, 1, 2, 3, 4, 5
P = 0x10000
lib = api._lib


def test_empty_norms_have_null_pointers():
    """The data pointer of a tensor without elements is null."""
    d = dict(rows=0, cols=64, gate_rows=1, x_dtype=0, y_dtype=0, post_norm=1, pre_norm=2, alpha=1.0, eps=1e-5)
    nulls = (None,) * 9
    assert lib.pd_norm_gate_residual_norm(ctypes.byref(NormGateResidualDesc(**d)), *nulls, None) == OK
    for bad in (dict(cols=0), dict(eps=-1.0), dict(x_dtype=2), dict(pre_norm=3)):   # still looked at
        assert lib.pd_norm_gate_residual_norm(ctypes.byref(NormGateResidualDesc(**{**d, **bad})), *nulls, None) == SHAPE
    d["rows"] = 1
    assert lib.pd_norm_gate_residual_norm(ctypes.byref(NormGateResidualDesc(**d)), *nulls, None) == NULLP


def paged(**kw):
    d = dict(batch=1, tokens=128, heads_q=32, heads_kv=8, head_dim=128, num_pages=8192, page_size=16, max_pages=8192,
             max_q_len=128, max_kv_len=131072, window=0, sinks=0, scale=0.125, ld_q=4096, ld_out=4096, page_stride=16384,
             slot_stride=1024, head_stride=128)
    d.update(kw)
    return PagedAttentionDesc(**d)


def test_workspace_does_not_grow_with_padding():
    """Partial results belong to tokens: at most max_q_len for each sequence, however long the token tensors are."""
    def need(**kw):
        return lib.pd_attention_paged_workspace_bytes(ctypes.byref(paged(**kw)))
    full = need()
    assert 0 < full < 32 << 20                              # (about 148 tiles of 256 rows, 129 floats each, at most)
    for tokens in (129, 65536, 1 << 20):
        assert need(tokens=tokens) == full
    for d in (64, 128):
        assert need(batch=3, max_q_len=40, tokens=65536, head_dim=d) == need(batch=3, max_q_len=40, tokens=120, head_dim=d)
    assert need(batch=3, max_q_len=128, tokens=200) <= need(batch=3, max_q_len=128, tokens=384)


def test_scale_is_finite_in_powers_of_two_as_well():
    """The kernels compute with scale * log2 e: infinite, it would make NaN of a score of zero."""
    def need(scale):
        return lib.pd_attention_paged_workspace_bytes(ctypes.byref(paged(scale=scale)))
    assert need(2.0 ** 127) == need(0.125) > 0
    d = paged(scale=3e38)
    assert need(3e38) == 0
    assert lib.pd_attention_paged_fwd(ctypes.byref(d), *(None,) * 8, 0, None) == SHAPE   # (no pointer, so it cannot run either way)
