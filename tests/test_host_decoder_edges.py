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
