"""The same as for the kernels over bf16 caches: a CTA of the row kernel over an 8-bit cache ends with no copy in flight, whichever of its
warps gives up a bounded wait; the chunk kernel's converters of an 8-bit cache, which load without asynchronous copies, request none."""
import re

from test_cluster_start import kernel_body
from test_wait_drains import DRAIN, enclosing_conditions


def test_last_requests_are_waited_for_on_every_way_out():
    body = kernel_body("paged_rows_q8.cuh", "paged_attention_q8_rows_kernel")
    found = [enclosing_conditions(body, m.start()) for m in DRAIN.finditer(body)]
    assert len(found) == 1
    for conditions in found:
        assert not any("ok" in c for c in conditions), conditions


def test_converters_make_no_asynchronous_copies():
    import os
    from test_cluster_start import CSRC
    with open(os.path.join(CSRC, "paged_attention_tcgen05.cu")) as f:
        text = f.read()
    start = text.index("void convert_tiles(")
    body = text[start:text.index("\n}\n", start)]
    assert not re.search(r"tma_load|cp\.async|copy_async", body)
