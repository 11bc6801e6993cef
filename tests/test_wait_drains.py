"""A CTA of the paged attention kernels ends with no copy and no product in flight, whichever of its warps gives up a bounded wait:
the warps that request them wait for their last ones on every way out, not only when they have given up themselves.

A copy that lands in the memory of a CTA that is gone is not something to be tried out, so the source is checked."""
import re

import pytest

from test_cluster_start import kernel_body

DRAIN = re.compile(r"&never\b")


def enclosing_conditions(body, at):
    """The texts in front of the braces that enclose position `at`."""
    depth, found = 0, []
    for i in range(at, -1, -1):
        if body[i] == "}":
            depth += 1
        elif body[i] == "{":
            if depth == 0:
                found.append(body[max(body.rfind(c, 0, i) for c in ";{}") + 1:i].strip())
            else:
                depth -= 1
    return found


@pytest.mark.parametrize("file,name,drains", [("paged_attention_rows.cu", "paged_attention_rows_kernel", 1),
                                              ("paged_attention_tcgen05.cu", "paged_attention_chunk_kernel", 2),
                                              ("paged_attention_tcgen05.cu", "paged_attention_chunk_narrow_kernel", 2)])
def test_last_requests_are_waited_for_on_every_way_out(file, name, drains):
    body = kernel_body(file, name)
    found = [enclosing_conditions(body, m.start()) for m in DRAIN.finditer(body)]
    assert len(found) == drains
    for conditions in found:
        assert not any("ok" in c for c in conditions), conditions
