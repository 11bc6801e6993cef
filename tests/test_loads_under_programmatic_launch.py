"""The kernels around the paged caches are launched before the ones in front of them have ended, and wait for these by
griddepcontrol.wait.  What such a kernel writes (queries, the caches, their scales) is then written during the lifetime of the
kernel that reads it, where the non-coherent path (ld.global.nc, __ldg) may not be used; that path is for what no kernel of the
library writes: tables, lengths, frequencies, masks.  Whether a stale line is met is a matter of timing, so the source is checked."""
import os
import re

import pytest

from test_cluster_start import CSRC

WRITTEN_BY_NONE = re.compile(r"\bblock_table\b|\bcu_q\b|\bcu\b|\bkv_len\b|\binv_freq\b|\bmask\b")


@pytest.mark.parametrize("file", ["paged_rows_q8.cuh", "paged_rows.cuh", "paged_attention_rows.cu", "paged_attention_tcgen05.cu", "paged_cache.cuh", "paged_join.cuh",
                                  "cache_q8.cuh", "rope_kv_cache_append.cu", "kv_cache_append.cu", "penalize_logits.cu"])
def test_what_a_kernel_in_front_may_write_is_read_coherently(file):
    with open(os.path.join(CSRC, file)) as f:
        text = re.sub(r"//[^\n]*", "", f.read())
    assert not re.search(r"\.nc\b", text)
    for m in re.finditer(r"__ldg\(", text):
        depth, i = 1, m.end()
        while depth:
            depth += {"(": 1, ")": -1}.get(text[i], 0)
            i += 1
        assert WRITTEN_BY_NONE.search(text[m.end():i]), text[m.start():i]
