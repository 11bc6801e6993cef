"""Distributed shared memory is accessed only once every CTA of the cluster is known to run: in each kernel that reads or
writes another CTA's shared memory, a cluster barrier is completed in front of the first such access.

Whether a CTA has started when its neighbour writes to it is a matter of timing that no run can be relied on to show, so the
order is checked in the source."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2511_03586_b200", "csrc")
BARRIER = re.compile(r"\bcluster_started_wait\(\)|\bcluster_sync_all\(\)|\bcluster\.sync\(\)")
REMOTE = re.compile(r"\bmap_shared_rank\(|\bcluster_allreduce\w*(?:<\w+>)?\(|\bst_cluster_\w+\(|\bst_async_\w+\(|"
                    r"\bmbar_arrive_cluster\w*\(|\bsum_histograms\(|\bsum_bins\(|\bslow_path<")


def kernel_body(file, name):
    with open(os.path.join(CSRC, file)) as f:
        text = re.sub(r"//[^\n]*", "", f.read())
    at = re.search(r"__global__[^;{]*?\b" + name + r"\s*\(", text)
    assert at, f"{file} has no kernel {name}"
    start = text.index("{", at.end())
    depth = 0
    for i in range(start, len(text)):
        depth += {"{": 1, "}": -1}.get(text[i], 0)
        if depth == 0:
            return text[start:i]
    raise AssertionError(f"{file}: {name} does not end")


@pytest.mark.parametrize("file,name", [
    ("sample.cu", "sample_rows_cluster"), ("softmax.cu", "softmax_rows_cluster"), ("layernorm.cu", "layernorm_rows_cluster"),
    ("rmsnorm.cu", "rmsnorm_rows_cluster"), ("gemm_tcgen05_2cta.cu", "gemm_bf16_tcgen05_pair_kernel"),
    ("gemm_tcgen05_ln.cu", "gemm_bias_residual_layernorm_kernel"), ("gemm_tcgen05_splitk.cu", "gemm_bf16_splitk_cluster_kernel")])
def test_cluster_barrier_before_the_first_remote_access(file, name):
    body = kernel_body(file, name)
    remote, barrier = REMOTE.search(body), BARRIER.search(body)
    assert remote, "no access to another CTA's shared memory found"
    assert barrier and barrier.start() < remote.start(), f"{remote.group()} comes before any cluster barrier"
