"""Shared memory of another CTA of a cluster may only be touched once that CTA has started: in every
kernel a barrier of the whole cluster comes before the first remote access."""
import os
import re

from paper_1909_09010_b200 import build

REMOTE = re.compile(r"st_remote\(|arrive_remote\(|st\.async|mbarrier\.arrive[^\"]*shared::cluster")
BARRIER = re.compile(r"cluster_sync\(\)|cluster_wait\(\)")


def kernels():
    """(name, body) of every kernel in the CUDA sources, comments taken out."""
    for file in sorted(os.listdir(build.CSRC)):
        text = re.sub(r"//[^\n]*", "", open(os.path.join(build.CSRC, file)).read())
        for m in re.finditer(r"__global__ void[^;{]*?(\w+)\s*\(const[^;{]*\)\s*\{|__global__ void[^;{]*?(\w+)\s*\([^;{]*\)\s*\{", text):
            depth, at = 1, m.end()
            while depth:
                depth += {"{": 1, "}": -1}.get(text[at], 0)
                at += 1
            yield m.group(1) or m.group(2), text[m.end():at]


def test_cluster_has_started_before_the_first_remote_access():
    seen = set()
    for name, body in kernels():
        remote = REMOTE.search(body)
        if remote:
            seen.add(name)
            barrier = BARRIER.search(body)
            assert barrier and barrier.start() < remote.start(), f"{name}: remote access before a cluster barrier"
    assert {"column_sum_kernel", "linear_tc_kernel", "cross_entropy_ring_kernel"} <= seen
