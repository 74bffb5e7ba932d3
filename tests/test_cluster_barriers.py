"""A CTA's shared memory may be touched by the others of its cluster only once it is known to have started: in every kernel with a
cluster, a barrier of the cluster stands in front of the first access to another CTA's shared memory.  A missing one is not
seen on the GPU (the order in which CTAs usually start hides it), so this reads the source."""
import pathlib
import re

import pytest

CSRC = pathlib.Path(__file__).parent.parent / "paper_2603_18489_b200" / "csrc"
WAIT = re.compile(r"\b(?:cluster_wait|cluster\.sync|cluster\.barrier_wait)\s*\(")
REMOTE = re.compile(r"\b(?:map_shared_rank|map_to_cta|bulk_copy_to_peer)\s*\(")


def source(name):
    return re.sub(r"//[^\n]*", "", (CSRC / name).read_text())


def body_of(src, head):
    """What stands between the braces behind `head`."""
    start = src.index("{", src.index(head)) + 1
    depth, i = 1, start
    while depth:
        depth += {"{": 1, "}": -1}.get(src[i], 0)
        i += 1
    return src[start:i]


def test_sampling_kernel_arrives_at_the_start_and_waits_before_the_first_publish():
    src = source("ec_sample.cu")
    assert REMOTE.search(body_of(src, "void publish(int slot, u64 v)"))       # what makes publish() an access to other CTAs
    run = body_of(src, "__device__ void run(const SampleArgs& a, int r)")
    first, wait = re.search(r"\bpublish\(", run).start(), WAIT.search(run)
    assert wait and wait.start() < first
    # nothing on the way there touches another CTA, and all threads come by
    assert not REMOTE.search(run[:wait.start()]) and "return" not in run[:wait.start()]
    for name in ("void first_pass(F f)", "void block_min_max(u64& a, u64& b)"):
        assert not REMOTE.search(body_of(src, name)) and not WAIT.search(body_of(src, name))
    # its other half, once, at the kernel's start
    kernel = body_of(src, "sample_kernel(const SampleArgs a, int segment)")
    arrive = re.search(r"\bcluster_arrive\w*\(", kernel)
    assert arrive and arrive.start() < kernel.index("row.run(")
    assert len(re.findall(r"\bcluster_arrive\w*\(", src)) == len(re.findall(r"\bcluster_wait\(", src)) == 1


def test_attention_kernels_pass_a_barrier_before_they_read_from_others():
    seen = 0
    for path in sorted(CSRC.glob("*.cu")):
        src = source(path.name)
        for m in re.finditer(r"__global__[^;{]*\)\s*\{", src):
            kernel = body_of(src[m.start():], "__global__")
            remote = REMOTE.search(kernel)
            if remote:
                seen += 1
                wait = WAIT.search(kernel)
                assert wait and wait.start() < remote.start(), path.name
    assert seen >= 4
