"""What a run cannot show about the kernels, read in their sources."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2502_15572_b200", "csrc")


def body(source, head):
    """The braces behind `head`, comments left out."""
    text = re.sub(r"//[^\n]*", "", source)
    at = text.index("{", text.index(head))
    depth = 0
    for i in range(at, len(text)):
        depth += {"{": 1, "}": -1}.get(text[i], 0)
        if depth == 0:
            return text[at:i + 1]
    raise ValueError(head)


def read(name):
    with open(os.path.join(CSRC, name)) as f:
        return f.read()


def test_sampling_reaches_other_ctas_only_when_they_have_begun():
    """A CTA's shared memory may be reached by the others of its cluster once it has begun: a cluster barrier comes before the first access.
    maximum() is what a sequence's first row begins with; its wait belongs to the arrival at the kernel's entry."""
    source = read("k13_sample.cu")
    kernel, maximum = body(source, "sample_kernel(const SampleArgs"), body(source, "int maximum(")
    assert kernel.index("cluster_arrive()") < kernel.index("pdl_wait()") < kernel.index("one.maximum(")
    for reach in ("in_cta(", "one.few(", "select<", "one.draw("):
        assert reach not in kernel[:kernel.index("one.maximum(")]
    assert "cluster_wait()" in maximum[:maximum.index("in_cta(")]
    assert re.search(r"one\.maximum\(\w+, t == 0\)", kernel) and re.search(r"if \(first\) cluster_wait\(\)", maximum)


@pytest.mark.parametrize("name,kernel,reach", [("k14_kv_pages.cu", "reserve_kernel(const KvArgs", "scan_cluster("), ("k14_kv_pages.cu", "compact_kernel(const KvArgs", "scan_cluster("),
                                               ("k15_w4.cu", "matmul_mma_kernel(const W4Args", "mapa_rank("), ("k16_w4_umma.cu", "matmul_umma_kernel(const __grid_constant__", "mapa_rank(")])
def test_a_cluster_barrier_comes_before_the_first_access(name, kernel, reach):
    text = body(read(name), kernel)
    before = text[:text.index(reach)]
    assert "cluster_sync_all()" in before or "cluster_wait()" in before


@pytest.mark.parametrize("name", sorted(n for n in os.listdir(CSRC) if n.endswith((".cu", ".cuh", ".h"))))
def test_what_calls_remember_is_atomic(name):
    """Calls of several host threads may be the first ones together: what a function keeps for the process is an atomic, a thread's own, or constant."""
    text = re.sub(r"//[^\n]*", "", read(name))
    kept = re.findall(r"^ +static (?!const|__device__|cudaError_t|inline)([^;=({]+)[;={]", text, re.M)
    assert all(k.startswith(("std::atomic<", "thread_local ")) for k in kept), kept
