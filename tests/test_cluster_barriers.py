"""Kernels of a thread-block cluster, by their sources: shared memory of another block may be touched only once that block is
known to run, so a cluster barrier stands before the first address of another block is formed."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2506_15050_b200", "csrc")
BARRIER = re.compile(r"cluster_(sync_all|wait)\(\)")


def kernels():
    """(file, text from one __global__ to the next) of every kernel that addresses another block of its cluster."""
    out = []
    for path in sorted(glob.glob(os.path.join(CSRC, "*.cu*"))):
        with open(path) as f:
            text = re.sub(r"//[^\n]*", "", f.read())
        out += [(os.path.basename(path), k) for k in text.split("__global__")[1:] if "map_to_cta(" in k]
    return out


def test_kernels_are_found():
    assert {"dense_gemm.cuh", "fp8_matmul.cu", "grad_norm.cu", "policy_cluster.cu", "umma_gemm_pair.cuh"} <= {f for f, _ in kernels()}


@pytest.mark.parametrize("file,text", kernels(), ids=lambda v: v if v.endswith((".cu", ".cuh")) else "kernel")
def test_a_barrier_stands_before_the_first_remote_address(file, text):
    first = BARRIER.search(text)
    assert first and first.start() < text.index("map_to_cta("), file


def test_a_warp_meets_in_front_of_each_aligned_barrier():
    """The warp-aligned barriers follow code that a single thread ran (it set up mbarriers, or stored a sum)."""
    found = 0
    for path in sorted(glob.glob(os.path.join(CSRC, "*.cu*"))):
        with open(path) as f:
            text = f.read()
        for m in re.finditer(r'asm volatile\("barrier\.cluster\.', text):
            found += 1
            assert text[:m.start()].rstrip().endswith("__syncwarp();"), os.path.basename(path)
    assert found >= 1
