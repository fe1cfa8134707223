"""Which kernel the grouped product with experts in 4 bits takes (csrc/mx_rule.h), checked without a GPU: for the sizes by which the GPU tests mean to
reach each of them, for both kernels' largest batches, and at the rule's lines."""
import ctypes
import os
import subprocess

import pytest

import test_gpu_mx_tiles as sizes

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2310_18859_amd", "csrc")
KERNELS = ("split", "rows32", "rows64", "rows128")

SOURCE = r"""
#include "mx_rule.h"
extern "C" int pick(bool x4, long M, long groups, long N, long K) { return (int)sida::mx_tiles(x4, M, groups, N, K); }
"""


@pytest.fixture(scope="module")
def pick(tmp_path_factory):
    d = tmp_path_factory.mktemp("mx_rule")
    src, so = str(d / "rule.cpp"), str(d / "rule.so")
    with open(src, "w") as f:
        f.write(SOURCE)
    subprocess.run(["g++", "-O1", "-std=c++17", "-fPIC", "-shared", "-Wall", "-I" + CSRC, "-o", so, src], check=True)
    fn = ctypes.CDLL(so).pick
    fn.argtypes = [ctypes.c_bool] + [ctypes.c_long] * 4
    return lambda *a: KERNELS[fn(*a)]


@pytest.mark.parametrize("size", sizes.SIZES + sizes.ALIGNED + sizes.EACH + sizes.FAR, ids=repr)
def test_sizes_reach_the_kernel_they_name(pick, size):
    assert pick(size.x4, size.M, len(size.counts), size.N, size.K) == size.kernel


def test_each_kernel_is_reached():
    for of in (sizes.SIZES, sizes.ALIGNED, sizes.EACH):
        assert {(s.kernel, s.x4) for s in of} == {(k, x4) for k in KERNELS for x4 in (False, True)} - {("rows128", False)}


@pytest.mark.parametrize("kernel,blocks", [("rows32", 1), ("rows64", 2), ("rows128", 4)])
def test_tiles_of_each_number_of_blocks(kernel, blocks):
    """... of 32 rows: a way of its own through the kernel each."""
    for s in sizes.SIZES + sizes.ALIGNED + sizes.EACH:
        if s.kernel == kernel:
            rest = {(-(-((n - 1) % (32 * blocks) + 1) // 32)) for n in s.counts if n}
            rest |= {blocks} if max(s.counts) >= 32 * blocks else set()
            assert rest == set(range(1, blocks + 1)), s


@pytest.mark.parametrize("x4,M,groups,N,K,want", [
    (False, 1, 128, 1024, 4096, "split"), (False, 128, 128, 3072, 768, "rows32"), (False, 1111, 64, 768, 3072, "rows32"),
    (False, 16384, 128, 3072, 768, "rows64"), (True, 999, 64, 4096, 1024, "rows32"), (True, 32768, 128, 1024, 4096, "rows128"),
    (True, 16384, 64, 3072, 768, "rows64"), (True, 192 * 64, 64, 1024, 2048, "rows128"), (True, 192 * 64 - 1, 64, 1024, 2048, "rows64"),
    (True, 192 * 64, 64, 1024, 2016, "rows64"), (False, 33 * 64, 64, 2048, 1024, "rows64"), (False, 33 * 64 - 1, 64, 2048, 1024, "rows32"),
    (False, 64, 1, 1024, 384, "split"), (False, 64, 1, 1024, 380, "rows32"),
])
def test_lines(pick, x4, M, groups, N, K, want):
    assert pick(x4, M, groups, N, K) == want
