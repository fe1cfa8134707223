"""Which kernels the products of plain bf16 experts take, and how the sort and the weights' gradient are cut up (csrc/expert_rule.h), checked without a GPU: for
the sizes by which the GPU tests mean to reach each of them, and at the rules' lines."""
import ctypes
import os
import subprocess

import pytest

import test_gpu_expert_tiles as sizes

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2310_18859_amd", "csrc")
KERNELS = ("few", "rows32", "rows64", "square128", "rows256")
HEIGHT = {"few": 32, "rows32": 32, "rows64": 64, "square128": 128, "rows256": 256}

SOURCE = r"""
#include "expert_rule.h"
using namespace sida;
extern "C" {
int pick(long M, long groups, long cols, long length) { return (int)expert_tiles(M, groups, cols, length); }
int chunk(long M, long groups, long N, long K) { return expert_weights_chunk(M, groups, N, K); }
int small(long groups, long N, long K) { return expert_weights_small(groups, N, K); }
long parts(long M, long groups, long chunk) { return expert_weights_parts(M, groups, chunk); }
long most(long groups, long N, long K) { return expert_weights_most(groups, N, K) + groups; }
int sort_chunk(long pairs) { return expert_sort_chunk(pairs); }
int sort_chunks(long pairs) { return expert_sort_chunks(pairs); }
long sort_most(long pairs) { return expert_sort_most(pairs); }
int lanes(int pieces) { return 1 << rows_lanes_log2(pieces); }
}
"""


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    d = tmp_path_factory.mktemp("expert_rule")
    src, so = str(d / "rule.cpp"), str(d / "rule.so")
    with open(src, "w") as f:
        f.write(SOURCE)
    subprocess.run(["g++", "-O1", "-std=c++17", "-fPIC", "-shared", "-Wall", "-I" + CSRC, "-o", so, src], check=True)
    lib = ctypes.CDLL(so)
    for name, n, res in (("pick", 4, ctypes.c_int), ("chunk", 4, ctypes.c_int), ("small", 3, ctypes.c_int), ("parts", 3, ctypes.c_long), ("most", 3, ctypes.c_long),
                         ("sort_chunk", 1, ctypes.c_int), ("sort_chunks", 1, ctypes.c_int), ("sort_most", 1, ctypes.c_long)):
        getattr(lib, name).argtypes, getattr(lib, name).restype = [ctypes.c_long] * n, res
    return lib


@pytest.mark.parametrize("kernel,counts,cols,length", sizes.SIZES)
def test_sizes_reach_the_kernel_they_name(rule, kernel, counts, cols, length):
    assert KERNELS[rule.pick(sum(counts), len(counts), cols, length)] == kernel


@pytest.mark.parametrize("kernel,counts,N,K", sizes.WEIGHTS)
def test_gradients_reach_the_kernel_they_name(rule, kernel, counts, N, K):
    chunk = rule.chunk(sum(counts), len(counts), N, K)
    assert ("parts" if chunk else "square128" if rule.small(len(counts), N, K) else "rows256") == kernel


def test_each_kernel_and_number_of_blocks_is_reached():
    """... of 32 rows: a way of its own through a kernel each."""
    assert {s[0] for s in sizes.SIZES} == set(KERNELS) and {s[0] for s in sizes.WEIGHTS} == {"rows256", "square128", "parts"}
    for kernel, height in HEIGHT.items():
        blocks = {-(-((n - 1) % height + 1) // 32) for k, counts, _, _ in sizes.SIZES if k == kernel for n in counts if n}
        blocks |= {height // 32} if any(k == kernel and max(c) >= height for k, c, _, _ in sizes.SIZES) else set()
        assert blocks == set(range(1, height // 32 + 1)), kernel


@pytest.mark.parametrize("M,groups,cols,length,want", [
    (1, 8, 4096, 1024, "few"), (1, 1, 8, 8, "few"), (1111, 64, 2048, 1024, "rows32"), (2048, 64, 4096, 1024, "rows64"), (8192, 64, 4096, 1024, "square128"),
    (32768, 64, 4096, 1024, "rows256"), (32768, 64, 1024, 4096, "rows256"), (24 * 64, 64, 4096, 1024, "rows32"), (25 * 64, 64, 4096, 1024, "rows64"),
    (96 * 64, 64, 4096, 1024, "rows64"), (97 * 64, 64, 4096, 1024, "square128"), (512, 1, 1024, 1024, "rows32"), (4096, 1, 1024, 1024, "square128"),
    (1 << 24, 1, 2048, 8, "rows256"), (1 << 24, 256, 8, 8, "rows256"),
])
def test_lines(rule, M, groups, cols, length, want):
    assert KERNELS[rule.pick(M, groups, cols, length)] == want


def test_parts_fit_their_workspace(rule):
    """As many parts as a call can have, for every number of rows, within what the largest number asks for."""
    cut = 0
    for groups, N, K in ((1, 8, 8), (1, 1024, 1024), (1, 4096, 1024), (2, 256, 256), (4, 520, 264), (8, 1024, 512), (50, 200, 128), (100, 64, 64), (255, 8, 8)):
        for M in list(range(1, 3000, 37)) + [4096, 16385, 65537, 1 << 20, 1 << 24]:
            chunk = rule.chunk(M, groups, N, K)
            if chunk:
                cut += 1
                assert chunk >= 256 and chunk % 64 == 0
                assert rule.parts(M, groups, chunk) <= rule.most(groups, N, K)
                assert rule.chunk(M + 1, groups, N, K) > 0             # and no fewer rows make a call ask for more
    assert cut > 100


@pytest.mark.parametrize("groups,N,K", [(1, 8, 8), (1, 128, 128), (1, 256, 128), (2, 128, 64), (16, 8, 128), (100, 64, 64)])
def test_parts_fit_their_workspace_a_little_above_a_multiple(rule, groups, N, K):
    """Rows that are a few more than an even share for each part: one part more than there are shares, if the share were rounded down."""
    most = rule.most(groups, N, K) - groups
    for share in (256, 320, 4096):
        for M in range(share * most, share * most + 600, 7):
            assert rule.parts(M, groups, rule.chunk(M, groups, N, K)) <= most + groups


def test_sorts_chunks(rule):
    for pairs in list(range(1, 9000, 61)) + [4096, 4097, 524288, 524289, 600000, 1 << 20, (1 << 26) - 1]:
        chunk, n = rule.sort_chunk(pairs), rule.sort_chunks(pairs)
        assert chunk % 1024 == 0 and n <= 256 and (n - 1) * chunk < pairs <= n * chunk
        assert n <= rule.sort_most(pairs) <= rule.sort_most(pairs + 1)


def test_lanes_of_a_row(rule):
    assert [rule.lanes(p) for p in (0, 1, 8, 9, 16, 17, 32, 33, 64, 65, 100000)] == [8, 8, 8, 16, 16, 32, 32, 64, 64, 64, 64]
