"""Which items a workgroup of the products of plain bf16 experts takes (csrc/expert_rule.h), walked without a GPU: each has to be taken exactly once, by the kernel of few rows,
whose workgroups take one each, as by those that walk on."""
import ctypes
import os
import subprocess

import pytest

import test_gpu_expert_few as sizes

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2310_18859_amd", "csrc")
SOURCE = r"""
#include <cstring>
#include "expert_rule.h"
using namespace sida;
static unsigned char taken[1 << 21];
// Items that are not taken exactly once; a workgroup takes `each` at most (0: until there are none).
extern "C" int walk(long n, int workgroups, int most, int each)
{
    std::memset(taken, 0, n);
    for (int b = 0; b < workgroups; ++b) {
        Items items(n, workgroups, most, b);
        for (int i = 0; !each || i < each; ++i) {
            const int id = items.next();
            if (id < 0) break;
            if (id >= n || ++taken[id] > 1) return -1;
        }
    }
    int missing = 0;
    for (long i = 0; i < n; ++i) missing += taken[i] == 0;
    return missing;
}
extern "C" long grid(long M, long groups, long cols) { return expert_few_grid(M, groups, cols); }
extern "C" int most() { return kFewInARow; }
extern "C" int walking_most() { return kItemsInARow; }
extern "C" int pick(long M, long groups, long cols, long length) { return (int)expert_tiles(M, groups, cols, length); }
extern "C" int pick_input(long M, long groups, long cols, long length) { return (int)expert_tiles(M, groups, cols, length, true); }
"""


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    d = tmp_path_factory.mktemp("expert_items")
    src, so = str(d / "items.cpp"), str(d / "items.so")
    with open(src, "w") as f:
        f.write(SOURCE)
    subprocess.run(["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall", "-I" + CSRC, "-o", so, src], check=True)
    lib = ctypes.CDLL(so)
    lib.walk.argtypes = [ctypes.c_long, ctypes.c_int, ctypes.c_int, ctypes.c_int]
    lib.grid.argtypes, lib.grid.restype = [ctypes.c_long] * 3, ctypes.c_long
    lib.pick.argtypes = lib.pick_input.argtypes = [ctypes.c_long] * 4
    return lib


def test_few_rows_one_item_each(rule):
    most = rule.most()
    for n in range(1, 9000):
        assert rule.walk(n, (n + 7) // 8 * 8, most, 1) == 0, n
    for n in (1, 7, 500, 513, 514, 640, 768, 4000):                   # fewer tiles than the host had to reckon with
        for spare in (8, 64, 1000):
            assert rule.walk(n, (n + 7) // 8 * 8 + spare * 8, most, 1) == 0, (n, spare)


def test_few_rows_every_size_that_the_rule_sends_there(rule):
    """Groups of one row are the most tiles that rows can make, all in one group the fewest."""
    seen = set()
    for groups in (1, 2, 8, 64, 256):
        for M in list(range(1, 40)) + [64, 200, 500]:
            for cols in (8, 72, 1024, 2048, 4096, 5464, 14336, 28672, 65536):
                for length in (8, 1024, 2064, 4096, 8192, 14336, 65536):
                    if rule.pick(M, groups, cols, length):
                        continue
                    width, grid = (cols + 31) // 32, rule.grid(M, groups, cols)
                    for tiles in {min(M, groups) * width, (M + 31) // 32 * width, (M // 32 + min(M, groups)) * width}:
                        assert (tiles, grid) in seen or rule.walk(tiles, grid, rule.most(), 1) == 0, (M, groups, cols, length, tiles)
                        seen.add((tiles, grid))
    assert max(t for t, _ in seen) > 8000


@pytest.mark.parametrize("counts,cols,length", sizes.SIZES)
def test_sizes_of_the_gpu_tests(rule, counts, cols, length):
    tiles = sum(-(-n // 32) for n in counts) * -(-cols // 32)
    assert rule.pick(sum(counts), len(counts), cols, length) == 0 and tiles >= 512
    assert rule.walk(tiles, rule.grid(sum(counts), len(counts), cols), rule.most(), 1) == 0


@pytest.mark.parametrize("workgroups", [8, 16, 24, 128, 240, 256, 512])
def test_walking_workgroups(rule, workgroups):
    for n in list(range(1, 5000, 13)) + [511, 512, 513, 514, 4096, 16385, 65536, 1000003]:
        assert rule.walk(n, workgroups, rule.walking_most(), 0) == 0, n


@pytest.mark.parametrize("M,cols,length,product,input_gradient", [
    (2, 8192, 8192, "few", "few"), (1, 16416, 8192, "few", "rows32"), (5, 4096, 4096, "few", "rows32"), (6, 4096, 4096, "few", "rows32"), (7, 4096, 4096, "rows32", "rows32"),
    (3, 4096, 1024, "few", "few"), (4, 4096, 1024, "rows32", "rows32"), (4, 4096, 2048, "few", "few"), (1, 8192, 8, "few", "few"), (1, 8448, 8, "rows32", "rows32"),
])
def test_lines_of_few_rows(rule, M, cols, length, product, input_gradient):
    """As many tiles as the length of the sum allows, for the input's gradient no more than two rounds of workgroups."""
    names = ("few", "rows32")
    assert (names[rule.pick(M, 8, cols, length)], names[rule.pick_input(M, 8, cols, length)]) == (product, input_gradient)
