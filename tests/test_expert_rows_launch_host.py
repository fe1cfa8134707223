"""The launches of the way of tokens to their experts and back (csrc/expert_rule.h), without a GPU: fewer than 2^32 threads in whole workgroups, up to the most pairs that a
call takes."""
import ctypes
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2310_18859_amd", "csrc")
SOURCE = r"""
#include "expert_rule.h"
extern "C" int lanes(int pieces, long tokens) { return 1 << sida::rows_lanes_log2(pieces, tokens); }
"""


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    d = tmp_path_factory.mktemp("rows_launch")
    src, so = str(d / "rule.cpp"), str(d / "rule.so")
    with open(src, "w") as f:
        f.write(SOURCE)
    subprocess.run(["g++", "-O1", "-std=c++17", "-fPIC", "-shared", "-Wall", "-I" + CSRC, "-o", so, src], check=True)
    lib = ctypes.CDLL(so)
    lib.lanes.argtypes = [ctypes.c_int, ctypes.c_long]
    return lib


@pytest.mark.parametrize("pieces", [0, 1, 8, 9, 32, 33, 64, 65, 8192, 65536])
def test_threads(rule, pieces):
    for tokens in [1, 1000, 1 << 25] + list(range((1 << 26) - 20, 1 << 26)):
        lanes = rule.lanes(pieces, tokens)
        assert (tokens * lanes + 255) // 256 * 256 < 1 << 32, tokens
        assert lanes == min(64, max(8, 1 << max(0, pieces - 1).bit_length())) or tokens * 64 > (1 << 32) - 256
