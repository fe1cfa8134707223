"""The grouped product's loop reads a stage's tokens from LDS after waiting until at most N of a wavefront's vector memory operations are outstanding: right
only where at least N were asked for behind that stage's token loads, in the order in which the compiler has left them.  Checked on
the assembly of the library's own source, without a GPU: in front of each loop, and in each of its turns."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2310_18859_amd import build

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
KERNEL = re.compile(r"mx_gemm_tilesILb(\d)ELi(\d+)ELi(\d+)ELi(\d+)ELi(\d+)E")


@pytest.fixture(scope="module")
def functions(tmp_path_factory):
    if shutil.which(HIPCC) is None:
        pytest.skip("needs the HIP compiler")
    out = tmp_path_factory.mktemp("asm") / "mx_gemm.s"
    subprocess.run([HIPCC, "--offload-arch=gfx950", "-O3", "-std=c++17", "-x", "hip", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
                    "-I" + os.path.join(build.ROOT, "include"), "-I" + build.CSRC, "--cuda-device-only", "-S", "-o", str(out),
                    os.path.join(build.CSRC, "mx_gemm.hip")], check=True, capture_output=True)
    found = {}
    for text in re.split(r"\n(?=_ZN4sida\S+:)", out.read_text()):
        m = KERNEL.search(text.split(":", 1)[0])
        if m:
            found[text.split(":", 1)[0]] = ([int(v) for v in m.groups()], text)
    assert found
    return found


def events(text):
    """('lds' | 'load', ...) for what a wavefront asks for, ('barrier', N) with the strictest wait since the last of them (None: there is none),
    ('end', ...) where a way through the kernel ends, in the order of the listing."""
    most = None
    for line in text.split("\n"):
        line = line.split(";")[0].strip()
        if re.match(r"(buffer|global)_load", line):
            most = None
            yield "lds" if line.endswith("lds") else "load", line
        elif line.startswith("s_barrier"):
            yield "barrier", most
        elif m := re.match(r"s_waitcnt vmcnt\((\d+)\)", line):
            most = int(m.group(1)) if most is None else min(most, int(m.group(1)))
        elif re.match(r"(buffer|global)_store|s_endpgm", line):
            yield "end", line


def test_first_stage(functions):
    for name, ((x4, mi, ns, nb, wb), text) in functions.items():
        loops, run, ahead = 0, [], True                                 # ahead: in front of a loop
        for kind, what in events(text):
            if kind in ("lds", "load"):
                run.append(kind)
            elif kind == "end":
                ahead, run = True, []
            elif ahead and what == 0:
                run = []                                                # everything has arrived
            elif ahead:
                lds = [j for j, k in enumerate(run) if k == "lds"]
                per = len(lds) // nb                                    # token loads of a stage: as many as blocks of 32 tokens, and a scale
                assert what is not None and lds and len(lds) == nb * per and 1 <= per - x4 <= mi, (name, run)
                later = len(run) - 1 - lds[per - 1]                     # asked for behind the first stage's last token load
                assert later >= what, (name, per, later, what)
                loops += 1
                ahead = False
        assert loops == mi, (name, loops)                               # a way through the kernel for each number of blocks


def test_turns_of_the_loop(functions):
    """Between two waits that leave anything outstanding a wavefront asks for one stage's tokens and then for one stage's weights, or more."""
    for name, ((x4, mi, ns, nb, wb), text) in functions.items():
        turns, run, most, ahead = 0, [], 0, True
        for kind, what in events(text):
            if kind in ("lds", "load"):
                run.append(kind)
            elif kind == "end":
                ahead, run, most = True, [], 0
            else:
                tokens = run.count("lds")
                weights = len(run) - tokens
                if not ahead and most:
                    assert run[:tokens] == ["lds"] * tokens and 1 <= tokens - x4 <= mi, (name, run)
                    assert weights >= ns * (5 if x4 else 1), (name, run)
                    # a stage's tokens have NB - 1 later stages' tokens and WB stages' weights, at least, behind them
                    assert most <= (nb - 1) * tokens + wb * ns * (5 if x4 else 1), (name, most, tokens, weights)
                    turns += 1
                ahead, run, most = False, [], what
        assert turns >= mi, (name, turns)
