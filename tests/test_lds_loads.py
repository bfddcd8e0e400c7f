"""Loads from memory straight into LDS take their LDS base from M0.  The compiler has to know that they write it: code around
them that has a value of its own in M0 must get it back.  Looks at the assembly of a few lines that use both."""
import os
import re
import subprocess

import pytest

from paper_2406_10774_amd import build

SOURCE = """
#include "quest_rows_core.h"
extern "C" __global__ void around(const char* from) {
  __shared__ __align__(16) char lds[2048];
  __builtin_amdgcn_s_sendmsg(1, 0x1234);
  %s
  quest::dma_arrived<0>();
  __builtin_amdgcn_s_sendmsg(1, 0x1234);
}
"""


@pytest.mark.parametrize("load", ["quest::dma16(quest::lds_address(lds + 1024), from, threadIdx.x * 16);",
                                  "quest::dma16(quest::lds_address(lds + 1024), from + threadIdx.x * 16);"])
def test_m0_is_set_again_behind_a_load(tmp_path, load):
    source, out = tmp_path / "around.hip", tmp_path / "around.s"
    source.write_text(SOURCE % load)
    hipcc = build.shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    subprocess.run([hipcc, *[f for f in build.HIPCC_FLAGS if f != "-Wall"], "-I", build.CSRC, "-S", "--cuda-device-only", str(source),
                    "-o", str(out)], check=True, capture_output=True, env=dict(os.environ))
    steps = []
    for line in out.read_text().splitlines():
        write = re.match(r"\s+s_\w+ m0, (.*)", line)
        if write:
            steps.append(write[1].strip())
        elif "s_sendmsg" in line:
            steps.append("message")
        elif "global_load_lds" in line:
            steps.append("load")
    first, second = [i for i, s in enumerate(steps) if s == "message"]
    load = steps.index("load")
    assert first < load < second
    assert steps[first - 1] == "0x1234" == steps[second - 1], steps      # each message with its own value
    assert steps[load - 1] not in ("message", "0x1234"), steps              # the load with its base
