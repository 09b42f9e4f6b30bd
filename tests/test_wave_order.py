"""Lanes of a wave that hand each other values through LDS: what the compiler is told of it (no GPU).

A fence of wavefront scope orders a lane's own accesses.  It does not say that the lanes come together: behind a branch or a loop that only some
of them enter, code may run for some lanes before others have stored what it reads.  A convergent operation between a release and an acquire says both."""
import os
import re
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2310_12670_amd", "csrc")


def fenced():
    return sorted(f for f in os.listdir(CSRC) if f.endswith(".hip") and '"wavefront"' in open(os.path.join(CSRC, f)).read())


@pytest.mark.parametrize("source", fenced())
def test_lanes_meet_where_they_exchange_values(source, tmp_path):
    out = tmp_path / "device.ll"
    subprocess.run(["hipcc", "--offload-arch=gfx950", "--offload-device-only", "-O3", "-std=c++17", "-w", "-S", "-emit-llvm", "-Xclang",
                    "-disable-llvm-passes", "-o", str(out), os.path.join(CSRC, source)], check=True)
    lines = [line.strip() for line in out.read_text().splitlines()]
    fences = [i for i, line in enumerate(lines) if line.startswith('fence syncscope("wavefront")')]
    meet = ['fence syncscope("wavefront") release', "call void @llvm.amdgcn.wave.barrier()", 'fence syncscope("wavefront") acquire']
    assert fences and all([re.sub(r"[,;].*| #\d+$", "", line) for line in lines[i:i + 3]] == meet for i in fences[::2])
    assert fences[1::2] == [i + 2 for i in fences[::2]]
