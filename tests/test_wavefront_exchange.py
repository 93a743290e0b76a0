"""Lanes of one wavefront that pass values through LDS need no barrier of the workgroup, but the compiler has to be kept
from moving their accesses over the point of exchange: the wavefront's barrier alone orders instructions, not memory.
Checked in the source, because a build that happens to keep the order shows nothing."""
import glob
import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_1707_04585_amd", "csrc")
FENCE = r'__builtin_amdgcn_fence\(__ATOMIC_%s, "(wavefront|workgroup)"(, "local")?\);'


def code_lines(path):
    with open(path) as f:
        text = re.sub(r"/\*.*?\*/", "", f.read(), flags=re.S)
    lines = (re.sub(r"//.*", "", line).strip() for line in text.splitlines())
    return [line for line in lines if line]


def test_every_barrier_of_a_wavefront_stands_between_two_fences():
    seen = 0
    for path in sorted(glob.glob(os.path.join(CSRC, "*.h")) + glob.glob(os.path.join(CSRC, "*.hip"))):
        lines = code_lines(path)
        for i, line in enumerate(lines):
            if "__builtin_amdgcn_wave_barrier" not in line:
                continue
            seen += 1
            where = (os.path.basename(path), lines[max(i - 1, 0):i + 2])
            assert line == "__builtin_amdgcn_wave_barrier();", where
            assert re.fullmatch(FENCE % "RELEASE", lines[i - 1]) and re.fullmatch(FENCE % "ACQUIRE", lines[i + 1]), where
    assert seen
