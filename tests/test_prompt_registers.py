"""The attention over packed tokens moves registers between its warps (csrc/prompt.cu): what the launch brings has to be what the split counts
on, and no role may spill, by the compiler's own account."""
import os
import re
import subprocess

import pytest

from paper_2509_18824_b200 import build


def test_registers_of_the_launch_and_no_spills(tmp_path):
    nvcc = build._nvcc()
    if not os.path.exists(nvcc):
        pytest.skip("no nvcc")
    text = open(os.path.join(build.CSRC, "prompt.cu")).read()
    soft, other = (int(x) for x in re.search(r"kSoftmaxRegs = (\d+), kOtherRegs = (\d+)", text).groups())
    launch, threads = int(re.search(r"kLaunchRegs = (\d+)", text).group(1)), int(re.search(r"kPThreads = (\d+)", text).group(1))
    assert threads // 2 * (soft + other) <= threads * launch and soft % 8 == 0 and other % 8 == 0
    r = subprocess.run([nvcc] + build.NVCC_FLAGS + ["-Xptxas", "-v", "-c", os.path.join(build.CSRC, "prompt.cu"), "-o", str(tmp_path / "p.o")],
                       capture_output=True, text=True, check=True)
    said = re.search(r"Function properties for \S*13prompt_kernel\S*\n\s+\d+ bytes stack frame, (\d+) bytes spill stores, (\d+) bytes spill loads\n"
                     r"ptxas info\s+: Used (\d+) registers", r.stdout + r.stderr)
    assert said, r.stderr
    assert [int(x) for x in said.groups()] == [0, 0, launch]
