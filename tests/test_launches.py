"""What the blocks of a launch touch, with the kernels' source run on the CPU: no block behind
the last row or the last weights touches memory, which no GPU is asked to show."""
import os
import subprocess

import pytest

from tests import helpers

CSRC = os.path.join(helpers.ROOT, "paper_2606_02916_amd", "csrc")
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")


@pytest.mark.parametrize("what", ["rows", "weights"])
def test_blocks_behind_the_end_touch_nothing(what):
    """Of rows and weights put into 8 bits, with fewer and more blocks than one dimension of a
    grid holds."""
    exe = helpers.build_helper("overhang.cpp", subdir="host",
                               compiler=os.path.join(ROCM, "llvm", "bin", "clang++"),
                               extra=["-x", "c++", "-std=c++17", "-Wno-align-mismatch", f"-I{ROCM}/include",
                                      "-I" + os.path.join(helpers.ROOT, "include"), "-I" + CSRC])
    out = subprocess.run([exe, what], capture_output=True, text=True)
    assert out.returncode == 0, out.stdout
    assert int(out.stdout.split()[-2]) >= 36
