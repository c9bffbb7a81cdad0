"""CPU: the waits of the recurrence's scan over tiles end however few workgroups run at
once, for every width: a model of the tiles' order (tests/layer_check/progress.cpp) over the
kernels' own rule for the channels that a workgroup looks at."""

import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CLANGXX = "/opt/rocm/llvm/bin/clang++"


def test_every_wait_ends(tmp_path):
    if not os.path.exists(CLANGXX):
        pytest.skip(f"{CLANGXX} not available")
    out = str(tmp_path / "progress")
    r = subprocess.run([CLANGXX, "-O2", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-isystem", "/opt/rocm/include", "-I",
                        os.path.join(ROOT, "paper_2609_32114_amd", "csrc"),
                        os.path.join(ROOT, "tests", "layer_check", "progress.cpp"), "-o", out], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([out], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and "every wait ends" in r.stdout, r.stdout
