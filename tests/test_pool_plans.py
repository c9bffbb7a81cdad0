"""CPU: forks and compactions of state pools by the kernels' own source, compiled for the host
(tests/mixer_check/on_host.h) under AddressSanitizer and UndefinedBehaviorSanitizer: no plan
reads or writes outside its tables and workspace, and each does what the rules say, whatever
the numbers of slots and children."""

import os
import shutil
import subprocess

from test_host_sanitizers import CLANGXX, ROOT, SAN, _need


def test_plans_of_all_sizes_on_the_host(tmp_path):
    _need(CLANGXX)
    csrc, check = os.path.join(ROOT, "paper_2609_32114_amd", "csrc"), os.path.join(ROOT, "tests", "mixer_check")
    for name in ("k12_pool.hip", "api_mixer.cpp", "mixer.h", "layer.h"):
        shutil.copy(os.path.join(csrc, name), tmp_path)
    for name in ("device.h", "prefill.h", os.path.join("hip", "hip_runtime.h")):
        path = tmp_path / name
        path.parent.mkdir(exist_ok=True)
        path.write_text('#include "on_host.h"\n')
    exe = str(tmp_path / "pools")
    r = subprocess.run([CLANGXX, "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer", *SAN, "-I", str(tmp_path), "-I",
                        check, "-I", os.path.join(ROOT, "include"), os.path.join(check, "pools.cpp"), "-o", exe],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0:detect_stack_use_after_return=0", UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=300)
    assert r.returncode == 0 and "pool plans passed" in r.stdout, r.stdout + r.stderr
