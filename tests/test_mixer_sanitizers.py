"""CPU: the host code of the convolution's, the scan's and the pools' entry points under
AddressSanitizer and UndefinedBehaviorSanitizer, as test_layer_sanitizers.py does for the others:
api.cpp and api_mixer.cpp with the sanitizers on their host side, linked with stubs of the
launchers and driven by tests/mixer_check/mixer_check.c."""

import os
import subprocess

from test_host_sanitizers import CLANG, CLANGXX, HIPCC, ROOT, SAN, SAN_HOST, _need


def test_mixer_host_code_under_sanitizers(tmp_path):
    for t in (HIPCC, CLANG, CLANGXX):
        _need(t)
    csrc = os.path.join(ROOT, "paper_2609_32114_amd", "csrc")
    tests = os.path.join(ROOT, "tests")
    inc = ["-I", os.path.join(ROOT, "include"), "-I", csrc]
    hip = [HIPCC, "-x", "hip", "--offload-arch=gfx950", "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer",
           *SAN_HOST, *inc]
    objects = {"api": os.path.join(csrc, "api.cpp"), "api_mixer": os.path.join(csrc, "api_mixer.cpp"),
               "stubs": os.path.join(tests, "host_check", "stubs.cpp"),
               "mixer_stubs": os.path.join(tests, "mixer_check", "stubs.cpp")}
    steps = [hip + ["-c", src, "-o", str(tmp_path / f"{name}.o")] for name, src in objects.items()]
    steps.append([CLANG, "-O1", "-g", *SAN, *inc, "-c", os.path.join(tests, "mixer_check", "mixer_check.c"), "-o",
                  str(tmp_path / "check.o")])
    steps.append([CLANGXX, *SAN, str(tmp_path / "check.o"), *[str(tmp_path / f"{n}.o") for n in objects],
                  "-L/opt/rocm/lib", "-lamdhip64", "-Wl,-rpath,/opt/rocm/lib", "-o", str(tmp_path / "check")])
    for cmd in steps:
        r = subprocess.run(cmd, capture_output=True, text=True)
        assert r.returncode == 0, f"{' '.join(cmd)}\n{r.stderr}"
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([str(tmp_path / "check")], capture_output=True, text=True, env=env, timeout=300)
    assert r.returncode == 0 and "mixer checks passed" in r.stdout, r.stdout + r.stderr
