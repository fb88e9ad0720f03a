"""The host code of the 8-bit cache and the rotary positions (vc_q8_api.cpp),
built with the address and undefined-behaviour sanitizers and run on the CPU
over ordinary, extreme and wrong arguments (tests/sanitize/q8_driver.cpp): no
call overflows, and every plan that reaches a launcher keeps what its kernel
takes for granted (workgroups, workspace regions, tiles that are cut)."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SAN = ["-fsanitize=address,undefined", "-fno-sanitize-recover=undefined", "-fno-omit-frame-pointer", "-g", "-O1"]


@pytest.mark.timeout(300)
def test_q8_host_code_under_sanitizers(tmp_path):
    gxx = shutil.which("g++")
    if not gxx:
        pytest.skip("no host compiler")
    exe = str(tmp_path / "q8_driver")
    subprocess.check_call([gxx, "-std=c++17", "-I", os.path.join(ROOT, "include"), "-I", "/opt/rocm/include",
                           "-D__HIP_PLATFORM_AMD__"] + SAN +
                          [os.path.join(ROOT, "paper_2608_24063_amd", "csrc", "vc_q8_api.cpp"),
                           os.path.join(ROOT, "tests", "sanitize", "q8_driver.cpp"), "-o", exe])
    env = dict(os.environ, ASAN_OPTIONS="halt_on_error=1:exitcode=99",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=200)
    assert r.returncode == 0, f"rc {r.returncode}\n{r.stdout[-2000:]}\n{r.stderr[-4000:]}"
    assert "q8 host checks ok" in r.stdout and "runtime error" not in r.stderr, r.stderr[-4000:]
