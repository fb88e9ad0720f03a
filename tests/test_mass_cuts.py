"""The calls of tests/mass_paths.py are cut as they say (the host code of vc_mass_api.cpp
with launchers that print their plan), so that the GPU's tests of them reach the ways
through the kernels that they are there for."""
import os
import shutil
import subprocess

import pytest

from tests import mass_paths as mp

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.timeout(300)
def test_paths_are_cut_as_they_say(tmp_path):
    gxx = shutil.which("g++")
    if not gxx:
        pytest.skip("no host compiler")
    exe = str(tmp_path / "mass_cuts")
    subprocess.check_call([gxx, "-std=c++17", "-O1", "-I", os.path.join(ROOT, "include"), "-I", "/opt/rocm/include",
                           "-D__HIP_PLATFORM_AMD__",
                           os.path.join(ROOT, "paper_2608_24063_amd", "csrc", "vc_mass_api.cpp"),
                           os.path.join(ROOT, "tests", "sanitize", "mass_cuts.cpp"), "-o", exe])
    for d in (64, 128):
        for p in mp.TOKENS + mp.PROMPTS:
            rows = max(mp.sizes(p)[1])
            line = subprocess.check_output([exe] + [str(x) for x in (p.L, p.B, p.Hq, p.Hkv, d, p.n, rows)], text=True)
            got = dict(x.split("=") for x in line.split())
            assert got["kind"] == ("token" if p in mp.TOKENS else "prompt"), p.name
            assert {k: int(got[k]) for k in p.cut} == p.cut, (p.name, line)
    # The second launch of units that are cut: rows a thread, workgroups.
    for L, B, rows, finish, wgs in ((1, 1, 5000, 1, 5), (8, 8, 9000, 4, 192), (1, 7, 2 ** 31 - 1, 4, 7 << 19)):
        line = subprocess.check_output([exe] + [str(x) for x in (L, B, 4, 1, 64, 1, rows)], text=True)
        got = dict(x.split("=") for x in line.split())
        assert int(got["npmax"]) > 1 and (int(got["finish"]), int(got["finish_wgs"])) == (finish, wgs), line
