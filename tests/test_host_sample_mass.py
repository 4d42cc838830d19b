"""A token's mass in sampling (csrc/fq_mass.h) on the host, where a conversion out of its type's range does not happen to end at the type's largest number."""
import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2505_20839_amd", "csrc")
CXX = shutil.which("g++") or shutil.which("clang++", path=os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin"))


@pytest.mark.skipif(CXX is None, reason="needs a C++ compiler")
def test_masses_of_every_share(tmp_path):
    exe = str(tmp_path / "sample_mass_check")
    subprocess.run([CXX, "-O1", "-std=c++17", "-I", CSRC, os.path.join(HERE, "host", "sample_mass_check.cpp"), "-o", exe], check=True)
    out = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert out.returncode == 0 and "wrong 0" in out.stdout, out.stdout
