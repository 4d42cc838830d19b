"""The short quotients of the paged append must give the codes and scales of IEEE divisions: the same FP32 operations on the host
(C, hardware FMA), every significand of a maximum, every INT4 scale, and numbers around every border between two codes."""
import os
import shutil
import subprocess

import pytest

SRC = os.path.join(os.path.dirname(os.path.abspath(__file__)), "host", "paged_quotient_check.c")


def _cpu_has_fma():
    try:
        return " fma " in open("/proc/cpuinfo").read().replace("\n", " ")
    except OSError:
        return False


@pytest.mark.skipif(shutil.which("gcc") is None or not _cpu_has_fma(), reason="needs gcc and a CPU with FMA")
def test_short_quotients_give_the_ieee_codes(tmp_path):
    exe = str(tmp_path / "paged_quotient_check")
    subprocess.run(["gcc", "-O2", "-mfma", "-fopenmp", "-ffp-contract=off", SRC, "-o", exe, "-lm"], check=True)
    # every 61st maximum (9e8 numbers, a second or two); FQ_EXHAUSTIVE=1 runs all
    out = subprocess.run([exe, "1" if os.environ.get("FQ_EXHAUSTIVE") else "61"], capture_output=True, text=True)
    assert out.returncode == 0 and "differences 0" in out.stdout, out.stdout
