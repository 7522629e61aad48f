"""How shared-prefix decode divides its workgroups and counts its slots, on the host: the
header's division compiled for the CPU and driven with random batches."""

import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc")
def test_division_covers_the_work_and_fits_the_workspace(tmp_path):
    exe = str(tmp_path / "check")
    subprocess.run(["hipcc", "-x", "hip", "--offload-host-only", "-O2", "-std=c++17",
                    "-I" + os.path.join(ROOT, "paper_2609_33536_amd", "csrc"),
                    os.path.join(ROOT, "tests", "shared_plan", "check.cpp"), "-o", exe], check=True, timeout=300)
    run = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert run.returncode == 0, run.stdout
