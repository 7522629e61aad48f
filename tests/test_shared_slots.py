"""Shared-prefix decode on the host, by the functions that the entry point, the kernel and
the merge use: random launches piece by piece."""

import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc")


def compiled(name, tmp_path):
    """A program of tests/shared_plan, for the host."""
    exe = str(tmp_path / name)
    subprocess.run(["hipcc", "-x", "hip", "--offload-host-only", "-O2", "-std=c++17",
                    "-I" + os.path.join(ROOT, "paper_2609_33536_amd", "csrc"),
                    os.path.join(ROOT, "tests", "shared_plan", name + ".cpp"), "-o", exe], check=True, timeout=300)
    return exe


def test_pieces_have_slots_of_their_own_and_the_merge_reads_them_all(tmp_path):
    run = subprocess.run([compiled("slots", tmp_path)], capture_output=True, text=True, timeout=300)
    assert run.returncode == 0, run.stdout
