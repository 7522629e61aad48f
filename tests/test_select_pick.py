"""The pick of block selection on the host: its keys and bins compiled for the CPU and
driven with random scores, infinite and undefined ones among them."""

import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc")


def _run(tmp_path, *flags):
    exe = str(tmp_path / "check")
    subprocess.run(["hipcc", "-x", "hip", "--offload-host-only", "-O2", "-std=c++17", *flags,
                    "-I" + os.path.join(ROOT, "paper_2609_33536_amd", "csrc"),
                    os.path.join(ROOT, "tests", "select_pick", "check.cpp"), "-o", exe], check=True, timeout=300)
    return subprocess.run([exe], capture_output=True, text=True, timeout=300)


def test_the_largest_scores_are_picked_and_never_more(tmp_path):
    run = _run(tmp_path)
    assert run.returncode == 0, run.stdout


def test_the_walk_finds_bins_whose_end_wraps(tmp_path):
    assert _run(tmp_path, "-DWRAPPING").returncode == 1
