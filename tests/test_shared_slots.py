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


def test_the_cases_of_the_gpu_tests_reach_their_paths(tmp_path):
    from tests.shared_plan.cases import CASES
    exe = compiled("plan", tmp_path)
    for name, (hq, hkv, prefix, start, own, _, want) in CASES.items():
        for bytes8 in (0, 1):
            counts = [b - a for a, b in zip(start, start[1:])]
            blocks = [-(-max(lens) // 16) for lens in (prefix, own)]
            text = [hkv, hq // hkv, bytes8, *blocks, start[0], len(prefix), *(x for pair in zip(counts, prefix) for x in pair), len(own), *own]
            run = subprocess.run([exe], input=" ".join(map(str, text)), capture_output=True, text=True, timeout=60)
            assert run.returncode == 0, name
            plan = {k: int(v) for k, v in (x.split("=") for x in run.stdout.split())}
            assert eval(want, {}, plan), (name, bytes8, want, plan)
