"""Lengths at the ends of the 32-bit range are clamped as the header promises, by the arithmetic that all planners share (compiled for the
host under UndefinedBehaviorSanitizer), and by the host planner through the C ABI."""
import os
import shutil
import subprocess

import numpy as np
import pytest

import paper_2404_15778_amd as bass

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
TOP = 2 ** 31 - 1


def clamp(L, n, kmax, Lcap):
    """0 <= n <= min(kmax, Lcap), 0 <= L <= Lcap - n, in whole numbers without bounds."""
    q = min(max(n, 0), kmax, Lcap)
    l = min(max(L, 0), Lcap - q)
    return l, q, int((l, q) != (L, n))


@pytest.mark.skipif(shutil.which("g++") is None, reason="no host compiler")
def test_the_shared_arithmetic(tmp_path):
    exe = str(tmp_path / "clamp_lengths")
    subprocess.run(["g++", "-O1", "-std=c++17", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I", os.path.join(ROOT, "paper_2404_15778_amd", "csrc"),
                    "-o", exe, os.path.join(ROOT, "tests", "host", "clamp_lengths.cpp")], check=True, capture_output=True, text=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stderr
    lines = r.stdout.splitlines()
    assert len(lines) == 5 * 3 * 7 * 13
    for line in lines:
        given, got = (tuple(map(int, part.split())) for part in line.split("->"))
        assert got == clamp(*given), line


@pytest.mark.parametrize("L", [TOP, TOP - 1, TOP - 3, TOP - 4, 1000, 997, -TOP - 1])
def test_one_bad_length_leaves_the_other_sequences_alone(L):
    """The host planner: the same plan as for the length that the bad one is clamped to."""
    desc = bass.make_desc(3, 4, 8, 2, 128, 1000, "bf16", 0.1)
    plan, status = bass.bass_attention_plan_host(desc, [100, L, 640], [4, 4, 2])
    want, fine = bass.bass_attention_plan_host(desc, [100, clamp(L, 4, 4, 1000)[0], 640], [4, 4, 2])
    assert (status, fine) == (bass.STATUS_LEN_CLAMPED, 0)
    plan, want = (np.asarray(p).view(np.int32).copy() for p in (plan, want))
    plan[12] = want[12]  # the header's word that says whether a length was clamped
    assert np.array_equal(plan, want)
