"""Pages for lengths up to the end of the 32-bit range, by the arithmetic of bass_page_tables compiled for the host under UndefinedBehaviorSanitizer."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(shutil.which("g++") is None, reason="no host compiler")
def test_pages_of_any_length(tmp_path):
    exe = str(tmp_path / "num_pages")
    subprocess.run(["g++", "-O1", "-std=c++17", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I", os.path.join(ROOT, "paper_2404_15778_amd", "csrc"),
                    "-o", exe, os.path.join(ROOT, "tests", "host", "num_pages.cpp")], check=True, capture_output=True, text=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0 and r.stdout.startswith("ok"), r.stdout + r.stderr
