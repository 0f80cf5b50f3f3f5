"""The plan headers are plain C++ that compiles by itself, included first (g++, no GPU code)."""
import glob
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2604_22312_amd", "csrc")
HEADERS = sorted(os.path.basename(p) for p in glob.glob(os.path.join(CSRC, "*_plan.h")))


@pytest.mark.skipif(shutil.which("g++") is None, reason="no host compiler")
@pytest.mark.parametrize("header", HEADERS)
def test_header_compiles_alone(header, tmp_path):
    source = tmp_path / "alone.cpp"
    source.write_text('#include "%s"\n' % header)
    r = subprocess.run(["g++", "-std=c++17", "-Wall", "-fsyntax-only", "-I" + os.path.join(ROOT, "include"), "-I" + CSRC,
                        str(source)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
