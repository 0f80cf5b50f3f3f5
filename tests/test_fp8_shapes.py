"""The sizes of tests/fp8_shapes.py reach every kernel that a product's plan can choose (CPU: the plans are made here)."""
import os
import shutil
import subprocess

import pytest

from tests.fp8_shapes import NARROW, SIZES

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no host compiler")
    exe = tmp_path_factory.mktemp("plan") / "plan_fp8"
    subprocess.run(["g++", "-std=c++17", "-O2", "-I" + os.path.join(ROOT, "include"),
                    "-I" + os.path.join(ROOT, "paper_2604_22312_amd", "csrc"), os.path.join(ROOT, "tests", "c_abi", "plan_fp8.cpp"),
                    "-o", str(exe)], check=True)

    def run(lines, more=0):
        r = subprocess.run([str(exe), str(more)], input="\n".join(lines), capture_output=True, text=True, timeout=120, check=True)
        return [line.split(" ", 3) for line in r.stdout.splitlines()]
    return run


def reached(plans):
    ask = ["%d %d %d %d" % (M, N, K, wide) for M, N, K, types in SIZES for wide in (0, 1)
           if (wide and "f32" in types) or (not wide and set(NARROW) <= set(types))]
    return {p[3] for p in plans(ask)}


def test_every_kernel_is_reached(plans):
    want = {"rows,512,0,%d", "rows,1024,0,%d", "row pairs,512,0,%d", "rows32,512,0,%d"}
    want |= {"%s,256,%d,%%d" % (s, split) for s in ("low", "narrow", "square") for split in (0, 1)}
    want = {w % wide for w in want for wide in (0, 1)} | {"large,512,0,0", "large,512,1,0"}
    assert reached(plans) == want


def test_random_sizes_reach_no_other(plans):
    """200000 products over the whole range of sizes are planned with kernels that the sizes above reach."""
    there = reached(plans)
    got = plans([], 200000)
    assert len(got) == 200000
    assert {p[3] for p in got} == there
