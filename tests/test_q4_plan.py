"""The 4-bit attention's launch plan, run without a GPU over its sizes, and what the
built kernels reserve (not gpu)."""
import os
import re
import subprocess

import pytest

import code_objects

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def check(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("plan") / "q4_plan_check")
    subprocess.run(["g++", "-std=c++17", "-O2", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                    "-I" + os.path.join(ROOT, "include"),
                    "-I" + os.path.join(ROOT, "paper_2603_19610_amd", "csrc"),
                    os.path.join(ROOT, "tests", "plan", "q4_plan_check.cpp"), "-o", exe], check=True)

    def run(what):
        r = subprocess.run([exe, what], capture_output=True, text=True, timeout=300)
        assert r.returncode == 0, r.stdout + r.stderr
    return run


def test_plan_fits_its_workspace(check):
    check("areas")


def test_waves_and_runs_are_what_the_kernels_are_compiled_for(check):
    check("waves")


def test_kernels_fit_a_compute_unit():
    """A workgroup's waves start together: their registers and LDS are there."""
    seen = set()
    for name, (regs, lds) in code_objects.kernels().items():
        m = re.search(r"q4_(part|mass)_kernelILi(\d+)ELi(\d+)E(?:Lb([01])E)?", name)
        if not m:
            continue
        D, tiles = int(m[2]), int(m[3])
        # LDS of the waves' values: 32 rows of bf16 with their padding each
        ring = 8 * 32 * (2 * D + 32) if m[1] == "part" else 0
        waves = 4 if m[1] == "mass" and tiles <= 3 else 2
        assert waves * regs <= 512 and lds + ring <= 160 * 1024, (name, regs, lds, ring)
        seen.add((m[1], D, tiles, m[4]))
    assert len([x for x in seen if x[0] == "part"]) == 12 and len([x for x in seen if x[0] == "mass"]) == 10
