"""The 8-bit verify's launch plan, run without a GPU over its sizes, and what
the built kernels reserve (not gpu)."""
import os
import re
import subprocess

import pytest

import code_objects

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def check(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("plan") / "q8_plan_check")
    subprocess.run(["g++", "-std=c++17", "-O2", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                    "-I" + os.path.join(ROOT, "include"),
                    "-I" + os.path.join(ROOT, "paper_2603_19610_amd", "csrc"),
                    os.path.join(ROOT, "tests", "plan", "q8_plan_check.cpp"), "-o", exe], check=True)

    def run(what):
        r = subprocess.run([exe, what], capture_output=True, text=True, timeout=300)
        assert r.returncode == 0, r.stdout + r.stderr
    return run


def test_plan_fits_its_workspace(check):
    check("areas")


def test_shares_hold_every_unit_once(check):
    """Workgroups take equal shares of all groups' units in a row: every unit once, a record for every piece, and the
    holders that the later kernels compute are those that wrote."""
    check("shares")


def test_waves_are_what_the_kernels_are_compiled_for(check):
    check("waves")


def test_kernels_fit_a_compute_unit():
    """A workgroup's waves start together: their registers and LDS are there."""
    seen = set()
    for name, (regs, lds) in code_objects.kernels().items():
        m = re.search(r"q8_(part|mass)_kernelILi(\d+)ELi(\d+)E", name)
        if not m:
            continue
        D, RT = int(m[2]), int(m[3])
        if m[1] == "part":
            tw, cw = (2 if RT <= 6 else 1), (4 if RT <= 4 else 2)
            waves, ring = RT * tw + 2 * cw, 2 * tw * 2 * 64 * D * 2
        else:
            rw = (RT + 2) // 3
            tw = 2 if rw <= 3 else 1
            waves, ring = rw * tw + 2, 2 * tw * 64 * D * 2
        assert -(-waves // 4) * regs <= 512 and lds + ring <= 160 * 1024, (name, waves, regs, lds)
        seen.add((m[1], D, RT))
    assert len(seen) == 40
