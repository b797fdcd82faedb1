"""The arithmetic by which the 8-bit verify's kernels find their shares: the
kernels' own functions, run without a GPU (not gpu)."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def check(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("shares") / "q8_shares_check")
    subprocess.run(["g++", "-std=c++17", "-O2", "-fsanitize=signed-integer-overflow", "-fno-sanitize-recover=all",
                    "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I" + os.path.join(ROOT, "include"),
                    "-I" + os.path.join(ROOT, "paper_2603_19610_amd", "csrc"),
                    os.path.join(ROOT, "tests", "plan", "q8_shares_check.cpp"), "-o", exe], check=True)

    def run(what):
        return subprocess.run([exe, what], capture_output=True, text=True, timeout=300)
    return run


@pytest.mark.parametrize("what", ["ragged", "extremes"])
def test_the_kernels_shares_hold_every_token_once(check, what):
    r = check(what)
    assert r.returncode == 0, r.stdout + r.stderr


def test_a_workspace_does_not_grow_with_the_capacity(check):
    """64 decoding sequences of 16384 tokens with room for 131072 once reserved 282 MB, 268 of them never touched."""
    r = check("workspace")
    assert r.returncode == 0, r.stdout + r.stderr


def test_a_planted_slip_is_seen(check):
    r = check("planted")
    assert r.returncode == 1 and "plans" in r.stdout, r.stdout + r.stderr


def test_the_kernels_have_no_shares_of_their_own():
    """The checked functions are those that the kernels call."""
    src = open(os.path.join(ROOT, "paper_2603_19610_amd", "csrc", "q8_attn.hip")).read()
    assert "q8_find<true>(a, Wave(a), blockIdx.x, 0)" in src and "q8_find<false>(a, Wave(a), 0, b)" in src
    assert "holders(a, p.per" in src and "struct Piece : QPiece" in src
    for own in ("struct Shares", "Holders holders(", "int aligned(", "int units_of("):
        assert own not in src, own
