"""Tokens of the append's and the reading's launches, up to the largest total that the calls take (2^31 - 1)."""

import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(ROOT, "paper_2506_01986_amd", "csrc")
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")


def test_tokens_stay_within_32_bits(tmp_path):
    exe = str(tmp_path / "rows_token")
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-ftrapv", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROCM, "include"), "-I",
                        os.path.join(ROOT, "include"), "-I", CSRC, os.path.join(HERE, "c", "rows_token.cpp"), "-o", exe],
                       capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stderr[-4000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, (r.returncode, r.stdout)


def test_kernels_take_their_tokens_so():
    """No kernel forms a token as the launch's first plus a thread's place: that sum passed 2^31 - 1 in the last block."""
    text = open(os.path.join(CSRC, "kv_rows.hip")).read()
    assert text.count("rows_token(a.tok0, a.tok1, ") >= 4 and "a.tok0 +" not in text
