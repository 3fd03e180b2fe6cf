"""Host plans of the serving calls, from the library's own sources built for the host: the
launch sizes they lead to, and the forms that the GPU tests' cases are there for."""

import os
import subprocess

import numpy as np
import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(ROOT, "paper_2506_01986_amd", "csrc")
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")
CUS, GRID_Y = 256, 65536                  # compute units, blocks in y of the largest launch (hipDeviceProp_t::maxGridSize)


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("plan") / "serving_plan")
    r = subprocess.run(["g++", "-std=c++17", "-O2", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROCM, "include"), "-I",
                        os.path.join(ROOT, "include"), "-I", CSRC, os.path.join(HERE, "c", "serving_plan.cpp"),
                        os.path.join(CSRC, "walk_plan.cpp"), "-o", exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stderr[-4000:]

    def ask(*words):
        r = subprocess.run([exe], input=" ".join(str(w) for w in words), capture_output=True, text=True, timeout=60)
        assert r.returncode == 0, r.stderr
        return [[int(v) for v in line.split()] for line in r.stdout.splitlines()]

    return ask


def rules(plan, dt, vocab, sizes):
    """(node rows a block, blocks in y) of the logit rules over trees of these sizes."""
    return plan("rules", {"fp32": 1024, "bf16": 2048}[dt], vocab, len(sizes), sum(sizes), max(sizes), CUS)[0]


@pytest.mark.parametrize("dt", ["fp32", "bf16"])
@pytest.mark.parametrize("vocab", [1, 1000, 3000, 32000])
def test_rules_launches_fit(plan, dt, vocab):
    """One large tree among many small ones: the row groups of the largest tree times the sequences."""
    for B in sorted({1, 2, 100, 511, 512, 513, 1023, 1024, 1025, 2000, 2047, 2048, 3899, 3968, 3969, 4095, 4096}):
        for big in (1, 2, 9, 64, 127, 128):
            rows, y = rules(plan, dt, vocab, [big] + [1] * (B - 1))
            assert 1 <= rows <= 8 and y <= GRID_Y, (B, big, rows, y)


def test_rules_rows_fill_the_chip(plan):
    assert rules(plan, "bf16", 32000, [64] * 10) == [8, 80]
    assert rules(plan, "bf16", 8263, [63] * 8) == [4, 128]
    assert rules(plan, "fp32", 1000, [16]) == [1, 16]
