"""Host plans of the serving calls, from the library's own sources built for the host: the
launch sizes they lead to, and the forms that the GPU tests' cases are there for."""

import os
import subprocess

import pytest

from tests import serving_forms, test_gpu_rules_batches

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


@pytest.mark.parametrize("dt,vocab,times,rows", test_gpu_rules_batches.CASES)
def test_rules_cases_take_the_rows_they_are_for(plan, dt, vocab, times, rows):
    assert rules(plan, dt, vocab, test_gpu_rules_batches.SIZES * times)[0] == rows


def sets(plan, name, dt, head_dim):
    """Kinds of the sets of a case, as serving_forms.WANT names them."""
    causal = name in serving_forms.PROMPTS
    case = serving_forms.PROMPTS[name] if causal else serving_forms.TREES[name][1:]
    n_q, n_kv, L, P, shared = *case[:2], *case[-3:]
    n = serving_forms.nodes(name)
    shared = list(range(len(n))) if shared is None else shared
    words = ["walk", int(dt == "bf16"), int(causal), n_kv, n_q // n_kv, head_dim, CUS, len(n)]
    for b in range(len(n)):
        words += [n[b], L[b], P[shared.index(shared[b])], 10 ** 5 * shared[b], 10 ** 8 + 10 ** 5 * b]
    head, *rows = plan(*words)
    out = {"table"} if head[3] else set()
    for _, rb, _, _, nch, slab, _, with_packed in rows:
        out.add(("own" if slab else "packed") + ("+" if with_packed >= 0 else "") + f" {rb} " + ("cut" if nch > 1 else "whole"))
    return out


@pytest.mark.parametrize("name", list(serving_forms.WANT))
def test_cases_take_the_forms_they_are_for(plan, name):
    assert sets(plan, name, "bf16", 128) >= serving_forms.WANT[name]


def test_fp32_cases_pack(plan):
    for name in ("packed128", "packed128_table", "t16_packed128", "single_two_prefixes", "single_table"):
        got = sets(plan, name, "fp32", 48)
        assert any(s.startswith("packed 32") for s in got) and any(s.startswith("own+ 32") for s in got), name
    assert "packed 32 cut" in sets(plan, "single_two_prefixes", "fp32", 48)


@pytest.mark.parametrize("keys", [2, 300, 9000, 16000])
def test_a_lost_or_doubled_key_shows(keys):
    """The form of test_every_key_counts_once, with the mistake in the reference: some of 128 columns of values 1 and -1
    are off by more than twice the tolerance of bf16 results."""
    import numpy as np
    v = np.where(np.random.default_rng(keys).random((keys, 128)) < 0.5, 1.0, -1.0)
    ref = v.mean(0)
    for wrong in (v[1:].mean(0), (v.sum(0) + v[0]) / (keys + 1)):
        assert (np.abs(wrong - ref) > 2 * (2.0 ** -8 + 2.0 ** -22) * np.abs(ref)).sum() >= 8
