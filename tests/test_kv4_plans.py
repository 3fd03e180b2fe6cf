"""Host plans of the attention over 4-bit pools: the forms that its tests' batches are there for, and that every key of
every row block has its chunk."""

import os
import subprocess

import pytest

from tests import serving_forms
from tests.kv4_forms import MERGES

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(ROOT, "paper_2506_01986_amd", "csrc")
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")
CUS = 256
NAMES = ("T", "L", "P", "rb", "nrb", "ct", "nch", "tiles", "slab", "parts", "shared", "part0", "items")


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("plan") / "kv4_plan")
    r = subprocess.run(["g++", "-std=c++17", "-O2", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROCM, "include"), "-I",
                        os.path.join(ROOT, "include"), "-I", CSRC, os.path.join(HERE, "c", "kv4_plan.cpp"),
                        os.path.join(CSRC, "walk_plan.cpp"), "-o", exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stderr[-4000:]

    def ask(dtype, causal, n_q, n_kv, d, n, L, P, shared):
        shared = list(range(len(n))) if shared is None else shared
        words = [int(dtype == "bf16"), int(causal), n_kv, n_q // n_kv, d, CUS, len(n)]
        for b in range(len(n)):
            words += [n[b], L[b], P[shared.index(shared[b])], 10 ** 5 * shared[b], 10 ** 8 + 10 ** 5 * b]
        r = subprocess.run([exe], input=" ".join(str(w) for w in words), capture_output=True, text=True, timeout=60)
        assert r.returncode == 0, r.stderr
        *sets, total = [[int(v) for v in line.split()] for line in r.stdout.splitlines()]
        return [dict(zip(NAMES, s)) for s in sets], total

    return ask


def sound(sets, total, n_q, n_kv, n):
    g = n_q // n_kv
    own = [s for s in sets if s["slab"]]
    assert sorted(s["T"] for s in own) == sorted(x for x in n if x)
    parts = []
    for s in sets:
        assert s["nrb"] * s["rb"] >= s["T"] * g > (s["nrb"] - 1) * s["rb"]
        assert s["nch"] * s["ct"] >= s["tiles"] > (s["nch"] - 1) * s["ct"]         # chunks cover the longest block, none is empty
        if s["nch"] > 1 or s["parts"]:
            parts.append((s["part0"], s["items"] * n_kv * s["rb"] // 32))
    assert sum(s["items"] for s in sets) * n_kv == total[0]
    at = 0
    for part0, many in sorted(parts):                                              # side by side, without gaps
        assert part0 == at
        at += many
    assert at == total[1]


def case(name):
    causal = name in serving_forms.PROMPTS
    c = serving_forms.PROMPTS[name] if causal else serving_forms.TREES[name][1:]
    return causal, c[0], c[1], serving_forms.nodes(name), *c[-3:]


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("fp32", 32), ("fp32", 96)])
@pytest.mark.parametrize("name", list(serving_forms.WANT))
def test_plans_are_sound(plan, name, dtype, d):
    causal, n_q, n_kv, n, L, P, shared = case(name)
    sets, total = plan(dtype, causal, n_q, n_kv, d, n, L, P, shared)
    sound(sets, total, n_q, n_kv, n)
    for s in sets:
        rows = s["T"] * n_q // n_kv
        assert s["rb"] in ((32,) if dtype == "fp32" or rows <= 16 else (64, 128))    # the forms of the kernel


def test_few_rows_beside_long_prompts(plan):
    """One chunk of a prompt among single tokens, as a server has them."""
    n, L = [2048] + [1] * 32, [2048] + [4000] * 32
    sets, total = plan("bf16", True, 64, 8, 128, n, L, [0] * 33, None)
    sound(sets, total, 64, 8, n)
    assert {s["rb"] for s in sets} == {32, 128}


@pytest.mark.parametrize("d", [32, 64, 96, 128])
@pytest.mark.parametrize("name", list(MERGES))
def test_batches_that_merge(plan, name, d):
    n_q, n_kv, n, L, P, shared = MERGES[name]
    sets, total = plan("fp32", True, n_q, n_kv, d, n, L, P, shared)
    sound(sets, total, n_q, n_kv, n)
    assert ("packed" in name) == any(s["shared"] >= 0 for s in sets)
    assert name == "packed" or any(s["nch"] > 1 for s in sets)
