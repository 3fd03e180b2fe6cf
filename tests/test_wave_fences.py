"""Data that a wave's lanes pass one another through LDS without a barrier (csrc/kv4_attn.hip, walk4_few: V, converted by
some lanes, multiplied by others).  The compiler sees one lane's accesses alone; a wave-level fence tells it to keep the
order of the stores and the loads."""

import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2506_01986_amd", "csrc")


def test_v_of_a_wave_is_fenced():
    text = re.sub(r"//.*", "", open(os.path.join(CSRC, "kv4_attn.hip")).read())
    body = text[text.index("walk4_few("):text.index("walk4_attn_bf16(")]
    at = [(m.start(), m.group()) for m in re.finditer(r"few_swz\(r,|ds_read_tr16_b64|wave_fence\(\)|part \+ \(\(4|__syncthreads", body)]
    kinds = "".join({"few_swz(r,": "s", "ds_read_tr16_b64": "l", "wave_fence()": "f", "part + ((4": "p", "__syncthreads": "b"}[k] for _, k in at)
    # stores of V, fence, loads of it, fence (before the next tile's stores and the parts', which take its place), parts, barrier
    assert kinds == "sfllfpb", kinds


def test_the_fence_orders_a_wave():
    text = open(os.path.join(CSRC, "device.h")).read()
    body = text[text.index("void wave_fence()"):]
    body = body[:body.index("}\n")]
    assert re.search(r'__ATOMIC_RELEASE, "wavefront".*wave_barrier\(\).*__ATOMIC_ACQUIRE, "wavefront"', body, re.S)
