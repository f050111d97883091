"""Ordering across a pair of CTAs in the 8-bit products (csrc/esp_fp8_gemm.cu), by the source: a stage of tensor memory
that the other CTA's warps hand back by an arrival at cluster scope is waited for at cluster scope. (A wait at CTA scope
has no ordering with an arrival from outside the CTA, whatever a run shows.)"""

import os
import re

from paper_2608_07971_gb300 import build

SRC = open(os.path.join(build.CSRC, "esp_fp8_gemm.cu")).read()


def body(name):
    m = re.search(r"__device__ __forceinline__ \w+ " + name + r"\(.*?\n}\n", SRC, re.S)
    assert m, name
    return m.group(0)


def test_arrival_and_wait_have_the_same_scope():
    assert "mbarrier.arrive.relaxed.cluster.shared::cluster" in body("mbar_arrive")
    assert "mbarrier.try_wait.parity.relaxed.cluster.shared::cta" in body("mbar_try")
    waits = re.findall(r"(mbar_wait(?:<[^>]*>)?)\(tempty ", SRC)
    assert waits == ["mbar_wait<CG == 2>"]
    # the tensor-memory fences stand on both sides: the loads before the arrival, the MMAs after the wait
    for at in (m.start() for m in re.finditer(r"mbar_arrive\(tempty0", SRC)):
        before = SRC[:at]
        assert before.rfind("fence_before();") > before.rfind("tmem_ld16(")
    after = SRC[SRC.index("mbar_wait<CG == 2>(tempty "):]
    assert after.index("fence_after();") < after.index("mma_codes<CG>(")
