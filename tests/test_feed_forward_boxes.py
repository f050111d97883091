"""Ordering of a warp's staging boxes in the gated feed-forward blocks (csrc/esp_ff_gemm.cu), by the source: a box that the
lanes read and write themselves is handed to a bulk copy, in either direction, by a proxy fence of every lane and a barrier
of the warp. (Without the fence the lanes' accesses and the copy's have no order, whatever a run shows.)"""

import os
import re

from paper_2608_07971_gb300 import build

SRC = open(os.path.join(build.CSRC, "esp_ff_gemm.cu")).read()
FENCE = 'asm volatile("fence.proxy.async.shared::cta;" ::: "memory");'


def handed_over(text):
    """Whether the first thing that one lane does follows the fence of all of them and the warp's barrier."""
    return text.index(FENCE) < text.index("__syncwarp();") < text.index("if (lane == 0)")


def test_boxes_are_fenced_before_a_load():
    loads = re.findall(r"load_box<CG>\(smem_u32\([gu]box\)", SRC)
    body = re.search(r"const auto load_pre = \[&\]\(int c\) \{\n(.*?)\n            \};\n", SRC, re.S).group(1)
    assert len(loads) == 2 == len(re.findall(r"load_box<CG>\(smem_u32\([gu]box\)", body))   # nowhere else
    assert handed_over(body)
    # what the lanes read out of a box is in registers, and the stores out of it have been read, before the next load
    for at in (m.start() for m in re.finditer(r"load_pre\((?:first|c \+ 32)\);", SRC)):
        assert SRC[:at].rstrip().endswith("boxes.drain();")


def test_boxes_are_fenced_before_a_store():
    stores = [m.start() for m in re.finditer(r"cp\.async\.bulk\.tensor\.3d\.global\.shared::cta", SRC)]
    assert len(stores) == 1
    body = re.search(r"void box_store\(.*?\n}\n", SRC, re.S)
    assert body.start() < stores[0] < body.end() and handed_over(body.group(0))
