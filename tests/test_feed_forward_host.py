"""Host-side checks of the gated feed-forward blocks and of clipping that need no GPU: null handles, weights and lists of
gradients that are refused, the products' work items (tests/ff_tiles_driver.cpp)."""

import copy
import ctypes
import os
import pickle
import re
import subprocess

import pytest
import torch

from paper_2608_07971_gb300 import build, esp, moe

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def lib():
    build.build()
    return moe.load_library()


def test_null_handle_rejected(lib):
    bad, N = esp.ESP_ERR_INVALID_ARG, None
    w, k, t = moe._CGated(), moe._CKept(), (moe._CTensor * 1)()
    assert lib.esp_moe_feed_forward(N, w, 0, 1, N, 0, N, N, 1, N, k) == bad
    assert lib.esp_moe_feed_forward_backward(N, w, 0, 1, N, 0, N, N, k, 1, N, 1, N, 0, N, N) == bad
    assert lib.esp_moe_clip(N, 1, t, 1.0, 1.0, N) == bad


def test_work_items_stay_in_range(tmp_path):
    cuda = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(build.nvcc()))), "include")
    out = str(tmp_path / "driver")
    subprocess.run(["g++", "-std=c++17", "-g", "-O1", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                    "-I", build.INCLUDE, "-I", build.CSRC, "-I", cuda, os.path.join(HERE, "ff_tiles_driver.cpp"), "-o", out],
                   check=True, capture_output=True, text=True)
    res = subprocess.run([out], capture_output=True, text=True, timeout=120)
    assert (res.returncode, res.stdout) == (0, "ok\n"), res.stdout + res.stderr


def test_matrices_that_meet(tmp_path):
    out = str(tmp_path / "driver")
    subprocess.run(["g++", "-std=c++17", "-g", "-O1", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                    "-I", build.CSRC, os.path.join(HERE, "spans_driver.cpp"), "-o", out], check=True, capture_output=True, text=True)
    res = subprocess.run([out], capture_output=True, text=True, timeout=120)
    assert (res.returncode, res.stdout) == (0, "ok\n"), res.stdout + res.stderr


def weights(E=2, F=16, H=24, dtype=torch.bfloat16):
    return torch.zeros(E, 2 * F, H, dtype=dtype), torch.zeros(E, H, F, dtype=dtype)


def test_weights_are_checked():
    inner, outer = weights()
    w = moe.GatedWeight(inner, outer, "gelu")
    assert (w.E, w.F, w.H) == (2, 16, 24)
    odd = torch.zeros(2, 32, 23, dtype=torch.bfloat16)
    for a, b, act in ((inner, outer, "tanh"), (inner, outer[:1], "silu"), (inner[:, :31], outer, "silu"), (inner, outer.half(), "silu"),
                      (inner.float(), outer.float(), "silu"), (inner[0], outer[0], "silu"), (inner[:, :, ::2], outer[:, ::2], "silu"),
                      (odd, torch.zeros(2, 23, 16, dtype=torch.bfloat16), "silu"), (inner[:0], outer[:0], "silu"),
                      (inner.transpose(1, 2), outer, "silu")):
        with pytest.raises(ValueError):
            moe.GatedWeight(a, b, act)


def test_assigned_weights_are_checked_anew():
    inner, outer = weights()
    w = moe.GatedWeight(inner, outer)
    w._arg()
    w.outer = outer[:, :8]
    with pytest.raises(ValueError):
        w._arg()
    w.outer = outer
    w.activation = "relu"
    assert w._arg() is not None and w._c.activation == 3
    w.inner.data = torch.ones_like(inner)   # moved
    w._arg()
    assert w._c.inner == w.inner.data_ptr()


def test_weights_can_be_copied():
    w = moe.GatedWeight(*weights(), "gelu_tanh")
    for v in (copy.copy(w), copy.deepcopy(w), pickle.loads(pickle.dumps(w))):
        assert v.activation == "gelu_tanh" and torch.equal(v.inner, w.inner) and v._c.inner == v.inner.data_ptr()


def test_weights_of_padded_rows():
    room = torch.zeros(2, 32, 64, dtype=torch.float16)[:, :, :23]
    w = moe.GatedWeight(room, torch.zeros(2, 23, 16, dtype=torch.float16))
    assert w.H == 23 and w._c.ld_inner == 64 and w._c.ld_outer == 16


def test_lists_of_gradients_are_checked():
    g = [torch.zeros(4), torch.zeros(3, dtype=torch.bfloat16)]
    li = moe.Gradients(g, None, -1)   # -1: tensors on the CPU
    assert len(li._arg()) == 2 and li._arg()[1].dtype == 1 and li._arg()[1].out == g[1].data_ptr()
    for tensors, out in (([torch.zeros(4).double()], None), ([torch.zeros(4, 4).t()], None), (g, g[:1]), (g, [g[0], g[1].float()]),
                         ([torch.zeros(4)], [torch.zeros(5)])):
        with pytest.raises(ValueError):
            moe.Gradients(tensors, out, -1)
    with pytest.raises(ValueError):
        moe.Gradients(g, None, 0)
    assert ctypes.sizeof(moe._CTensor) == 32


def test_weights_of_another_shape_in_place():
    """``.data`` at the same address: what is told to the library is what the tensors are now, or the call is refused."""
    inner, outer = weights()
    w = moe.GatedWeight(inner, outer)
    at = inner.data_ptr(), outer.data_ptr()
    inner.data, outer.data = inner.data[:1], outer.data[:1]
    w._arg()
    assert (w._c.inner, w._c.outer) == at and (w._c.E, w.E) == (1, 1)
    inner.data, outer.data = (t.data.view(torch.float16) for t in (inner, outer))
    w._arg()
    assert w._c.dtype == moe._DTYPES[torch.float16]
    room = torch.zeros(1, 32, 32, dtype=torch.float16)
    inner.data = room[:, :, :24]
    w._arg()
    assert w._c.ld_inner == 32
    inner.data = room.flatten()[:32 * 24].view(1, 32, 24)
    w._arg()
    assert w._c.ld_inner == 24 and w._c.inner == room.data_ptr()
    outer.data = outer.data[:, :8]
    with pytest.raises(ValueError):
        w._arg()


def test_weights_assigned_with_other_sizes():
    """E, F and H follow the tensors before rows and offsets are checked against them."""
    w = moe.GatedWeight(*weights())
    w.inner, w.outer = weights(E=3, F=8, H=40)
    m = object.__new__(moe.Moe)   # no handle: the checks alone
    m.h, m._index, m.device, m._side = None, -1, torch.device("cpu"), None
    x, offsets = torch.zeros(5, 40, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int32)
    assert m._block_rows(x, w, offsets, None) == (5, 40) and (w.E, w.F, w.H) == (3, 8, 40)
    w.inner, w.outer = weights()
    for x1, offsets1 in ((x, offsets), (x, offsets[:3]), (x[:, :24], offsets)):
        with pytest.raises(ValueError):
            m._block_rows(x1, w, offsets1, None)
    w.inner, w.outer = weights(F=80)
    assert m.keep(2, w).pre.shape == (2, 2, 128)


def test_codes_of_another_shape_in_place():
    q, s = torch.zeros(2, 10, 32, dtype=torch.uint8), torch.zeros(2, 1, 1)
    w = moe.Weight(2, 10, 20, q, s)
    w._arg()
    q.data = q.data[:1]
    with pytest.raises(ValueError):
        w._arg()
    q.data = torch.zeros(2, 10, 64, dtype=torch.uint8)
    w._arg()
    assert w._c.ld == 64
    s.data = s.data.view(torch.int32)
    with pytest.raises(ValueError):
        w._arg()


def test_gradients_of_another_length_in_place():
    a, b, o = torch.zeros(100), torch.zeros(6, 4), torch.zeros(6, 4)
    li, to = moe.Gradients([a, b], None, -1), moe.Gradients([b], [o], -1)
    a.data = a.data[:10]
    assert (li._arg()[0].n, li._arg()[0].grad) == (10, a.data_ptr())
    a.data = a.data.view(torch.bfloat16)
    assert (li._arg()[0].n, li._arg()[0].dtype) == (20, moe._DTYPES[torch.bfloat16])
    o.data = o.data[:3]
    with pytest.raises(ValueError):
        to._arg()
    o.data = torch.zeros(6, 4)
    assert to._arg()[0].out == o.data_ptr()
    room = torch.zeros(6, 8)
    b.data = room.flatten()[:24].view(6, 4)
    assert to._arg()[0].grad == room.data_ptr()
    b.data = room[:, :4]   # the same address, not contiguous
    for v in (li, to):
        with pytest.raises(ValueError):
            v._arg()


def test_clip_counts_its_chunks_in_32_bits():
    """By the source: the limit that the header states is the one that is checked, and a launch's chunks at it, with the
    steps past the last one, stay within int32."""
    src = open(os.path.join(build.CSRC, "esp_moe_clip.cu")).read()
    bits = int(re.search(r"kMostBytes = \(int64_t\)1 << (\d+);", src).group(1))
    assert f"2^{bits} bytes in all" in open(os.path.join(build.INCLUDE, "esp_moe.h")).read()
    number = {n: int(v) for n, v in re.findall(r"\b(k\w+) = (\d+)\b(?! <<)", src)}
    least = re.search(r"launch_clip<8, (\w+), N>", src).group(1)   # groups of a thread in k_scale's chunk
    chunk = 16 * number["kThreads"] * (int(least) if least.isdigit() else number[least])
    ctas = 1024 * number["kScaleCtas"]   # a step, on more SMs than any GPU has
    assert (1 << bits) // chunk + 2 * number["kManyTensors"] + ctas < 1 << 31
