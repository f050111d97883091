"""Host-side checks of the expert layer's C entry points that need no GPU: exports, null handles, no GPU."""

import ctypes
import os
import re

import pytest

from paper_2608_07971_gb300 import esp, moe

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    from paper_2608_07971_gb300 import build
    build.build()
    return moe.load_library()


def test_exports_every_declared_function(lib):
    src = open(os.path.join(ROOT, "include", "esp_moe.h")).read()
    src = re.sub(r"/\*.*?\*/", "", src, flags=re.S)
    names = set(re.findall(r"^\s*(?:const\s+)?\w+\s*\*?\s*(esp_\w+)\s*\(", src, flags=re.M))
    assert names == set(moe.EXPORTED) and len(names) >= 14
    for n in names:
        assert hasattr(lib, n), n


def test_null_handle_rejected(lib):
    bad, N = esp.ESP_ERR_INVALID_ARG, None
    gate, w, n = moe._CGate(0, 1, 1.0), moe._CWeight(), ctypes.c_int64()
    assert lib.esp_moe_create(N, -1, N) == bad
    assert lib.esp_moe_set_stream(N, N) == bad
    assert lib.esp_moe_route(N, gate, 0, 0, 1, 1, 1, N, N, N, N, N, N, N, N, N) == bad
    assert lib.esp_moe_balance(N, gate, 0, 0, 1, 1, 1, N, N, 1, N, N, N, N, N) == bad
    assert lib.esp_moe_route_backward(N, gate, 0, 0, 1, 1, 1, N, N, N, 1, N, N, N, N, 1, N) == bad
    assert lib.esp_moe_step_prices(N, 1, N, 0.1, 1.0, N) == bad
    assert lib.esp_moe_quantize_weight(N, 0, N, 1, w) == bad
    assert lib.esp_moe_linear(N, 0, 0, 1, N, 0, N, w, N, 1, N) == bad
    assert lib.esp_moe_linear_backward(N, 0, 0, 1, N, 0, N, w, N, 1, N, 1, N, 1, N) == bad
    assert lib.esp_moe_combine(N, 0, 0, 1, 1, 0, 1, N, N, N, 1, N) == bad
    assert lib.esp_moe_combine_backward(N, 0, 0, 1, 1, 0, 1, N, 1, N, N, N, 1, N, N) == bad
    assert lib.esp_moe_debug_set_wait_limit(N, 0) == bad
    assert lib.esp_moe_debug_hold_load(N) == bad
    assert lib.esp_moe_synchronize(N) == bad
    assert lib.esp_moe_last_launch_count(N, ctypes.byref(n)) == bad
    lib.esp_moe_destroy(N)


def test_create_without_gpu_is_unsupported(lib):
    import torch
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    h = ctypes.c_void_p()
    assert lib.esp_moe_create(ctypes.byref(h), -1, None) == esp.ESP_ERR_UNSUPPORTED


def test_unknown_gate_rejected():
    with pytest.raises(ValueError):
        moe.Gate("relu")
