"""The expert layer's host code without a GPU: its handle against a fake CUDA runtime (work space under captured graphs,
the order of work across streams, failures: tests/moe_handle_driver.cpp), kernels' shared-memory limits
(tests/moe_smem_driver.cpp), the products' work items (tests/moe_tiles_driver.cpp)."""

import os
import subprocess

import pytest

from paper_2608_07971_gb300 import build

HERE = os.path.dirname(os.path.abspath(__file__))

CHECKS = [
    "graph_keeps_its_block",
    "growing_while_captured",
    "handles_beside_a_capture",
    "order_across_a_capture",
    "order_after_a_capture_in_place",
    "synchronize_across_a_capture",
    "timeout_is_reported_by_the_next_call",
]


def compiled(out, *sources):
    cuda = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(build.nvcc()))), "include")
    subprocess.run(["g++", "-std=c++17", "-g", "-O1", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                    "-I", build.INCLUDE, "-I", build.CSRC, "-I", cuda, "-x", "c++", *sources, "-o", out, "-lpthread"],
                   check=True, capture_output=True, text=True)
    return out


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    return compiled(str(tmp_path_factory.mktemp("moe_handle") / "driver"), os.path.join(build.CSRC, "esp_moe.cu"),
                    os.path.join(HERE, "moe_handle_driver.cpp"))


def test_every_check_is_listed(driver):
    res = subprocess.run([driver], capture_output=True, text=True)
    assert res.returncode == 2 and res.stdout.split() == sorted(CHECKS)


@pytest.mark.parametrize("name", CHECKS)
def test_handle(driver, name):
    res = subprocess.run([driver, name], capture_output=True, text=True)
    assert (res.returncode, res.stdout) == (0, "ok\n"), res.stdout + res.stderr


def test_shared_memory_limit(tmp_path):
    """One limit per kernel, its greatest, also where two threads set it at once."""
    out = compiled(str(tmp_path / "driver"), os.path.join(HERE, "moe_smem_driver.cpp"))
    res = subprocess.run([out], capture_output=True, text=True, timeout=60)
    assert (res.returncode, res.stdout) == (0, "ok\n"), res.stdout + res.stderr


def test_work_items_stay_in_range(tmp_path):
    """The products' work items cover every row once, and stay in bounds for offsets that do not ascend."""
    out = compiled(str(tmp_path / "driver"), os.path.join(HERE, "moe_tiles_driver.cpp"))
    res = subprocess.run([out], capture_output=True, text=True, timeout=120)
    assert (res.returncode, res.stdout) == (0, "ok\n"), res.stdout + res.stderr
