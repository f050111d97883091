"""Handles of the expert layer on the GPU: captured graphs beside direct calls, streams, work space."""

import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def moe():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2608_07971_gb300 import build, moe
    build.build()
    return moe


def test_graph_outlives_growing_work_space(moe):
    """A step captured for a few tokens replays with the same results after calls that need far more work space."""
    m = moe.Moe()
    g = torch.Generator(device="cuda").manual_seed(0)
    x, z = torch.randn(150, 2048, generator=g, device="cuda").bfloat16(), torch.randn(150, 16, generator=g, device="cuda")
    q = m.quantize_weight(torch.randn(16, 256, 2048, generator=g, device="cuda"))
    r, y = m.routing(150, 16, 4), torch.empty(600, 256, dtype=torch.bfloat16, device="cuda")

    def step():
        m.route(z, 4, out=r)
        m.linear(x, q, offsets=r.offsets, rows=r.rows, out=y)

    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        step()
    torch.cuda.synchronize()
    want = (y.clone(), r.pos.clone())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        step()
    for T in (3000, 20000):
        big = m.route(torch.randn(T, 16, generator=g, device="cuda"), 4)
        m.linear(torch.randn(T, 2048, generator=g, device="cuda"), q, offsets=big.offsets, rows=big.rows)
        fill = torch.full((64 << 20,), 255, dtype=torch.uint8, device="cuda")   # memory that was freed is used again
        y.zero_()
        r.pos.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want[0]) and torch.equal(r.pos, want[1]) and bool((fill == 255).all())
    m.synchronize()
    del graph
    m.close()


def test_captured_call_that_needs_more_work_space(moe):
    """It gets it; the capture, its graph and the handle go on."""
    g = torch.Generator(device="cuda").manual_seed(1)
    z, big = torch.randn(700, 32, generator=g, device="cuda"), torch.randn(30000, 32, generator=g, device="cuda")
    other = moe.Moe()
    want, want_big = other.route(z, 3), other.route(big, 3)
    for first in (False, True):
        m = moe.Moe()
        r, rb = m.routing(700, 32, 3), m.routing(30000, 32, 3)
        if first:
            m.route(z, 3, out=r)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            m.route(z, 3, out=r)
            m.route(big, 3, out=rb)
        m.route(torch.randn(90000, 32, device="cuda"), 3)
        r.rows.zero_()
        rb.rows.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(r.rows, want.rows) and torch.equal(r.weight, want.weight)
        assert torch.equal(rb.rows, want_big.rows) and torch.equal(rb.pos, want_big.pos)
        m.synchronize()
        del graph
        m.close()
    other.close()


def test_order_across_a_capture(moe):
    """Work on one stream, a capture on a second, work on a third, with no wait of the program's: the calls that are
    not captured share the work space one after the other."""
    m, other = moe.Moe(), moe.Moe()
    g = torch.Generator(device="cuda").manual_seed(2)
    x, y, z = (torch.randn(n, 64, generator=g, device="cuda") for n in (40000, 500, 30000))
    want = [other.route(v, 4) for v in (x, y, z)]
    a, b, c = (torch.cuda.Stream() for _ in range(3))
    r = [m.routing(v.shape[0], 64, 4) for v in (x, y, z)]
    for v, out in zip((x, y, z), r):
        m.route(v, 4, out=out)
    torch.cuda.synchronize()
    for _ in range(3):
        for out in r:
            for t in (out.rows, out.pos, out.counts):
                t.zero_()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.stream(a):
            torch.cuda._sleep(20_000_000)
            m.route(x, 4, out=r[0])
        with torch.cuda.stream(b):
            graph.capture_begin()
            m.route(y, 4, out=r[1])
            graph.capture_end()
        with torch.cuda.stream(c):
            m.route(z, 4, out=r[2])
        m.synchronize()
        for i in (0, 2):
            assert torch.equal(r[i].rows, want[i].rows) and torch.equal(r[i].pos, want[i].pos)
            assert torch.equal(r[i].counts, want[i].counts)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(r[1].rows, want[1].rows)
    m.close()
    other.close()


def test_first_call_at_the_default_shared_memory_limit(moe):
    """In a process of their own, the sizes whose dynamic shared memory alone would fit the default limit: static
    memory counts too (625 experts: 49,100 bytes and 64)."""
    code = """
import torch
from paper_2608_07971_gb300 import moe
m = moe.Moe()
for E in (624, 625, 626, 1024, 625):
    for dt in (torch.float32, torch.bfloat16, torch.float16):
        z = torch.randn(4, E, device="cuda").to(dt)
        r = m.route(z, 2)
        assert torch.equal(r.idx.long(), torch.sort(z, dim=1, descending=True, stable=True)[1][:, :2]), (E, dt)
        z = torch.randn(600, E, device="cuda").to(dt)
        b = m.balance(z, m.route(z, 2).idx)
        assert int(b.counts.sum()) == 1200
m.synchronize()
print("ok")
"""
    res = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, cwd=ROOT, timeout=200)
    assert res.returncode == 0 and res.stdout.strip() == "ok", res.stdout + res.stderr


def delayed(stream):
    """Keeps `stream` busy for some tens of milliseconds."""
    with torch.cuda.stream(stream):
        torch.cuda._sleep(100_000_000)


@pytest.mark.parametrize("busy", ["current", "own"])
def test_handle_with_a_stream_of_its_own(moe, busy):
    """What its calls allocate, fill and lay out is ordered with its kernels, whatever the caller's current stream is
    at; results are those of a handle that follows it."""
    s = torch.cuda.Stream()
    m, other = moe.Moe(stream=s.cuda_stream), moe.Moe()
    g = torch.Generator(device="cuda").manual_seed(3)
    T, k, H = 600, 4, 512
    y, d = (torch.randn(n, H, generator=g, device="cuda") for n in (T * k, T))
    pos = torch.randperm(T * k, generator=g, device="cuda").int().view(T, k)
    pos[::7, 1] = -1
    w = torch.rand(T, k, generator=g, device="cuda")
    q = other.quantize_weight(torch.randn(3, 50, 77, generator=g, device="cuda"), transposed=True)
    codes = q.codes().contiguous()
    x, off = torch.randn(9, 77, generator=g, device="cuda"), torch.tensor([0, 2, 2, 9], device="cuda").int()
    dz = torch.randn(9, 50, generator=g, device="cuda")

    def calls(h):
        v = h.load_weight(codes, q.scale, transposed=True)
        return (*h.combine_backward(d, y, pos, w), h.linear(x, v, offsets=off), *h.linear_backward(dz, x, v, offsets=off),
                h.combine(y, pos, w))

    want = calls(other)
    calls(m)   # kernels are loaded, memory is there
    m.synchronize()
    torch.cuda.synchronize()
    delayed(torch.cuda.current_stream() if busy == "current" else s)
    got = calls(m)
    m.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    torch.cuda.synchronize()   # nothing of the calls was left on the current stream
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    m.close()
    other.close()


def test_results_on_a_stream_of_its_own_share_no_memory_in_use(moe):
    """Memory freed on the current stream, but read there by queued work, is not a result's on another stream; nor the
    other way round."""
    s = torch.cuda.Stream()
    m = moe.Moe(stream=s.cuda_stream)
    n = 1 << 16
    y, pos = torch.full((n, 64), 3.0, device="cuda"), torch.arange(n, device="cuda").int().view(-1, 1)
    a, out = torch.ones(n, 64, device="cuda"), torch.zeros(n, 64, device="cuda")
    out.copy_(a)
    m.combine(y, pos)
    out.zero_()
    torch.cuda.synchronize()
    delayed(torch.cuda.current_stream())
    out.copy_(a)
    del a
    r = m.combine(y, pos)
    m.synchronize()
    torch.cuda.synchronize()
    assert bool((out == 1).all()) and bool((r == 3).all())
    del r
    torch.cuda.synchronize()
    delayed(s)
    r = m.combine(y, pos)
    del r
    b = torch.full((n, 64), 5.0, device="cuda")
    m.synchronize()
    torch.cuda.synchronize()
    assert bool((b == 5).all())
    m.close()


def test_own_streams_by_number(moe):
    """The legacy stream as 0, and set_stream to another one."""
    z = torch.randn(100, 8, device="cuda")
    m = moe.Moe(stream=0)
    want = m.route(z, 2)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    m.set_stream(s.cuda_stream)
    r = m.route(z, 2)
    m.synchronize()
    assert torch.equal(r.rows, want.rows)
    m.close()


def test_set_stream_of_a_handle_that_followed(moe):
    """After set_stream a handle stays on that stream, whatever the current one is."""
    m, s = moe.Moe(), torch.cuda.Stream()
    z = torch.randn(5000, 32, device="cuda")
    want = m.route(z, 4)
    torch.cuda.synchronize()
    m.set_stream(s.cuda_stream)
    out = m.route(z, 4)
    m.synchronize()
    delayed(s)
    busy = torch.cuda.Event()
    out.rows.zero_()
    torch.cuda.current_stream().synchronize()
    r = m.route(z, 4, out=out)   # waits behind the delay
    busy.record(s)
    seen = out.rows.cpu()
    assert not busy.query() and not bool(seen.any())
    m.synchronize()
    assert busy.query() and torch.equal(r.rows, want.rows)
    m.close()


@pytest.mark.parametrize("M", [40, 2000])
def test_wait_that_runs_out_is_seen_by_the_next_call(moe, M):
    """A program that waits for the device by itself learns of a given-up wait from its next call."""
    from paper_2608_07971_gb300 import esp
    m = moe.Moe()
    x, w = torch.randn(M, 1024, device="cuda"), torch.randn(300, 1024, device="cuda")
    q = m.quantize_weight(w)
    m.linear(x, q)
    m.synchronize()
    lib = moe.load_library()
    esp._check(lib.esp_moe_debug_set_wait_limit(m.h, 20), "set_wait_limit")
    esp._check(lib.esp_moe_debug_hold_load(m.h), "hold_load")
    m.linear(x, q)
    torch.cuda.synchronize()
    for status in (esp.ESP_ERR_TIMEOUT, esp.ESP_ERR_STATE, esp.ESP_ERR_STATE):
        with pytest.raises(esp.EspError) as err:
            m.route(x[:, :8], 2)
        assert err.value.status == status
    m.close()


def test_handles_made_and_closed_during_a_capture(moe):
    """Neither ends the capture of another stream's work."""
    m, spare = moe.Moe(), moe.Moe()
    z = torch.randn(3000, 32, device="cuda")
    r, want = m.routing(3000, 32, 3), spare.route(z, 3)
    m.route(z, 3, out=r)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        spare.close()
        new = moe.Moe()
        m.route(z, 3, out=r)
    r.rows.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(r.rows, want.rows) and torch.equal(new.route(z, 3).rows, want.rows)
    new.close()
    del graph
    m.close()
