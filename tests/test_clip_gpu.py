"""Norm and clipping of many gradients (include/esp_moe.h: esp_moe_clip) against 64 bits.

Bounds, u = 2^-24: a thread adds at most 64 squares in fp32 (each one rounding, at most 9 partial sums): the sum of squares
is within 72 u, its root within 36 u, rounded to fp32: 37 u. A result is value * factor, the factor within 38 u: 39 u and the
rounding unit of its type, relative, with the absolute unit below the normal range.
"""

import ctypes
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
UNIT = {torch.float32: (U, 2.0 ** -149), torch.bfloat16: (2.0 ** -8, 2.0 ** -134), torch.float16: (2.0 ** -11, 2.0 ** -25)}
TYPES = list(UNIT)


@pytest.fixture(scope="module")
def mm():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2608_07971_gb300 import build, moe
    build.build()
    m = moe.Moe()
    yield m
    m.synchronize()
    m.close()


def make(sizes, types, seed, size=1.0, lead=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [(torch.randn(n + lead, generator=g, device="cuda") * size).to(types[i % len(types)])[lead:]
            for i, n in enumerate(sizes)]


def norm_of(grads, scale=1.0):
    return scale * math.sqrt(sum(float(g.double().square().sum()) for g in grads))


def check(grads, got, norm, max_norm, scale):
    want = norm_of(grads, scale)
    assert abs(float(norm) - want) <= 37 * U * want
    by = scale * min(1.0, max_norm / want) if want > 0 else scale
    for g, o in zip(grads, got):
        rel, tiny = UNIT[o.dtype]
        w = g.double() * by
        assert o.dtype is g.dtype
        assert ((o.double() - w).abs() <= (rel + 39 * U) * w.abs() + tiny).all()


@pytest.mark.parametrize("sizes", [[1], [7], [8, 0, 1, 3], [4096], [2047, 2048, 2049], [100003, 5, 77777],
                                   [1000] * 300, [3_000_001, 2], [40_000_000, 13]])
@pytest.mark.parametrize("lead", [0, 3])
def test_clip(mm, sizes, lead):
    for types in ([torch.float32], [torch.bfloat16], [torch.float16], TYPES):
        for max_norm, scale in ((1.0, 1.0), (1e9, 0.25), (math.inf, 1.0)):
            grads = make(sizes, types, len(sizes), 0.5, lead)
            before = [g.clone() for g in grads]
            norm = mm.clip(grads, max_norm, scale=scale)                   # in place
            check(before, grads, norm, max_norm, scale)
            out = make(sizes, types, 9, 1.0, (lead + 1) % 4)                # groups of 16 bytes at other places
            again = mm.clip(mm.gradients(before, out=out), max_norm, scale=scale)
            check(before, out, again, max_norm, scale)
            if lead == 0:   # the same groups of 16 bytes, so the same sums
                assert torch.equal(norm, again) and all(torch.equal(a, b) for a, b in zip(out, grads))
            assert norm.shape == () and norm.dtype is torch.float32


def test_neighbours_are_left_alone(mm):
    """Slices of one buffer: what lies between them stays as it was."""
    for dt in TYPES:
        room = torch.full((5000,), 3.0, dtype=dt, device="cuda")
        cuts = [(1, 8), (9, 9), (17, 1000), (1001, 4990)]
        mm.clip([room[a:b] for a, b in cuts], 1.0)
        mask = torch.ones(5000, dtype=torch.bool, device="cuda")
        for a, b in cuts:
            mask[a:b] = False
        assert (room[mask] == 3.0).all() and (room[~mask] < 1.0).all()


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_values_whose_squares_leave_32_bits(mm, dt):
    for size in (2.0 ** 100, 2.0 ** -100, 2.0 ** -60):
        grads = make([3000, 50], [dt], 4, size)
        before = [g.clone() for g in grads]
        want = norm_of(before)
        norm = mm.clip(grads, want / 3)
        check(before, grads, norm, want / 3, 1.0)
    mixed = [torch.full((100,), 2.0 ** 100, dtype=dt, device="cuda"), torch.full((100,), 2.0 ** -100, dtype=dt, device="cuda")]
    assert float(mm.clip(mixed)) == pytest.approx(10 * 2.0 ** 100, rel=37 * U)


def test_values_that_are_not_finite(mm):
    """The norm says so; the gradients are scaled, not clipped."""
    for dt in TYPES:
        for v in (math.inf, -math.inf, math.nan):
            g = make([3000, 100, 10], [dt], 2)
            g[1][50] = v
            before = [t.clone() for t in g]
            norm = mm.clip(g, 1.0, scale=0.5)
            assert math.isnan(float(norm)) if math.isnan(v) else float(norm) == math.inf
            for a, b in zip(g, before):
                assert torch.equal(a.nan_to_num(nan=7.0), (b.float() * 0.5).to(dt).nan_to_num(nan=7.0))


def test_nothing_and_zeros(mm):
    assert float(mm.clip([], 1.0)) == 0.0
    z = [torch.zeros(5, device="cuda"), torch.zeros(0, device="cuda"), torch.zeros(100000, device="cuda").half()]
    assert float(mm.clip(z, 1.0)) == 0.0 and not any(t.any() for t in z)
    empty = [torch.empty(0, device="cuda")]
    assert float(mm.clip(empty, 1.0)) == 0.0


def test_norm_alone_in_c(mm):
    """out NULL: counted, not written."""
    from paper_2608_07971_gb300 import esp, moe
    a, b = make([1000, 333], [torch.float32], 1)
    a0, b0 = a.clone(), b.clone()
    norm = torch.zeros(1, device="cuda")
    c = (moe._CTensor * 2)((a.data_ptr(), None, 1000, 0), (b.data_ptr(), b.data_ptr(), 333, 0))
    mm._on_stream()
    esp._check(moe.load_library().esp_moe_clip(mm.h, 2, c, 1.0, 1.0, norm.data_ptr()), "clip")
    check([a0, b0], [a0 / norm_of([a0, b0]), b], norm, 1.0, 1.0)
    assert torch.equal(a, a0)


def test_past_32_bits(mm):
    """More elements than 2^32 in one tensor, the last ones counted."""
    n = (1 << 32) + 5
    t = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    t[-5:] = 2.0
    t[0] = 4.0
    norm = mm.clip([t], 3.0)
    assert float(norm) == 6.0 and float(t[-1]) == 1.0 and float(t[0]) == 2.0 and not t[1:-5].any()


def test_repeatable_and_in_graphs(mm):
    from paper_2608_07971_gb300 import moe
    m = moe.Moe()
    sizes = [100_000, 3_000_000, 17, 999] * 40
    grads = make(sizes, TYPES, 3)
    out = [torch.empty_like(g) for g in grads]
    li = m.gradients(grads, out=out)
    first = m.clip(li, 1.0).clone()
    want = [o.clone() for o in out]
    for _ in range(3):
        assert torch.equal(m.clip(li, 1.0), first) and all(torch.equal(a, b) for a, b in zip(out, want))
    norm = torch.zeros((), device="cuda")
    g, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=s):
        m.clip(li, 1.0, norm=norm)
    for t in grads:
        t.mul_(2.0)
    g.replay()
    torch.cuda.synchronize()
    # powers of two: the same roundings
    assert float(norm) == 2.0 * float(first)
    check(grads, out, norm, 1.0, 1.0)
    with torch.cuda.stream(s):
        a = m.clip(li, 1.0)
    b = m.clip(li, 1.0)
    torch.cuda.synchronize()
    assert torch.equal(a, b) and torch.equal(a, norm)
    m.close()


def test_gradients_written_right_before(mm):
    """The scaling loads its first gradients ahead of the norm's end: never ones that earlier work still writes."""
    sizes = [300_000, 17, 40_000]
    sets = [make(sizes, TYPES, s, 0.5) for s in range(3)]
    grads, outs = make(sizes, TYPES, 9), [[torch.empty_like(t) for t in sets[0]] for _ in range(30)]
    lists = [mm.gradients(grads, out=o) for o in outs]
    norms = [torch.zeros((), device="cuda") for _ in outs]
    torch.cuda.synchronize()
    for i, li in enumerate(lists):
        for g, s in zip(grads, sets[i % 3]):
            g.copy_(s)
        mm.clip(li, 1.0, norm=norms[i])
    torch.cuda.synchronize()
    for i, o in enumerate(outs):
        check(sets[i % 3], o, norms[i], 1.0, 1.0)
    # in place, one after another: each call begins with what the one before left
    a, b = [t.clone() for t in sets[0]], [t.clone() for t in sets[0]]
    for k in range(20):
        before = [t.clone() for t in a]
        check(before, a, mm.clip(a, 2.0 ** -k), 2.0 ** -k, 1.0)
    for k in range(20):   # nothing waits between
        mm.clip(b, 2.0 ** -k)
    assert all(torch.equal(s, t) for s, t in zip(a, b))


def test_moved_memory_is_used(mm):
    p = [torch.ones(10, device="cuda"), torch.ones(6, device="cuda")]
    li = mm.gradients(p)
    assert float(mm.clip(li)) == 4.0
    p[0].data = torch.full((10,), 3.0, device="cuda")
    assert float(mm.clip(li)) == pytest.approx(math.sqrt(96.0), rel=1e-6)


def test_refusals(mm):
    from paper_2608_07971_gb300 import esp
    g = torch.ones(100, device="cuda")
    for f in (lambda: mm.clip([g.double()]), lambda: mm.clip([g.cpu()]), lambda: mm.clip([g[::2]]),
              lambda: mm.gradients([g], out=[]), lambda: mm.gradients([g], out=[g.half()]),
              lambda: mm.gradients([g], out=[g[:50]]), lambda: mm.clip([g], norm=torch.zeros(2, device="cuda")),
              lambda: mm.clip([g], norm=torch.zeros((), dtype=torch.float64, device="cuda"))):
        with pytest.raises(ValueError):
            f()
    for f in (lambda: mm.clip([g], 0.0), lambda: mm.clip([g], -1.0), lambda: mm.clip([g], math.nan),
              lambda: mm.clip([g], 1.0, scale=0.0), lambda: mm.clip([g], 1.0, scale=math.inf),
              lambda: mm.clip([g], 1.0, scale=math.nan),
              lambda: mm.clip([g, g], 1.0),                                         # the same tensor twice
              lambda: mm.clip([g[:60], g[40:]], 1.0),
              lambda: mm.clip(mm.gradients([g[:50], g[50:]], out=[g[50:], g[:50]]), 1.0),
              lambda: mm.clip(mm.gradients([g[:50]], out=[g[25:75]]), 1.0)):
        with pytest.raises(esp.EspError) as err:
            f()
        assert err.value.status == esp.ESP_ERR_INVALID_ARG
    assert float(mm.clip([g], 1e9)) == 10.0 and (g == 1.0).all()
    mm.synchronize()


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_factors_below_32_bits(mm, dt):
    """max_norm / norm, or scale times it, is subnormal in fp32, or 0: the results are not."""
    for size, max_norm, scale in ((2.0 ** 115, 2.0 ** -8, 1.0), (2.0 ** 100, 2.0 ** -60, 1.0), (2.0 ** 110, 1.0, 2.0 ** -126),
                                  (2.0 ** 100, 2.0 ** -125, 2.0 ** -40), (2.0 ** 120, math.inf, 2.0 ** -126)):
        grads = make([3000, 77, 50000], [dt], 6, size)
        before = [g.clone() for g in grads]
        check(before, grads, mm.clip(grads, max_norm, scale=scale), max_norm, scale)
        out = [torch.empty_like(g) for g in grads]
        check(before, out, mm.clip(mm.gradients(before, out=out), max_norm, scale=scale), max_norm, scale)


def test_scales_at_the_ends_of_32_bits(mm):
    from paper_2608_07971_gb300 import esp
    most = float(torch.finfo(torch.float32).max)
    for scale in (2.0 ** 128, 1e300, 2.0 ** -127, 1e-300):   # fp32 has them as infinity, 0 or with fewer bits
        z = torch.zeros(100, device="cuda")
        with pytest.raises(esp.EspError) as err:
            mm.clip([z], scale=scale)
        assert err.value.status == esp.ESP_ERR_INVALID_ARG
    for scale, size in ((most, 2.0 ** -90), (2.0 ** -126, 2.0 ** 20)):
        for grads in ([torch.zeros(100, device="cuda")], make([1000, 3], [torch.float32], 7, size)):
            before = [g.clone() for g in grads]
            check(before, grads, mm.clip(grads, scale=scale), math.inf, scale)


def test_norm_within_a_gradient(mm):
    """Refused: it would be written while the gradients are still read. Right beside them it is taken."""
    from paper_2608_07971_gb300 import esp, moe
    room = torch.ones(101, device="cuda")
    for at in (0, 57, 99):
        with pytest.raises(esp.EspError) as err:
            mm.clip([room[:100]], 1.0, norm=room[at])
        assert err.value.status == esp.ESP_ERR_INVALID_ARG
    with pytest.raises(esp.EspError):
        mm.clip(mm.gradients([torch.ones(7, device="cuda")], out=[room[:7]]), 1.0, norm=room[6])
    counted = (moe._CTensor * 1)((room.data_ptr(), None, 100, 0))   # not written, but not the call's to write either
    for norm in (room.data_ptr() + 40, room.data_ptr() + 402):       # the second one not on 4 bytes
        mm._on_stream()
        assert moe.load_library().esp_moe_clip(mm.h, 1, counted, 1.0, 1.0, norm) == esp.ESP_ERR_INVALID_ARG
    assert (room == 1.0).all()
    assert float(mm.clip([room[:100]], 1e9, norm=room[100])) == 10.0 and (room[:100] == 1.0).all()
