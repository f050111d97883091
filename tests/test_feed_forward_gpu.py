"""Gated feed-forward blocks (include/esp_moe.h: esp_moe_feed_forward and its gradients) against the formulas in 64 bits.

Bounds, element by element, with u = 2^-24 and r the rounding unit of the 16-bit type (bf16 2^-8, half a step relative to
the value; fp16 2^-11, and 2^-25 absolute below its normal range), |.| of matrices by element:
  a sum of n products      2 n u sum |a b| (a truncating adder), each added operand's error times the other operand
  g, u = x G^T, x U^T      e_g = 2 H u |x||G|^T, e_u likewise
  act(g)                   slope below 1.13: 1.13 e_g, and its own arithmetic 16 u (|g| + 16) (|g| + 1)
  h = act(g) u             |u| e_act + |act| e_u + e_act e_u, then r |h|
  y = h O^T                e_h |O|^T + 2 F u |h||O|^T, then r |y|
  dh = dy O                2 H u |dy||O|
  dg = dh u act'(g)        g and u as kept, in 32 bits; act'' below 1 (relu: 1 where g is within its error of 0),
                           act' itself 16 u (|g| + 16); the product rule, then r |dg|; du = dh act(g) likewise
  dx, dG, dU, dO           as y, from the errors of their operands
"""

import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DT = {"bf16": torch.bfloat16, "f16": torch.float16}
UNIT = {"bf16": (2.0 ** -8, 2.0 ** -134), "f16": (2.0 ** -11, 2.0 ** -25), "f32": (U, 2.0 ** -149)}
ACTS = ["silu", "gelu", "gelu_tanh", "relu"]


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


def rand(*shape, dt, seed, size=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * size).to(DT[dt])


def act(g, kind):
    """The activation and its slope, in 64 bits."""
    if kind == "silu":
        s = torch.sigmoid(g)
        return g * s, s * (1 + g * (1 - s))
    if kind == "gelu":
        c = 0.5 * (1 + torch.erf(g / math.sqrt(2)))
        return g * c, c + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    if kind == "gelu_tanh":
        a = math.sqrt(2 / math.pi)
        t = torch.tanh(a * (g + 0.044715 * g ** 3))
        return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * a * (1 + 3 * 0.044715 * g * g)
    return torch.clamp(g, min=0), (g > 0).double()


def product(a, ea, b, eb, n):
    """a b and the bound of its error."""
    return a @ b, ea @ b.abs() + a.abs() @ eb + ea @ eb + 2 * n * U * (a.abs() @ b.abs())


def expert(x, w, o, kind, dt, dy=None):
    """{name: (value, bound)} of one expert's rows; the bounds leave out the results' own rounding."""
    r, tiny = UNIT[dt]
    F, H = o.shape[1], o.shape[0]
    zero = torch.zeros_like
    G, Up = w[:F], w[F:]
    g, eg = product(x, zero(x), G.t(), zero(G.t()), H)
    u, eu = product(x, zero(x), Up.t(), zero(Up.t()), H)
    a, slope = act(g, kind)
    ea = 1.13 * eg + 16 * U * (g.abs() + 16) * (g.abs() + 1)
    h = a * u
    eh = u.abs() * ea + a.abs() * eu + ea * eu
    eh = eh + r * (h.abs() + eh) + tiny
    out = dict(y=product(h, eh, o.t(), zero(o.t()), F))
    if dy is None:
        return out
    dh, edh = product(dy, zero(dy), o, zero(o), H)
    es = eg + 16 * U * (g.abs() + 16) if kind != "relu" else (g.abs() <= eg).double()
    dg, du = dh * u * slope, dh * a
    edg = (dh.abs() + edh) * (u.abs() + eu) * (slope.abs() + es) - dg.abs()
    edu = (dh.abs() + edh) * (a.abs() + ea) - du.abs()
    edg, edu = (e + r * (d.abs() + e) + tiny for e, d in ((edg, dg), (edu, du)))
    dp, edp = torch.cat([dg, du], 1), torch.cat([edg, edu], 1)
    out["dx"] = product(dp, edp, w, zero(w), 2 * F)
    n = x.shape[0]
    out["dinner"] = product(dp.t(), edp.t(), x, zero(x), n)
    out["douter"] = product(dy.t(), zero(dy.t()), h, eh, n)
    return out


def close(got, want, bound, dt):
    rel, absolute = UNIT[dt]
    got = got.double()
    lim = bound + rel * (want.abs() + bound) + absolute
    bad = ~((got - want).abs() <= lim)
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} off, worst {float(((got - want).abs() / lim).max()):.3g} of the bound"


def check(mm, sizes, H, F, dt, kind, gathered=False, spare=0, dw_dtype=None, seed=0):
    """One block with gradients against the formulas; `spare` rows belong to no expert."""
    E, n = len(sizes), sum(sizes)
    M = n + spare
    T = max(1, n // 2) if gathered else M
    x = rand(T, H, dt=dt, seed=seed)
    inner, outer = rand(E, 2 * F, H, dt=dt, seed=seed + 1, size=H ** -0.5), rand(E, H, F, dt=dt, seed=seed + 2, size=F ** -0.5)
    dy = rand(M, H, dt=dt, seed=seed + 3)
    w = mm.gated_weight(inner, outer, kind)
    rows = None
    if gathered:
        rows = torch.as_tensor(np.random.default_rng(seed).integers(0, T, M).astype(np.int32)).cuda()
        rows[n:] = -1
    offsets = torch.tensor([0, *np.cumsum(sizes)], dtype=torch.int32, device="cuda") if E > 1 or spare else None
    plan = dict(offsets=offsets, rows=rows)
    kept = mm.keep(M, w)
    y0, dx0 = torch.full((M, H), 7.0, dtype=DT[dt], device="cuda"), torch.full((M, H), 9.0, dtype=DT[dt], device="cuda")
    y = mm.feed_forward(x, w, keep=kept, out=y0, **plan)
    dx, dinner, douter = mm.feed_forward_backward(dy, x, w, kept, out=(dx0, None, None), dtype=dw_dtype, **plan)
    assert (y[n:] == 7.0).all() and (dx[n:] == 9.0).all()
    bare = mm.feed_forward(x, w, **plan)
    assert torch.equal(bare[:n], y[:n])
    wt = "f32" if dw_dtype is torch.float32 else dt
    assert dinner.dtype is douter.dtype is (dw_dtype or DT[dt])
    a = 0
    for e, k in enumerate(sizes):
        at = slice(a, a + k)
        xe = (x[rows[at].long()] if gathered else x[at]).double()
        ref = expert(xe, inner[e].double(), outer[e].double(), kind, dt, dy[at].double())
        close(y[at], *ref["y"], dt)
        close(dx[at], *ref["dx"], dt)
        close(dinner[e], *ref["dinner"], wt)
        close(douter[e], *ref["douter"], wt)
        a += k


SHAPES = [  # rows of each expert, H, F, type, activation, gathered, rows of no expert
    ([1], 64, 64, "bf16", "silu", False, 0),
    ([1], 8, 8, "f16", "gelu", False, 0),
    ([3], 1, 1, "bf16", "relu", False, 0),
    ([128], 128, 128, "bf16", "silu", False, 0),
    ([256], 256, 256, "f16", "gelu_tanh", False, 0),
    ([257], 200, 136, "bf16", "gelu", False, 0),
    ([300], 77, 129, "f16", "silu", False, 0),
    ([65, 0, 1, 63], 130, 67, "bf16", "silu", True, 5),
    ([0, 0, 0], 64, 72, "bf16", "silu", False, 4),
    ([64, 128, 256], 264, 320, "f16", "relu", False, 0),
    ([513, 1, 700], 136, 520, "bf16", "gelu_tanh", True, 0),
    ([31] * 40, 96, 33, "bf16", "gelu", True, 17),
    ([1999], 1001, 515, "bf16", "silu", False, 0),
    ([2] * 130, 72, 40, "f16", "silu", True, 0),
]


@pytest.mark.parametrize("sizes,H,F,dt,kind,gathered,spare", SHAPES)
def test_block_and_its_gradients(mm, sizes, H, F, dt, kind, gathered, spare):
    check(mm, sizes, H, F, dt, kind, gathered, spare, seed=sum(sizes) + H)


@pytest.mark.parametrize("M", [1, 2, 3, 4, 5, 8, 9])
@pytest.mark.parametrize("H,F", [(1, 1), (40, 3), (130, 2049), (2048, 65), (2056, 4100), (4096, 8200), (8190, 129), (16500, 40)])
def test_single_tokens(mm, M, H, F):
    check(mm, [M], H, F, "bf16" if H % 2 else "f16", "silu", False, 0, seed=H)
    check(mm, [M], H, F, "bf16", "gelu_tanh", True, 0, seed=H)


def test_single_tokens_of_one_block_with_offsets(mm):
    """Rows outside the one block's offsets are left as they are."""
    w = mm.gated_weight(rand(64, 96, dt="bf16", seed=1), rand(96, 32, dt="bf16", seed=2))
    x = rand(2, 96, dt="bf16", seed=3)
    want = mm.feed_forward(x, w)
    for lo, hi in ((0, 1), (1, 2), (0, 0), (0, 2), (-3, 9)):
        y = mm.feed_forward(x, w, offsets=torch.tensor([lo, hi], dtype=torch.int32, device="cuda"),
                            out=torch.full((2, 96), 5.0, dtype=torch.bfloat16, device="cuda"))
        a, b = max(0, lo), min(2, hi)
        assert torch.equal(y[a:b], want[a:b]) and (y[:a] == 5.0).all() and (y[b:] == 5.0).all()


@pytest.mark.parametrize("kind", ACTS)
@pytest.mark.parametrize("dt", ["bf16", "f16"])
def test_activations(mm, kind, dt):
    check(mm, [90, 40], 200, 144, dt, kind, True, 3, seed=5)


@pytest.mark.parametrize("M", [1, 64])
@pytest.mark.parametrize("dt", ["bf16", "f16"])
def test_gelu_of_exact_gates(mm, M, dt):
    # x = (1, 0, ...), u = 1: hidden is gelu(g), g exact. c = (1 + erf) / 2 is q or 1 - q, q a fit to 4e-8 = 0.7 u times an
    # exponential (2 ulp = 4 u and |argument| u twice, argument g^2 / 2), a quotient (4 u), eight steps of Horner's rule whose terms
    # are below three times the sum (24 u) and two products (2 u): q (36 + g^2) u, and u for 1 - q and for g c.
    r, tiny = UNIT[dt]
    F, H = 4096, 64
    g = torch.linspace(-9, 9, F, device="cuda").to(DT[dt])
    x, inner = torch.zeros(M, H, device="cuda", dtype=DT[dt]), torch.zeros(1, 2 * F, H, device="cuda", dtype=DT[dt])
    x[:, 0], inner[0, :F, 0], inner[0, F:, 0] = 1, g, 1
    w = mm.gated_weight(inner, torch.zeros(1, H, F, device="cuda", dtype=DT[dt]), "gelu")
    kept = mm.keep(M, w)
    mm.feed_forward(x, w, keep=kept)
    g = g.double()
    q = 0.5 * torch.erfc(g.abs() / math.sqrt(2))
    want = g * torch.where(g > 0, 1 - q, q)
    lim = g.abs() * q * (36 + g * g) * U + 2 * U * want.abs()
    lim = lim + r * (want.abs() + lim) + tiny
    assert torch.equal(kept.pre[:, 0, :F].double(), g.expand(M, F))
    assert ((kept.hidden[:, :F].double() - want).abs() <= lim).all()


@pytest.mark.parametrize("sizes,H,F,dt,gathered", [
    ([2500], 8192, 1000, "bf16", False), ([300], 1071, 454, "f16", True), ([40], 8200, 130, "bf16", False),
    ([3, 0, 70, 1, 200], 2100, 200, "bf16", True), ([20, 30], 1071, 5, "f16", False)])
def test_signs_of_gates_near_zero(mm, sizes, H, F, dt, gathered):
    # relu's slope is 0 or 1: what is kept for it near 0 has to be right relative to itself. The terms a b are exact in 32
    # bits, the sum of n of them is off by at most u of itself and n 2 u^2 sum |a b|, and is rounded once.
    E, M = len(sizes), sum(sizes)
    x, inner = rand(M, H, dt=dt, seed=31), rand(E, 2 * F, H, dt=dt, seed=32, size=H ** -0.5)
    w = mm.gated_weight(inner, rand(E, H, F, dt=dt, seed=33, size=F ** -0.5), "relu")
    offsets = torch.tensor([0, *np.cumsum(sizes)], dtype=torch.int32, device="cuda")
    rows = torch.arange(M - 1, -1, -1, dtype=torch.int32, device="cuda") if gathered else None
    kept = mm.keep(M, w)
    mm.feed_forward(x, w, offsets=offsets, rows=rows, keep=kept)
    a = 0
    for e, n in enumerate(sizes):
        xe = (x.flip(0) if gathered else x)[a:a + n].double()
        g = xe @ inner[e, :F].double().t()
        got = kept.pre[a:a + n, 0, :F].double()
        lim = 2 * U * g.abs() + 2 * H * U * U * (xe.abs() @ inner[e, :F].double().abs().t())
        near = g.abs() < H * 2.0 ** -27   # of values around 1
        assert ((got - g).abs() <= lim)[near].all()
        a += n


@pytest.mark.parametrize("dt", ["bf16", "f16"])
def test_weight_gradients_in_32_bits(mm, dt):
    check(mm, [70, 0, 333], 136, 100, dt, "silu", True, 0, dw_dtype=torch.float32)


def test_long_inner_axes(mm):
    check(mm, [40, 300], 2050, 999, "f16", "gelu", False, 0)
    check(mm, [260], 72, 4100, "bf16", "silu", False, 0)


TILES = [  # rows of each expert, H, F, type: the choice of tiles in csrc/esp_ff_gemm.cu, on both sides of its rules
    ([100], 64, 25600, "bf16"),          # single CTAs: HIDDEN, DPRE
    ([100], 25600, 64, "f16"),           # single CTAs: OUT, DX
    ([20], 4160, 100, "bf16"),           # split inner axes: HIDDEN, DPRE; a tile of few rows
    ([140], 100, 4160, "f16"),           # split inner axes: OUT, DX
    ([5000], 64, 72, "bf16"),            # split inner axes: both weights' gradients
    ([4000, 9, 2300], 40, 200, "bf16"),  # the same, of experts of which one has fewer blocks than parts
    ([1500] * 6, 520, 264, "bf16"),      # pairs
]


@pytest.mark.parametrize("sizes,H,F,dt", TILES)
def test_tiles(mm, sizes, H, F, dt):
    check(mm, sizes, H, F, dt, "silu", False, 0, seed=H)
    if len(sizes) > 1:
        check(mm, sizes, H, F, dt, "gelu", True, 70, dw_dtype=torch.float32, seed=F)


def test_many_experts(mm):
    """As many experts as there can be, most of them with few rows or none."""
    rng = np.random.default_rng(3)
    check(mm, list(rng.integers(0, 5, 700)), 40, 24, "bf16", "silu", True, 10)
    check(mm, [0] * 1000 + [3] + [0] * 22 + [80], 32, 16, "f16", "relu", False, 0)


def test_a_stream_of_its_own(mm):
    from paper_2608_07971_gb300 import moe
    s = torch.cuda.Stream()
    m = moe.Moe(stream=s.cuda_stream)
    x, dy = rand(300, 96, dt="bf16", seed=1), rand(300, 96, dt="bf16", seed=2)
    inner, outer = rand(2, 128, 96, dt="bf16", seed=3, size=0.1), rand(2, 96, 64, dt="bf16", seed=4, size=0.1)
    off = torch.tensor([0, 130, 300], dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()

    def step(m):
        w = m.gated_weight(inner, outer)
        kept = m.keep(300, w)
        y = m.feed_forward(x, w, offsets=off, keep=kept)
        grads = m.feed_forward_backward(dy, x, w, kept, offsets=off)
        m.synchronize()
        norm = m.clip(list(grads), 1.0)
        m.synchronize()
        return (y, norm, *grads)

    assert all(torch.equal(a, b) for a, b in zip(step(m), step(mm)))
    m.close()


def test_growing_work_space_under_a_graph(mm):
    """A captured step is replayed after the same handle's work space has grown."""
    from paper_2608_07971_gb300 import moe
    m = moe.Moe()
    w = m.gated_weight(rand(2, 128, 96, dt="bf16", seed=3, size=0.1), rand(2, 96, 64, dt="bf16", seed=4, size=0.1))
    x = rand(300, 96, dt="bf16", seed=1)
    off = torch.tensor([0, 130, 300], dtype=torch.int32, device="cuda")
    rows = torch.arange(299, -1, -1, dtype=torch.int32, device="cuda")
    want = m.feed_forward(x, w, offsets=off, rows=rows)
    out = torch.empty_like(want)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        m.feed_forward(x, w, offsets=off, rows=rows, out=out)
    big = rand(200_000, 96, dt="bf16", seed=2)
    m.feed_forward(big, w, offsets=torch.tensor([0, 9, 200_000], dtype=torch.int32, device="cuda"))
    out.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    m.close()


def test_activations_far_out(mm):
    """Gate values of hundreds: the activations' tails and their slopes stay finite."""
    for kind in ACTS:
        x = torch.tensor([[-300.0, 1.0], [300.0, 1.0], [-30.0, 1.0], [30.0, 1.0], [0.0, 1.0]], device="cuda").bfloat16()
        inner = torch.eye(2, device="cuda").bfloat16()                       # g = x0, u = x1
        outer = torch.tensor([[1.0], [0.0]], device="cuda").bfloat16()
        w = mm.gated_weight(inner, outer, kind)
        kept = mm.keep(5, w)
        y = mm.feed_forward(x, w, keep=kept)
        dx, _, _ = mm.feed_forward_backward(torch.tensor([[1.0, 0.0]] * 5, device="cuda").bfloat16(), x, w, kept)
        a, slope = act(x[:, 0].double(), kind)
        assert ((y[:, 0].double() - a).abs() <= 2.0 ** -7 * a.abs() + 1e-6).all()
        assert ((dx[:, 0].double() - slope).abs() <= 2.0 ** -6 * slope.abs() + 1e-6).all()


def test_rows_of_others_do_not_reach_a_gradient(mm):
    """NaN and infinities in one expert's rows, and in the rows of none, stay there."""
    sizes = [70, 33, 129]
    n, H, F = sum(sizes), 128, 192
    x, dy = rand(n + 40, H, dt="bf16", seed=1), rand(n + 40, H, dt="bf16", seed=2)
    w = mm.gated_weight(rand(3, 2 * F, H, dt="bf16", seed=3, size=0.1), rand(3, H, F, dt="bf16", seed=4, size=0.1))
    offsets = torch.tensor([0, 70, 103, n], dtype=torch.int32, device="cuda")

    def both(x, dy):
        kept = mm.keep(n + 40, w)
        y = mm.feed_forward(x, w, offsets=offsets, keep=kept)
        return (y, *mm.feed_forward_backward(dy, x, w, kept, offsets=offsets))

    want = both(x, dy)
    x2, dy2 = x.clone(), dy.clone()
    x2[70:103], dy2[70:103] = math.nan, math.inf
    x2[n:], dy2[n:] = math.inf, math.nan
    got = both(x2, dy2)
    for a, b in zip(want[:2], got[:2]):
        assert torch.equal(a[:70], b[:70]) and torch.equal(a[103:n], b[103:n])
    for a, b in zip(want[2:], got[2:]):
        assert torch.equal(a[0], b[0]) and torch.equal(a[2], b[2]) and b[1].isnan().any()


def test_gradients_against_differences(mm):
    """Along random directions, the loss <y, c> in 64 bits changes as the gradients say."""
    sizes, H, F = [9, 14], 40, 56
    n = sum(sizes)
    x, c = rand(n, H, dt="f16", seed=1), rand(n, H, dt="f16", seed=2)
    inner, outer = rand(2, 2 * F, H, dt="f16", seed=3, size=0.2), rand(2, H, F, dt="f16", seed=4, size=0.2)
    offsets = torch.tensor([0, 9, n], dtype=torch.int32, device="cuda")
    for kind in ACTS[:3]:
        w = mm.gated_weight(inner, outer, kind)
        kept = mm.keep(n, w)
        mm.feed_forward(x, w, offsets=offsets, keep=kept)
        grads = mm.feed_forward_backward(c, x, w, kept, offsets=offsets)

        def loss(x, inner, outer):
            total = 0.0
            for e, at in enumerate((slice(0, 9), slice(9, n))):
                p = x[at] @ inner[e].t()
                total += float(((act(p[:, :F], kind)[0] * p[:, F:]) @ outer[e].t() * c[at].double()).sum())
            return total

        at = [t.double() for t in (x, inner, outer)]
        for i, g in enumerate(grads):
            d = torch.randn(at[i].shape, generator=torch.Generator(device="cuda").manual_seed(i), device="cuda").double()
            step = 1e-4
            hi, lo = ([t + s * step * d if j == i else t for j, t in enumerate(at)] for s in (1, -1))
            slope = (loss(*hi) - loss(*lo)) / (2 * step)
            # each product of the gradient carries at most four roundings to fp16 (2^-11), in either direction
            size = float((g.double().abs() * d.abs()).sum())
            assert abs(float((g.double() * d).sum()) - slope) <= 4 * 2.0 ** -11 * size + 1e-5 * size


def test_strided_and_misaligned(mm):
    """Views into wider buffers, and weights whose rows are not on 16 bytes, give what their copies give."""
    for dt in DT:
        base = rand(50, 333, dt=dt, seed=1)
        inner, outer = rand(130, 131, dt=dt, seed=2, size=0.1), rand(131, 65, dt=dt, seed=3, size=0.1)
        w = mm.gated_weight(inner, outer)
        assert w.inner.shape == (1, 130, 131) and torch.equal(w.inner[0], inner) and torch.equal(w.outer[0], outer)
        for at in (slice(5, 136), slice(8, 139)):
            x = base[:, at]
            wide = torch.zeros(50, 200, dtype=DT[dt], device="cuda")
            k1, k2 = mm.keep(50, w), mm.keep(50, w)
            y = mm.feed_forward(x, w, out=wide[:, 3:134], keep=k1)
            y2 = mm.feed_forward(x.contiguous(), w, keep=k2)
            assert torch.equal(y, y2) and not wide[:, :3].any() and not wide[:, 134:].any()
            dwide = torch.zeros(50, 200, dtype=DT[dt], device="cuda")
            g1 = mm.feed_forward_backward(y, x, w, k1, out=(dwide[:, 8:139], None, None))
            g2 = mm.feed_forward_backward(y2, x.contiguous(), w, k2)
            assert all(torch.equal(a, b) for a, b in zip(g1, g2)) and not dwide[:, :8].any() and not dwide[:, 139:].any()
            # results that start at an odd element
            room = torch.zeros(2 * 65 * 131 + 3, dtype=DT[dt], device="cuda")
            g3 = mm.feed_forward_backward(y2, x.contiguous(), w, k2, need=(False, True, False),
                                          out=(None, room[1:-2].view(1, 130, 131), None))
            assert torch.equal(g3[1], g2[1]) and g3[0] is None and g3[2] is None and not room[0] and not room[-2:].any()


def test_changed_weights_are_used(mm):
    x = rand(40, 128, dt="bf16", seed=1)
    w = mm.gated_weight(rand(2, 64, 128, dt="bf16", seed=2), rand(2, 128, 32, dt="bf16", seed=3))
    off = torch.tensor([0, 20, 40], dtype=torch.int32, device="cuda")
    first = mm.feed_forward(x, w, offsets=off)
    fresh = rand(2, 64, 128, dt="bf16", seed=4)
    w.inner = fresh
    second = mm.feed_forward(x, w, offsets=off)
    assert not torch.equal(first, second)
    w.inner.copy_(rand(2, 64, 128, dt="bf16", seed=2))
    assert torch.equal(mm.feed_forward(x, w, offsets=off), first)
    w.activation = "relu"
    assert not torch.equal(mm.feed_forward(x, w, offsets=off), first)
    with pytest.raises(ValueError):
        w.outer = fresh
        mm.feed_forward(x, w, offsets=off)


def test_offsets_past_32_bits(mm):
    """Rows whose element offsets pass 2^31, in place and gathered."""
    base = torch.empty(2100, 1 << 20, dtype=torch.bfloat16, device="cuda")
    x, out = base[:, 8:72], base[:, 128:192]
    x.copy_(torch.randn(2100, 64, device="cuda"))
    w = mm.gated_weight(rand(96, 64, dt="bf16", seed=1), rand(64, 48, dt="bf16", seed=2))
    want = mm.feed_forward(x.contiguous(), w)
    assert torch.equal(mm.feed_forward(x, w, out=out), want)
    rows = torch.arange(2099, -1, -1, dtype=torch.int32, device="cuda")
    assert torch.equal(mm.feed_forward(x, w, rows=rows), want.flip(0))


def test_empty(mm):
    w = mm.gated_weight(rand(2, 64, 32, dt="bf16", seed=1), rand(2, 32, 32, dt="bf16", seed=2))
    x, off = torch.empty(0, 32, dtype=torch.bfloat16, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    kept = mm.keep(0, w)
    y = mm.feed_forward(x, w, offsets=off, keep=kept)
    dx, dinner, douter = mm.feed_forward_backward(y, x, w, kept, offsets=off)
    assert y.shape == dx.shape == (0, 32) and not dinner.any() and not douter.any()


def test_rows_out_of_range_read_zeros(mm):
    w = mm.gated_weight(rand(64, 32, dt="bf16", seed=1), rand(32, 32, dt="bf16", seed=2))
    x = rand(6, 32, dt="bf16", seed=3)
    rows = torch.tensor([0, -1, 5, 6, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device="cuda")
    y = mm.feed_forward(x, w, rows=rows)
    assert torch.equal(y[[0, 2]], mm.feed_forward(x[[0, 5]], w)) and not y[[1, 3, 4, 5]].any()


def test_offsets_that_do_not_ascend_stay_in_range(mm):
    """Nothing outside the rows and gradients is written."""
    w = mm.gated_weight(rand(4, 64, 64, dt="bf16", seed=1), rand(4, 64, 32, dt="bf16", seed=2))
    x = rand(300, 64, dt="bf16", seed=3)
    want = mm.feed_forward(x[:100], w, offsets=torch.tensor([0, 25, 50, 75, 100], dtype=torch.int32, device="cuda"))
    for off in ([0, 300, 0, 300, 300], [-5, 900, 10, 2 ** 31 - 1, 3], [300, 200, 100, 50, 0]):
        room = torch.full((302, 64), 5.0, dtype=torch.bfloat16, device="cuda")
        offsets = torch.tensor(off, dtype=torch.int32, device="cuda")
        kept = mm.keep(300, w)
        mm.feed_forward(x, w, offsets=offsets, out=room[1:301], keep=kept)
        mm.feed_forward_backward(x, x, w, kept, offsets=offsets)
        assert (room[0] == 5.0).all() and (room[301] == 5.0).all()
    assert torch.equal(mm.feed_forward(x[:100], w, offsets=torch.tensor([0, 25, 50, 75, 100], dtype=torch.int32, device="cuda")), want)


def test_repeatable_on_streams_and_in_graphs(mm):
    """The same bits on every run, on other streams, and from a replayed graph whose inputs changed."""
    from paper_2608_07971_gb300 import moe
    m = moe.Moe()
    sizes = torch.tensor([0, 100, 100, 350, 400], dtype=torch.int32, device="cuda")
    w = m.gated_weight(rand(4, 256, 136, dt="bf16", seed=1, size=0.1), rand(4, 136, 128, dt="bf16", seed=2, size=0.1))
    x = [rand(200, 136, dt="bf16", seed=s) for s in (3, 4)]
    rows = torch.randint(0, 200, (400,), device="cuda").int()
    dy = rand(400, 136, dt="bf16", seed=5)

    def step(m, x, kept, out=None, grads=(None, None, None)):
        y = m.feed_forward(x, w, offsets=sizes, rows=rows, keep=kept, out=out)
        return (y, *m.feed_forward_backward(dy, x, w, kept, offsets=sizes, rows=rows, out=grads))

    want = [[t.clone() for t in step(m, v, m.keep(400, w))] for v in x]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    kept = [m.keep(400, w) for _ in range(2)]
    got = []
    for i in range(6):
        with torch.cuda.stream(streams[i % 2]):
            got.append((i % 2, step(m, x[i % 2], kept[i % 2])))
    m.synchronize()
    torch.cuda.synchronize()
    for i, g in got:
        assert all(torch.equal(a, b) for a, b in zip(g, want[i]))
    buf, keep = x[0].clone(), m.keep(400, w)
    out = [torch.empty_like(t) for t in want[0]]
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=streams[0]):
        step(m, buf, keep, out[0], tuple(out[1:]))
    for i in (1, 0, 1):
        buf.copy_(x[i])
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want[i]))
    m.close()


def test_weights_written_right_before(mm):
    """Single tokens load their first weights ahead of the launch before: never ones that earlier work still writes."""
    from paper_2608_07971_gb300 import moe
    H, F = 1024, 2048
    w = mm.gated_weight(rand(2 * F, H, dt="bf16", seed=0), rand(H, F, dt="bf16", seed=0))
    x = rand(1, H, dt="bf16", seed=1)
    sets = [(rand(1, 2 * F, H, dt="bf16", seed=s, size=H ** -0.5), rand(1, H, F, dt="bf16", seed=s + 9, size=F ** -0.5))
            for s in range(2, 6)]
    want = []
    for a, b in sets:
        torch.cuda.synchronize()
        want.append(mm.feed_forward(x, moe.GatedWeight(a, b)))
    torch.cuda.synchronize()
    out = [torch.empty_like(x) for _ in range(40)]

    def run():
        for i, y in enumerate(out):
            w.inner.copy_(sets[i % 4][0])
            w.outer.copy_(sets[i % 4][1])
            mm.feed_forward(x, w, out=y)

    run()
    torch.cuda.synchronize()
    assert all(torch.equal(y, want[i % 4]) for i, y in enumerate(out))
    for y in out:
        y.zero_()
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        run()
    g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(y, want[i % 4]) for i, y in enumerate(out))


def test_copies_of_weights_and_kept(mm):
    import copy
    import pickle
    x = rand(30, 64, dt="bf16", seed=1)
    w = mm.gated_weight(rand(1, 64, 64, dt="bf16", seed=2), rand(1, 64, 32, dt="bf16", seed=3), "gelu")
    want = mm.feed_forward(x, w)
    for v in (copy.copy(w), copy.deepcopy(w), pickle.loads(pickle.dumps(w))):
        assert v.activation == "gelu" and torch.equal(mm.feed_forward(x, v), want)


@pytest.mark.parametrize("which", ["forward", "dx", "weights"])
def test_wait_that_runs_out_is_reported(mm, which):
    """A product whose load never comes ends by its bounded waits; the handle then refuses work."""
    from paper_2608_07971_gb300 import esp, moe
    m = moe.Moe()
    sizes = torch.tensor([0, 700, 1010], dtype=torch.int32, device="cuda")
    x, dy = rand(1010, 512, dt="bf16", seed=1), rand(1010, 512, dt="bf16", seed=2)
    w = m.gated_weight(rand(2, 640, 512, dt="bf16", seed=3), rand(2, 512, 320, dt="bf16", seed=4))
    kept = m.keep(1010, w)
    want = m.feed_forward(x, w, offsets=sizes, keep=kept)
    m.synchronize()
    lib = moe.load_library()
    esp._check(lib.esp_moe_debug_set_wait_limit(m.h, 20), "set_wait_limit")
    esp._check(lib.esp_moe_debug_hold_load(m.h), "hold_load")
    if which == "forward":
        m.feed_forward(x, w, offsets=sizes, keep=kept)
    else:   # the first product of the call
        m.feed_forward_backward(dy, x, w, kept, offsets=sizes, need=(True, False, False) if which == "dx" else (False, False, True))
    with pytest.raises(esp.EspError) as err:
        m.synchronize()
    assert err.value.status == esp.ESP_ERR_TIMEOUT
    with pytest.raises(esp.EspError) as err:
        m.feed_forward(x, w, offsets=sizes)
    assert err.value.status == esp.ESP_ERR_STATE
    m.close()
    assert torch.equal(mm.feed_forward(x, w, offsets=sizes), want)   # another handle works on


def test_refusals(mm):
    from paper_2608_07971_gb300 import esp, moe
    x = rand(4, 32, dt="bf16", seed=1)
    inner, outer = rand(2, 48, 32, dt="bf16", seed=2), rand(2, 32, 24, dt="bf16", seed=3)
    w = mm.gated_weight(inner, outer)
    off = torch.tensor([0, 2, 4], dtype=torch.int32, device="cuda")
    kept = mm.keep(4, w)
    y = mm.feed_forward(x, w, offsets=off, keep=kept)
    bad = [
        lambda: mm.gated_weight(inner.float(), outer.float()),
        lambda: mm.gated_weight(inner, outer.half()),
        lambda: mm.gated_weight(inner[:, :47], outer),
        lambda: mm.gated_weight(inner, outer[:, :, :23]),
        lambda: mm.gated_weight(inner, outer, "tanh"),
        lambda: mm.gated_weight(inner.cpu(), outer.cpu()),
        lambda: mm.feed_forward(x, w),
        lambda: mm.feed_forward(x.half(), w, offsets=off),
        lambda: mm.feed_forward(x.float(), w, offsets=off),
        lambda: mm.feed_forward(x[:, :31], w, offsets=off),
        lambda: mm.feed_forward(x.cpu(), w, offsets=off),
        lambda: mm.feed_forward(x, w, offsets=off.long()),
        lambda: mm.feed_forward(x, w, offsets=off[:2]),
        lambda: mm.feed_forward(x, w, offsets=off, rows=torch.zeros(3, device="cuda")),
        lambda: mm.feed_forward(x, w, offsets=off, out=torch.empty(4, 31, dtype=torch.bfloat16, device="cuda")),
        lambda: mm.feed_forward(x, w, offsets=off, keep=mm.keep(5, w)),
        lambda: mm.feed_forward_backward(y[:3], x, w, kept, offsets=off),
        lambda: mm.feed_forward_backward(y.half(), x, w, kept, offsets=off),
        lambda: mm.feed_forward_backward(y, x, w, mm.keep(3, w), offsets=off),
        lambda: mm.feed_forward_backward(y, x, w, kept, offsets=off, dtype=torch.float16),
        lambda: mm.feed_forward_backward(y, x, w, kept, offsets=off, out=(None, torch.empty(2, 47, 32, device="cuda"), None)),
        lambda: mm.feed_forward_backward(y, x, w, kept, offsets=off, out=(
            None, torch.empty(2, 48, 32, device="cuda"), torch.empty(2, 32, 24, dtype=torch.bfloat16, device="cuda"))),
    ]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    # gathered rows, but kept from a pass over rows in place; rows that overlap one another; results in place of what is read
    for f in (lambda: mm.feed_forward_backward(y, x, w, kept, offsets=off, rows=torch.zeros(4, dtype=torch.int32, device="cuda")),
              lambda: mm.feed_forward(x[:1].expand(4, 32), w, offsets=off),
              lambda: mm.feed_forward(x, w, offsets=off, keep=kept, out=x),
              lambda: mm.feed_forward_backward(y, x, w, kept, offsets=off, out=(y, None, None)),
              lambda: mm.feed_forward_backward(y, x, w, kept, offsets=off, out=(x, None, None))):
        with pytest.raises(esp.EspError) as err:
            f()
        assert err.value.status == esp.ESP_ERR_INVALID_ARG
    assert torch.equal(mm.feed_forward(x, w, offsets=off), y)   # a refusal leaves the handle usable
    mm.synchronize()
    assert isinstance(moe.GatedWeight(inner, outer), moe.GatedWeight)


def test_a_layer_as_it_is_used(mm):
    """Routing, blocks, weighted return, all gradients, clipping: a training step against the same in 64 bits."""
    from paper_2608_07971_gb300 import moe
    T, E, k, H, F = 150, 6, 2, 96, 80
    x = rand(T, H, dt="bf16", seed=1)
    wr = rand(E, H, dt="bf16", seed=2, size=H ** -0.5)
    inner, outer = rand(E, 2 * F, H, dt="bf16", seed=3, size=H ** -0.5), rand(E, H, F, dt="bf16", seed=4, size=F ** -0.5)
    w = mm.gated_weight(inner, outer)
    logits = x.float() @ wr.float().t()
    r = mm.route(logits, k, gate=moe.Gate("softmax"))
    kept = mm.keep(T * k, w)
    y = mm.feed_forward(x, w, offsets=r.offsets, rows=r.rows, keep=kept)
    out = mm.combine(y, r.pos, r.weight)
    dout = rand(T, H, dt="bf16", seed=5)
    dy, dweight = mm.combine_backward(dout, y, r.pos, r.weight)
    dx, dinner, douter = mm.feed_forward_backward(dy, x, w, kept, offsets=r.offsets, rows=r.rows)
    dtoken = mm.combine(dx, r.pos)
    dwr = (mm.route_backward(logits, r.idx, dweight=dweight).t() @ x.float())
    grads = [dinner, douter, dwr]
    before = [g.clone() for g in grads]
    norm = mm.clip(grads, max_norm=0.5)

    v = [t.double().requires_grad_() for t in (x, wr, inner, outer)]
    z = v[0] @ v[1].t()
    p = torch.softmax(torch.gather(z, 1, r.idx.long()), -1)
    total = 0.0
    for e in range(E):
        t, j = torch.nonzero(r.idx == e, as_tuple=True)
        q = v[0][t] @ v[2][e].t()
        ye = (torch.nn.functional.silu(q[:, :F]) * q[:, F:]) @ v[3][e].t()
        total = total + torch.zeros(T, H, dtype=torch.float64, device="cuda").index_add(0, t, ye * p[t, j][:, None])
    total.backward(dout.double())
    # 16-bit roundings of h, y, dy, the gradients of the inner rows and the results: at most 8 of 2^-8 each, on sums of
    # hundreds of terms of either sign; 2 percent of a result's norm
    for got, want in ((out, total.detach()), (before[0], v[2].grad), (before[1], v[3].grad), (before[2], v[1].grad)):
        assert float((got.double() - want).norm() / want.norm()) < 0.02
    assert dtoken.shape == (T, H)
    n = math.sqrt(sum(float(g.double().square().sum()) for g in before))
    assert abs(float(norm) - n) <= 1e-6 * n
    for g, b in zip(grads, before):
        want = b.double() * (0.5 / n)
        unit = 2.0 ** -8 if g.dtype is torch.bfloat16 else U
        assert ((g.double() - want).abs() <= (unit + 1e-6) * want.abs() + 2.0 ** -134).all()


@pytest.mark.parametrize("sizes", [[1], [8], [9], [40, 70, 3]])   # on the CUDA cores, on the tensor cores
@pytest.mark.parametrize("kind", ACTS)
def test_nan_of_a_gate_reaches_the_results(mm, sizes, kind):
    """NaN in one weight of G alone, as of a step that went wrong: every sum that takes its g in is NaN, and the norm of the
    gradients; the others are what they are without it."""
    E, M, H, F, e, f = len(sizes), sum(sizes), 72, 40, len(sizes) // 2, 7
    x, dy = rand(M, H, dt="bf16", seed=51), rand(M, H, dt="bf16", seed=52)
    inner, outer = rand(E, 2 * F, H, dt="bf16", seed=53, size=H ** -0.5), rand(E, H, F, dt="bf16", seed=54, size=F ** -0.5)
    offsets = torch.tensor([0, *np.cumsum(sizes)], dtype=torch.int32, device="cuda")
    own = torch.zeros(M, dtype=torch.bool, device="cuda")
    own[int(offsets[e]):int(offsets[e + 1])] = True
    got = []
    for v in (0.5, math.nan):
        inner[e, f, 3] = v
        w, kept = mm.gated_weight(inner, outer, kind), mm.keep(M, mm.gated_weight(inner, outer, kind))
        y = mm.feed_forward(x, w, offsets=offsets, keep=kept)
        bare = mm.feed_forward(x, w, offsets=offsets)
        assert torch.equal(bare.nan_to_num(nan=7.0), y.nan_to_num(nan=7.0))
        got.append((y, *mm.feed_forward_backward(dy, x, w, kept, offsets=offsets)))
    plain, bad = got
    for a, b in zip(plain[:2], bad[:2]):   # y, dx: the rows of this expert
        assert a.isfinite().all() and b[own].isnan().all() and torch.equal(a[~own], b[~own])
    here = torch.zeros(E, 2 * F, dtype=torch.bool, device="cuda")
    here[e, [f, F + f]] = True   # the gradients of G x and of U x
    assert plain[2].isfinite().all() and bad[2][here].isnan().all() and torch.equal(plain[2][~here], bad[2][~here])
    a, b = (v[3].transpose(1, 2) for v in (plain, bad))
    here[e, F + f] = False
    assert a.isfinite().all() and b[here[:, :F]].isnan().all() and torch.equal(a[~here[:, :F]], b[~here[:, :F]])
    for i in (2, 3):
        assert math.isnan(float(mm.clip([bad[i].clone()], 1.0))) and math.isfinite(float(mm.clip([plain[i].clone()], 1.0)))


def cancelling(M, F, H, dt, seed):
    """Rows far from 0 and weights whose rows nearly sum to 0: g is far below the sums on the way to it."""
    G = torch.randn(F, H, generator=torch.Generator(device="cuda").manual_seed(seed + 1), device="cuda") * H ** -0.5
    return (rand(M, H, dt=dt, seed=seed).float() + 64).to(DT[dt]), (G - G.mean(1, keepdim=True)).to(DT[dt])


@pytest.mark.parametrize("sizes,H,F,dt,gathered", [
    ([2000], 2048, 1024, "bf16", False), ([2000], 8192, 512, "f16", False), ([300, 0, 90], 2050, 300, "bf16", True),
    ([40], 4100, 130, "f16", False)])   # the last one: split inner axes
def test_signs_of_gates_that_cancel(mm, sizes, H, F, dt, gathered):
    # As test_signs_of_gates_near_zero. S = |x||w| / sqrt H (lengths) is what the sums on the way to g are around; what an
    # adder of 24 bits that cuts off loses in H / 16 steps is below H / 16 2^-23 S = 2 H U S / 16, a g below that is summed again.
    E, M = len(sizes), sum(sizes)
    x, G = cancelling(M, E * F, H, dt, 61)
    inner = torch.cat([G.view(E, F, H), rand(E, F, H, dt=dt, seed=63, size=H ** -0.5)], 1)
    w = mm.gated_weight(inner, rand(E, H, F, dt=dt, seed=64, size=F ** -0.5), "relu")
    offsets = torch.tensor([0, *np.cumsum(sizes)], dtype=torch.int32, device="cuda")
    rows = torch.arange(M - 1, -1, -1, dtype=torch.int32, device="cuda") if gathered else None
    kept = mm.keep(M, w)
    mm.feed_forward(x, w, offsets=offsets, rows=rows, keep=kept)
    a = 0
    for e, n in enumerate(sizes):
        xe, Ge = (x.flip(0) if gathered else x)[a:a + n].double(), inner[e, :F].double()
        g, got = xe @ Ge.t(), kept.pre[a:a + n, 0, :F].double()
        lim = 2 * U * g.abs() + 2 * H * U * U * (xe.abs() @ Ge.abs().t())
        S = xe.norm(dim=1)[:, None] * Ge.norm(dim=1) / math.sqrt(H)
        assert ((got - g).abs() <= lim)[g.abs() < 2 * H * U * S / 16].all()
        assert ((got > 0) == (g > 0))[g.abs() > lim].all()
        a += n


@pytest.mark.parametrize("M", [1, 2, 4, 8])
@pytest.mark.parametrize("H,F,dt", [(1024, 2048, "bf16"), (4096, 500, "f16"), (7001, 300, "bf16")])
def test_signs_of_gates_of_few_rows(mm, M, H, F, dt):
    # One block, few rows: sums in 32 bits, each thread over 8 in 2048 elements in two chains of 4, those and the threads' joined in
    # 1 + 5 + 8 steps; at each step U of the sum on the way, itself below sum |a b|.
    n = 4 * -(-H // 2048) + 14
    plain = rand(M, H, dt=dt, seed=71), rand(F, H, dt=dt, seed=72, size=H ** -0.5)
    for x, G in (plain, cancelling(M, F, H, dt, 73)):
        inner = torch.cat([G, rand(F, H, dt=dt, seed=75, size=H ** -0.5)])
        w = mm.gated_weight(inner, rand(H, F, dt=dt, seed=76, size=F ** -0.5), "relu")
        kept = mm.keep(M, w)
        mm.feed_forward(x, w, keep=kept)
        g, got = x.double() @ G.double().t(), kept.pre[:, 0, :F].double()
        lim = n * (1 + n * U) * U * (x.double().abs() @ G.double().abs().t())
        assert ((got - g).abs() <= lim).all()
        assert ((got > 0) == (g > 0))[g.abs() > lim].all()


@pytest.mark.parametrize("size", [2.0 ** 80, 2.0 ** -60])
def test_signs_of_gates_of_large_and_small_rows(mm, size):
    # the lengths' squares are beyond 32 bits; one row is 0, one is not a number, one infinite: the others' g are summed again
    M, H, F = 64, 2048, 96
    x, inner = rand(M, H, dt="bf16", seed=81) * size, rand(2 * F, H, dt="bf16", seed=82, size=H ** -0.5)
    x[3], x[5, 9], x[7, 9], inner[4], inner[6, 1] = 0, math.nan, math.inf, 0, math.nan
    w = mm.gated_weight(inner, rand(H, F, dt="bf16", seed=83), "relu")
    kept = mm.keep(M, w)
    mm.feed_forward(x, w, keep=kept)
    g, got = x.double() @ inner[:F].double().t(), kept.pre[:, 0, :F].double()
    ok = g.isfinite()
    assert int(ok.sum()) == (M - 2) * (F - 1) and (got.isfinite() == ok).all()
    lim = 2 * U * g.abs() + 2 * H * U * U * (x.double().abs() @ inner[:F].double().abs().t())
    assert ((got - g).abs() <= lim)[ok & (g.abs() < H * 2.0 ** -27 * size)].all()
    assert (got[3] == 0).logical_or(~ok[3]).all() and (got[:, 4] == 0).logical_or(~ok[:, 4]).all()


def test_a_gate_whose_sum_is_cut_off_to_zero(mm):
    # 1 + 2^-30 - 1, a step of 16 apart: the sum on the way holds 24 bits
    M, H, F = 64, 64, 64
    x, inner = rand(M, H, dt="bf16", seed=91), rand(2 * F, H, dt="bf16", seed=92, size=H ** -0.5)
    x[9], inner[5] = 0, 0
    for k, v in ((0, 1.0), (17, 2.0 ** -30), (40, -1.0)):
        x[9, k], inner[5, k] = v, 1.0
    w = mm.gated_weight(inner, rand(H, F, dt="bf16", seed=93), "relu")
    kept = mm.keep(M, w)
    mm.feed_forward(x, w, keep=kept)
    assert float(kept.pre[9, 0, 5]) == 2.0 ** -30
    # rows without common elements: many sums of exactly 0 stay what they are
    x[:, ::2], inner[:F, 1::2] = 0, 0
    mm.feed_forward(x, w, keep=kept)
    assert not kept.pre[:, 0, :F].any()


def test_results_over_what_is_read(mm):
    """Refused wherever they overlap, not where they begin alone; columns of one matrix side by side are taken."""
    from paper_2608_07971_gb300 import esp
    M, H, F = 40, 64, 64
    bf = dict(dtype=torch.bfloat16, device="cuda")
    inner, outer = rand(1, 2 * F, H, dt="bf16", seed=2), rand(1, H, F, dt="bf16", seed=3)
    w = mm.gated_weight(inner, outer)
    room = torch.zeros(2 * M, 3 * H, **bf)
    x, dy, dx = (room[:M, i * H:(i + 1) * H] for i in range(3))
    x.copy_(rand(M, H, dt="bf16", seed=1))
    dy.copy_(rand(M, H, dt="bf16", seed=4))
    kept = mm.keep(M, w)
    y = mm.feed_forward(x, w, keep=kept, out=room[M:, :H])            # below x, beside dy
    want = mm.feed_forward_backward(dy.clone(), x.clone(), w, kept)
    got = mm.feed_forward_backward(dy, x, w, kept, out=(dx, None, None))
    assert torch.equal(y, mm.feed_forward(x.clone(), w)) and all(torch.equal(a, b) for a, b in zip(got, want))
    flat = torch.zeros(3 * H * F, **bf)
    apart = flat[:2 * H * F].view(1, 2 * F, H), flat[2 * H * F:].view(1, H, F)
    assert all(torch.equal(a, b) for a, b in zip(mm.feed_forward_backward(dy, x, w, kept, out=(None, *apart))[1:], want[1:]))
    some = dy.clone()
    assert torch.equal(mm.feed_forward(some, w, out=some), mm.feed_forward(dy, w))   # nothing is kept: in place
    before = room.clone(), kept.pre.clone(), kept.hidden.clone(), inner.clone(), outer.clone()
    both = flat[:2 * H * F].view(1, 2 * F, H), flat[H * F:2 * H * F].view(1, H, F)
    backward = lambda **a: mm.feed_forward_backward(dy, x, w, kept, **a)   # noqa: E731
    for f in (lambda: mm.feed_forward(x, w, keep=kept, out=room[:M, 8:H + 8]), lambda: mm.feed_forward(x, w, keep=kept, out=room[M - 1:2 * M - 1, :H]),
              lambda: mm.feed_forward(x, w, keep=kept, out=kept.hidden),
              lambda: mm.feed_forward(x, w, out=inner.view(-1)[:M * H].view(M, H)), lambda: mm.feed_forward(x, w, out=outer.view(-1)[-M * H:].view(M, H)),
              lambda: backward(out=(room[:M, H + 8:2 * H + 8], None, None)), lambda: backward(out=(room[M - 1:2 * M - 1, :H], None, None)),
              lambda: backward(out=(kept.hidden, None, None)), lambda: backward(out=(None, inner, None)),
              lambda: backward(out=(None, None, outer)), lambda: backward(out=(None, *both))):
        with pytest.raises((esp.EspError, ValueError)) as err:
            f()
        assert err.type is ValueError or err.value.status == esp.ESP_ERR_INVALID_ARG
    assert all(torch.equal(a, b) for a, b in zip(before, (room, kept.pre, kept.hidden, inner, outer)))
    rows = torch.arange(M, dtype=torch.int32, device="cuda")           # copied: x is not read again
    mm.feed_forward(x, w, rows=rows, keep=kept, out=y)
    assert torch.equal(mm.feed_forward_backward(dy, x, w, kept, rows=rows, out=(x, None, None))[0], want[0])
    with pytest.raises(esp.EspError):
        mm.feed_forward_backward(dy, x, w, kept, rows=rows, out=(kept.rows, None, None))
    mm.synchronize()
