"""The expert layer's CUDA path (include/esp_moe.h) against the fp64 oracle (oracle/moe_oracle.py).

Integers are compared for equality. Bounds for the rest, u = 2^-24 (fp32) and r the rounding unit of the
result's type (fp32 u, bf16 2^-8, fp16 2^-11 and 2^-25 absolute below its normal range):
  exponentials  exp(a - m) is within (2 |a - m| + 4) u of its value (the rounded argument, 2 ulp of expf),
                log sigmoid within 4 ulp; sums of a row add at most 40 roundings: with R = min(max |z|, 104)
                (smaller terms vanish) a softmax is within C u, C = 8 R + 200, relative.
  gradients     p (g - sum g p): C u p (|g| + sum |g| p), then r.
  losses, shares of n tokens: (C + n) u relative.
  products      128 products of a block are summed with at most 2 u each (a truncating adder), a scale is
                applied (2 roundings), at most nb blocks are added: (2 * 128 + nb + 8) u sum |x w|, then r.
  combine       (k + 2) u sum |w y|; its inner products (H + 8) u sum |d y|.
"""

import math

import numpy as np
import pytest

from oracle import moe_oracle as mo

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
UNIT = {"f32": (U, 2.0 ** -149), "bf16": (2.0 ** -8, 2.0 ** -134), "f16": (2.0 ** -11, 2.0 ** -25)}


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


def Gate(*a, **k):
    from paper_2608_07971_gb300 import moe
    return moe.Gate(*a, **k)


def dev(a, dt=None):
    t = torch.as_tensor(np.ascontiguousarray(a)).cuda()
    return t if dt is None else t.to(DT[dt])


def host(t):
    return t.detach().float().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def close(got, want, bound, dt="f32"):
    """|got - want| <= bound + rounding of the result's type; NaN only where wanted."""
    got, want = np.asarray(host(got), np.float64), np.asarray(want, np.float64)
    assert got.shape == want.shape
    rel, absolute = UNIT[dt]
    lim = bound + rel * np.abs(want) + rel * bound + absolute
    bad = ~(np.abs(got - want) <= lim) & ~(np.isnan(got) & np.isnan(want))
    assert not bad.any(), f"{bad.sum()} of {bad.size} off, worst {np.nanmax(np.abs(got - want) / lim):.3g} of the bound"


def make_logits(T, E, dt, seed=0, masked=False):
    rng = np.random.default_rng(seed)
    z = rng.normal(size=(T, E)) * 2.0
    z = dev(z, dt)
    if masked:
        closed = torch.as_tensor(rng.random((T, E)) < 0.3).cuda()
        z = torch.where(closed, torch.full_like(z, -math.inf), z)
        low = torch.as_tensor(rng.random((T, E)) < 0.1).cuda()
        z = torch.where(low, torch.full_like(z, torch.finfo(z.dtype).min), z)
        if T > 2:
            z[1] = -math.inf                       # nothing open
            z[2] = torch.finfo(z.dtype).min        # all at the lowest value
            z[T // 2, 0] = math.nan
            z[T - 1, E - 1] = math.inf
    return z


def const(z):
    f = np.abs(host(z))
    return (8.0 * min(float(f[np.isfinite(f)].max(initial=0.0)), 104.0) + 200.0) * U


ROUTES = [  # T, E, k, type, gate, renorm, prices, masked
    (1, 1, 1, "f32", "softmax", True, False, False),
    (1, 64, 6, "bf16", "softmax", True, True, False),
    (3, 5, 5, "f16", "sigmoid", True, True, True),
    (40, 31, 4, "f32", "softmax", False, True, True),
    (70, 33, 32, "bf16", "sigmoid", False, False, True),
    (257, 64, 8, "f32", "sigmoid", True, True, True),
    (600, 134, 5, "f16", "softmax", True, True, True),
    (1111, 256, 8, "bf16", "softmax", False, True, False),
    (300, 511, 3, "bf16", "sigmoid", True, False, True),
    (130, 1024, 32, "f32", "softmax", True, True, True),
    (5000, 12, 1, "bf16", "softmax", True, True, True),
]


@pytest.mark.parametrize("T,E,k,dt,gate,renorm,priced,masked", ROUTES)
def test_route(mm, T, E, k, dt, gate, renorm, priced, masked):
    rng = np.random.default_rng(T * 7 + E)
    z = make_logits(T, E, dt, T + E, masked)
    prices = np.maximum(0.0, rng.normal(size=E)).astype(np.float32) if priced else None
    valid = rng.random(T) < 0.8 if masked else None
    r = mm.route(z, k, gate=Gate(gate, renorm, 1.5), prices=None if prices is None else dev(prices),
                 valid=None if valid is None else dev(valid))
    idx = mo.choose(host(z), k, prices, valid)
    assert np.array_equal(host(r.idx), idx)
    counts, offsets, rows, pos = mo.plan(idx, E)
    for got, want in ((r.counts, counts), (r.offsets, offsets), (r.rows, rows), (r.pos, pos)):
        assert np.array_equal(host(got), want)
    w = mo.gate_weight(host(z), idx, gate, renorm, 1.5)
    close(r.weight, w, const(z) * w + 2.0 ** -120)
    bare = mm.route(z, k, gate=Gate(gate, renorm, 1.5), prices=None if prices is None else dev(prices),
                    valid=None if valid is None else dev(valid), plan=False)
    assert bare.rows is None and torch.equal(bare.idx, r.idx) and torch.equal(bare.counts, r.counts)


@pytest.mark.parametrize("T,E,k,dt,gate,renorm,priced,masked", ROUTES)
def test_route_backward(mm, T, E, k, dt, gate, renorm, priced, masked):
    rng = np.random.default_rng(T * 5 + E)
    z = make_logits(T, E, dt, T + E, masked)
    idx = mo.choose(host(z), k, None, rng.random(T) < 0.9 if masked else None)
    g = rng.normal(size=(T, k)).astype(np.float32)
    got = mm.route_backward(z, dev(idx.astype(np.int32)), gate=Gate(gate, renorm, 1.5), dweight=dev(g))
    want = mo.gate_weight_grad(host(z), idx, gate, renorm, 1.5, g)
    p = mo.gate_weight(host(z), idx, gate, renorm, 1.5)
    size = (np.abs(g) * p).sum(1, keepdims=True) + 1.5 * np.abs(g).max()
    close(got, want, const(z) * size, dt)


BALANCES = [  # T, E, k, type, gate, sequence bounds, masked
    (1, 4, 1, "f32", "softmax", None, False),
    (50, 8, 2, "f32", "sigmoid", None, True),
    (500, 61, 3, "bf16", "softmax", [0, 0, 13, 13, 200, 499, 500], True),
    (333, 256, 8, "f16", "sigmoid", [0, 100, 101, 333], False),
    (200, 700, 4, "f32", "softmax", list(range(0, 201, 4)), True),
    (1000, 17, 2, "bf16", "sigmoid", [0, 1000], False),
]


@pytest.mark.parametrize("T,E,k,dt,gate,seq,masked", BALANCES)
def test_balance_and_its_gradient(mm, T, E, k, dt, gate, seq, masked):
    rng = np.random.default_rng(E)
    z = make_logits(T, E, dt, E, masked)
    if masked:
        z = torch.where(torch.isinf(z) & (z > 0), torch.zeros_like(z), z)   # a logit of +inf has no finite loss
        z = torch.where(z == torch.finfo(z.dtype).min, torch.full_like(z, -30.0), z)
    idx = mo.choose(host(z), k, None, rng.random(T) < 0.8 if masked else None)
    di, ds = dev(idx.astype(np.int32)), None if seq is None else dev(np.asarray(seq, np.int32))
    b = mm.balance(z, di, gate=Gate(gate), seq_offsets=ds)
    loss, counts, share, tokens = mo.balance(host(z), idx, gate, seq)
    assert np.array_equal(host(b.counts), counts) and np.array_equal(host(b.tokens), tokens)
    c = const(z) + T * U
    close(b.share, share, c * share)
    close(b.loss, loss, 4 * c * (loss + 1.0))
    d = np.array([3.0, 0.25], np.float32)
    got = mm.route_backward(z, di, gate=Gate(gate), balance=b, seq_offsets=ds, dloss=dev(d))
    want = mo.balance_grad(host(z), idx, gate, d, seq)
    n, used = max(tokens.sum(), 1), max((tokens > 0).sum(), 1)
    size = 3.0 * E / (np.maximum(tokens, 1).min() * used) + 0.25 * 2 * (np.abs(host(z))[np.isfinite(host(z))].max() + 8) / n
    close(got, want, c * size, dt)
    # both sources of gradient in one call: their sum
    g = rng.normal(size=(T, k)).astype(np.float32)
    both = mm.route_backward(z, di, gate=Gate(gate), dweight=dev(g), balance=b, seq_offsets=ds, dloss=dev(d))
    close(both, want + mo.gate_weight_grad(host(z), idx, gate, True, 1.0, g), c * (size + 2 * np.abs(g).max()), dt)


def test_gradients_against_differences(mm):
    """The losses and weighted gate weights that the kernels return, differenced in single logits."""
    T, E, k, h = 12, 10, 3, 2.0 ** -5
    z = make_logits(T, E, "f32", 5)
    g = dev(np.random.default_rng(6).normal(size=(T, k)).astype(np.float32))
    seq, dl = dev(np.asarray([0, 5, 12], np.int32)), dev(np.asarray([2.0, 0.5], np.float32))
    for gate in (Gate("softmax"), Gate("sigmoid"), Gate("softmax", False), Gate("sigmoid", False)):
        idx = mm.route(z, k, gate=gate).idx
        b = mm.balance(z, idx, gate=gate, seq_offsets=seq)
        dz = host(mm.route_backward(z, idx, gate=gate, dweight=g, balance=b, seq_offsets=seq, dloss=dl))

        def value(v):
            r = mm.route(v, k, gate=gate)
            assert torch.equal(r.idx, idx)
            lo = mm.balance(v, idx, gate=gate, seq_offsets=seq).loss
            return float((r.weight.double() * g.double()).sum() + (lo.double() * dl.double()).sum())

        for t, e in ((0, 1), (4, 9), (5, 0), (11, 4)):
            f = []
            for s in (-h, h):
                v = z.clone()
                v[t, e] += s
                try:
                    f.append(value(v))
                except AssertionError:
                    f = []
                    break
            if len(f) == 2:
                # step error h^2 / 6 * third derivative (bounded by about 4), fp32 values of size 10 over 2 h
                assert abs((f[1] - f[0]) / (2 * h) - dz[t, e]) < 4 * h * h / 6 + 20 * 400 * U / (2 * h)


def test_step_prices(mm):
    rng = np.random.default_rng(0)
    for E in (1, 7, 1024):
        p, c = rng.random(E).astype(np.float32), rng.integers(0, 50, E)
        d = dev(p)
        mm.step_prices(d, dev(c), 0.05, 1.25)
        close(d, mo.step_prices(p, c, 0.05, 1.25), 2 * U)
    d = dev(np.ones(3, np.float32))
    mm.step_prices(d, dev(np.zeros(3, np.int64)), 0.05)
    assert host(d).tolist() == [1.0, 1.0, 1.0]


def test_prices_level_the_load(mm):
    """Repeated routing and price steps bring a skewed load near its mean (tatonnement)."""
    T, E, k = 4096, 16, 2
    z = make_logits(T, E, "f32", 1) + torch.linspace(0, 4, E).cuda()
    prices = torch.zeros(E, device="cuda")
    first = mm.route(z, k, prices=prices).counts.float()
    for _ in range(200):
        mm.step_prices(prices, mm.route(z, k, prices=prices).counts, 0.1)
    last = mm.route(z, k, prices=prices).counts.float()
    mean = T * k / E
    assert first.max() > 2.5 * mean and last.max() < 1.25 * mean


# ---- products

PRODUCTS = [  # sizes of the experts' rows, N, K, type, gathered
    ([1], 1, 1, "f32", False),
    ([1], 64, 128, "bf16", False),
    ([0], 16, 16, "bf16", False),
    ([130], 129, 257, "f16", False),
    ([3, 0, 1, 200, 0], 100, 300, "bf16", True),
    ([0, 0, 5], 260, 64, "f32", True),
    ([127, 128, 129], 384, 512, "bf16", True),
    ([1] * 40, 72, 1030, "f16", True),
    ([700, 33], 511, 140, "f32", False),
]


def product_inputs(sizes, N, K, dt, gathered, seed=0):
    rng = np.random.default_rng(seed + N + K)
    M = sum(sizes)
    T = max(1, M // 2) if gathered else M
    x = dev(rng.normal(size=(T, K)) * np.where(rng.random(K) < 0.05, 20.0, 1.0), dt)
    rows = rng.integers(0, T, M).astype(np.int32) if gathered else None
    w = dev(rng.normal(size=(len(sizes), N, K)) / math.sqrt(K), dt)
    offsets = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
    return x, rows, w, offsets


def product_bound(mag, blocks):
    return (2 * 128 + blocks + 8) * U * mag


@pytest.mark.parametrize("sizes,N,K,dt,gathered", PRODUCTS)
def test_linear_and_its_gradients(mm, sizes, N, K, dt, gathered):
    x, rows, w, offsets = product_inputs(sizes, N, K, dt, gathered)
    weights = [mo.quantize_weight(host(w[e])) for e in range(len(sizes))]
    q = mm.quantize_weight(w, transposed=True)
    assert np.array_equal(host(q.codes()), np.stack([c for c, _ in weights]))
    assert np.array_equal(host(q.scale), np.stack([s for _, s in weights]))
    if N <= q.qt.shape[2]:
        back = q.qt.view(torch.float8_e4m3fn)[:, :, :N].transpose(1, 2)
        assert np.array_equal(host(back), host(q.codes()))
    off = dev(offsets) if len(sizes) > 1 or gathered else None
    dr = None if rows is None else dev(rows)
    y = mm.linear(x, q, offsets=off, rows=dr)
    want, mag = mo.linear(host(x), weights, offsets, rows)
    close(y, want, product_bound(mag, -(-K // 128)), dt)
    M = sum(sizes)
    dy = dev(np.random.default_rng(1).normal(size=(M, N)) * 0.01, dt)
    dx, dw = mm.linear_backward(dy, x, q, offsets=off, rows=dr)
    wx, mx, ww, mw = mo.linear_backward(host(dy), host(x), weights, offsets, rows)
    close(dx, wx, product_bound(mx, -(-N // 128)), dt)
    close(dw, ww, product_bound(mw, max(sizes) // 128 + 1))
    only, none = mm.linear_backward(dy, x, q, offsets=off, rows=dr, need=(True, False))
    assert torch.equal(only, dx) and none is None
    none, only = mm.linear_backward(dy, x, q, offsets=off, rows=dr, need=(False, True))
    assert torch.equal(only, dw) and none is None


@pytest.mark.parametrize("M,N,K", [(1, 4096, 4096), (2, 1000, 4096), (16, 2048, 2000), (33, 512, 8192),
                                   (300, 256, 4096), (2000, 1100, 600), (1500, 2304, 384)])
def test_linear_long(mm, M, N, K):
    """Long inner axes with few rows, and many tiles: against the same codes in fp64 on the GPU."""
    g = torch.Generator(device="cuda").manual_seed(M)
    x = torch.randn(M, K, generator=g, device="cuda").bfloat16()
    w = (torch.randn(N, K, generator=g, device="cuda") / math.sqrt(K)).bfloat16()
    q = mm.quantize_weight(w)
    y = mm.linear(x, q)
    codes, scale = mo.quantize_rows(host(x))
    xd = torch.as_tensor(mo.spread_rows(codes, scale)).cuda()
    s = q.scale[0].double().repeat_interleave(128, 0)[:N].repeat_interleave(128, 1)[:, :K]
    wd = q.codes()[0].double() * s
    want, mag = (xd @ wd.t()).cpu().numpy(), (xd.abs() @ wd.abs().t()).cpu().numpy()
    close(y, want, product_bound(mag, -(-K // 128)), "bf16")
    again = mm.linear(x, q)
    assert torch.equal(y, again)


def test_linear_leaves_other_rows(mm):
    x, _, w, _ = product_inputs([200, 100], 130, 200, "bf16", False)
    q = mm.quantize_weight(w)
    out = torch.full((300, 130), 7.0, dtype=torch.bfloat16, device="cuda")
    offsets = np.array([3, 150, 290], np.int32)
    mm.linear(x, q, offsets=dev(offsets), out=out)
    weights = [mo.quantize_weight(host(w[e])) for e in range(2)]
    want, mag = mo.linear(host(x), weights, offsets)
    close(out[3:290], want[3:290], product_bound(mag[3:290], 2), "bf16")
    assert bool((out[:3] == 7).all()) and bool((out[290:] == 7).all())


def test_linear_rows_past_the_plan(mm):
    """rows of -1 past the last expert's, as a plan with padding leaves them."""
    x, _, w, _ = product_inputs([4, 4], 40, 70, "f32", False)
    q = mm.quantize_weight(w)
    rows = np.array([7, 0, 0, 5, -1, -1], np.int32)
    y = mm.linear(x, q, offsets=dev(np.array([0, 1, 4], np.int32)), rows=dev(rows))
    weights = [mo.quantize_weight(host(w[e])) for e in range(2)]
    want, mag = mo.linear(host(x), weights, [0, 1, 4], rows)
    close(y[:4], want[:4], product_bound(mag[:4], 1))


def test_values_that_are_not_finite(mm):
    x = torch.ones(5, 300, device="cuda")
    x[1, 130], x[3, 2] = math.inf, math.nan
    w = torch.ones(1, 20, 300, device="cuda") * 0.5
    q = mm.quantize_weight(w)
    y = host(mm.linear(x, q))
    assert np.isnan(y[[1, 3]]).all() and np.isfinite(y[[0, 2, 4]]).all()
    # gathered rows do not read the others
    y = host(mm.linear(x, q, offsets=dev(np.array([0, 2], np.int32)), rows=dev(np.array([2, 4], np.int32))))
    assert np.isfinite(y).all()
    w[0, 3, 5] = math.nan
    assert np.isnan(host(mm.quantize_weight(w).scale)).tolist() == [[[True, False, False]]]


def test_zero_and_tiny_blocks(mm):
    x = torch.zeros(2, 256, device="cuda")
    x[1, 0], x[1, 200] = 2.0 ** -140, 3.0 * 2.0 ** 100
    w = torch.randn(1, 16, 256, device="cuda")
    q = mm.quantize_weight(w)
    want, mag = mo.linear(host(x), [mo.quantize_weight(host(w[0]))], [0, 2])
    close(mm.linear(x, q), want, product_bound(mag, 2))


def test_loaded_weights(mm):
    for N, K in ((48, 160), (50, 77)):
        w = torch.randn(3, N, K, device="cuda")
        a = mm.quantize_weight(w, transposed=True)
        b = mm.load_weight(a.codes().contiguous(), a.scale, transposed=True)
        x = torch.randn(9, K, device="cuda")
        off = dev(np.array([0, 2, 2, 9], np.int32))
        assert torch.equal(mm.linear(x, a, offsets=off), mm.linear(x, b, offsets=off))
        dy = torch.randn(9, N, device="cuda")
        assert torch.equal(mm.linear_backward(dy, x, a, offsets=off)[0], mm.linear_backward(dy, x, b, offsets=off)[0])


# ---- combine

@pytest.mark.parametrize("T,k,H,dt", [(1, 1, 1, "f32"), (1, 6, 2048, "bf16"), (37, 3, 293, "f16"), (64, 8, 512, "f32"),
                                      (20, 32, 40, "bf16"), (129, 2, 4096, "bf16"), (11, 9, 1000, "f16")])
def test_combine_and_its_gradients(mm, T, k, H, dt):
    rng = np.random.default_rng(T + H)
    M = T * k
    pos = rng.permutation(M).reshape(T, k).astype(np.int32)
    pos[rng.random((T, k)) < 0.1] = -1
    y, d = dev(rng.normal(size=(M, H)), dt), dev(rng.normal(size=(T, H)), dt)
    w = rng.normal(size=(T, k)).astype(np.float32)
    for weight in (w, None):
        dwt = None if weight is None else dev(weight)
        out = mm.combine(y, dev(pos), dwt)
        mag = mo.combine(np.abs(host(y)), pos, None if weight is None else np.abs(weight))
        close(out, mo.combine(host(y), pos, weight), (k + 2) * U * mag, dt)
        dy, dw = mm.combine_backward(d, y, dev(pos), dwt)
        wy, ww = mo.combine_grad(host(d), host(y), pos, weight)
        close(dy, wy, U * np.abs(wy), dt)
        _, mag = mo.combine_grad(np.abs(host(d)), np.abs(host(y)), pos)
        close(dw, ww, (H + 8) * U * mag)


# ---- layout, streams, refusals

def test_strided_and_misaligned_inputs(mm):
    """Views into wider buffers, starting at an odd element, give what their copies give."""
    for dt in DT.values():
        base = torch.randn(40, 333, device="cuda").to(dt)
        z = base[:, 5:5 + 131]
        a, b = mm.route(z, 4), mm.route(z.contiguous(), 4)
        assert torch.equal(a.idx, b.idx) and torch.equal(a.weight, b.weight)
        g = torch.randn(40, 4, device="cuda")
        wide = torch.zeros(40, 200, dtype=dt, device="cuda")
        mm.route_backward(z, a.idx, dweight=g, out=wide[:, 3:134])
        assert torch.equal(wide[:, 3:134], mm.route_backward(z.contiguous(), a.idx, dweight=g))
        assert not wide[:, :3].any() and not wide[:, 134:].any()
        q = mm.quantize_weight(torch.randn(60, 131, device="cuda").to(dt), transposed=True)
        out = torch.zeros(40, 77, dtype=dt, device="cuda")
        mm.linear(z, q, out=out[:, 9:69])
        y = mm.linear(z.contiguous(), q)
        assert torch.equal(out[:, 9:69], y) and not out[:, :9].any() and not out[:, 69:].any()
        dx, dw = mm.linear_backward(out[:, 9:69], z, q)
        dx2, dw2 = mm.linear_backward(y, z.contiguous(), q)
        assert torch.equal(dx, dx2) and torch.equal(dw, dw2)
        pos = torch.randperm(40, device="cuda").int().reshape(20, 2)
        assert torch.equal(mm.combine(z, pos), mm.combine(z.contiguous(), pos))


def test_offsets_past_32_bits(mm):
    """Rows whose element offsets pass 2^31."""
    ld = 1 << 20
    base = torch.empty(2100, ld, dtype=torch.bfloat16, device="cuda")
    z = base[:, 3:67]
    z.copy_(torch.randn(2100, 64, device="cuda"))
    a, b = mm.route(z, 4), mm.route(z.contiguous(), 4)
    assert torch.equal(a.idx, b.idx)
    q = mm.quantize_weight(torch.randn(32, 64, device="cuda"))
    assert torch.equal(mm.linear(z, q), mm.linear(z.contiguous(), q))
    pos = torch.arange(2099, -1, -1, device="cuda").int().reshape(-1, 3)
    assert torch.equal(mm.combine(z, pos), mm.combine(z.contiguous(), pos))


def test_empty(mm):
    z = torch.empty(0, 8, device="cuda")
    r = mm.route(z, 2)
    assert not host(r.counts).any() and not host(r.offsets).any() and r.idx.shape == (0, 2)
    b = mm.balance(z, r.idx)
    assert not host(b.loss).any() and not host(b.counts).any() and not host(b.share).any() and not host(b.tokens).any()
    assert mm.route_backward(z, r.idx, dweight=r.weight).shape == (0, 8)
    q = mm.quantize_weight(torch.randn(2, 10, 8, device="cuda"), transposed=True)
    y = mm.linear(z, q, offsets=dev(np.zeros(3, np.int32)))
    assert y.shape == (0, 10)
    dx, dw = mm.linear_backward(y, z, q, offsets=dev(np.zeros(3, np.int32)))
    assert dx.shape == (0, 8) and not host(dw).any()
    assert mm.combine(y, r.pos, r.weight).shape == (0, 10)


def test_repeatable(mm):
    z = make_logits(3000, 64, "bf16", 9)
    r = mm.route(z, 4)
    b = mm.balance(z, r.idx)
    for _ in range(3):
        s = mm.route(z, 4)
        c = mm.balance(z, r.idx)
        assert torch.equal(r.rows, s.rows) and torch.equal(b.loss, c.loss) and torch.equal(b.share, c.share)


def test_other_streams(mm):
    """Calls follow the caller's current stream, one handle's work in order across streams."""
    from paper_2608_07971_gb300 import moe
    m = moe.Moe()
    z = make_logits(4000, 64, "f32", 3)
    want = m.route(z, 4)
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(5):
        with torch.cuda.stream(s1):
            a = m.route(z, 4)
        with torch.cuda.stream(s2):
            b = m.route(z, 4)
    m.synchronize()
    torch.cuda.synchronize()
    assert torch.equal(a.rows, want.rows) and torch.equal(b.rows, want.rows)
    with torch.cuda.stream(s1):
        m.linear(torch.randn(8, 64, device="cuda"), m.quantize_weight(torch.randn(32, 64, device="cuda")))
    m.synchronize()
    m.close()


def test_graph_capture(mm):
    from paper_2608_07971_gb300 import moe
    m = moe.Moe()
    z = make_logits(900, 64, "bf16", 4)
    x, w = torch.randn(900, 128, device="cuda").bfloat16(), torch.randn(64, 96, 128, device="cuda").bfloat16()
    q = m.quantize_weight(w)
    r, y, out = m.routing(900, 64, 4), torch.empty(3600, 96, dtype=torch.bfloat16, device="cuda"), \
        torch.empty(900, 96, dtype=torch.bfloat16, device="cuda")

    def layer():
        m.route(z, 4, out=r)
        m.linear(x, q, offsets=r.offsets, rows=r.rows, out=y)
        m.combine(y, r.pos, r.weight, out=out)

    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        layer()
    torch.cuda.synchronize()
    want = out.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        layer()
    out.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    m.close()


def test_refusals(mm):
    from paper_2608_07971_gb300 import esp
    z = torch.randn(4, 8, device="cuda")
    idx = torch.zeros(4, 2, dtype=torch.int32, device="cuda")
    q = mm.quantize_weight(torch.randn(2, 10, 8, device="cuda"))
    bad = [
        lambda: mm.route(z.cpu(), 2),
        lambda: mm.route(z.double(), 2),
        lambda: mm.route(z.t(), 2),
        lambda: mm.route(z, 2, prices=torch.zeros(7, device="cuda")),
        lambda: mm.route(z, 2, valid=torch.ones(4, device="cuda")),
        lambda: mm.route(z, 2, out=mm.routing(4, 8, 3)),
        lambda: mm.balance(z, idx.long()),
        lambda: mm.balance(z, idx[:3]),
        lambda: mm.route_backward(z, idx, dloss=torch.zeros(2, device="cuda")),
        lambda: mm.route_backward(z, idx, out=torch.empty(4, 9, device="cuda")),
        lambda: mm.linear(z, q),
        lambda: mm.linear(z[:, :7], q, offsets=torch.zeros(3, dtype=torch.int32, device="cuda")),
        lambda: mm.linear_backward(torch.zeros(4, 10, device="cuda"), z, q,
                                   offsets=torch.zeros(3, dtype=torch.int32, device="cuda")),
        lambda: mm.load_weight(torch.zeros(2, 10, 8, device="cuda"), q.scale),
        lambda: mm.combine(z, idx, torch.ones(4, 3, device="cuda")),
    ]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    for f in (lambda: mm.route(z, 0), lambda: mm.route(z, 9), lambda: mm.route(torch.randn(2, 1025, device="cuda"), 2),
              lambda: mm.route(torch.zeros(1, 8, device="cuda").expand(4, 8), 2),
              lambda: mm.combine(z, torch.zeros(1, 33, dtype=torch.int32, device="cuda")),
              lambda: mm.step_prices(torch.zeros(3, device="cuda"), torch.zeros(3, dtype=torch.int64, device="cuda"),
                                     0.0)):
        with pytest.raises(esp.EspError) as err:
            f()
        assert err.value.status == esp.ESP_ERR_INVALID_ARG
    mm.route(z, 2)   # a refusal leaves the handle usable
    mm.synchronize()


@pytest.mark.parametrize("M", [40, 2000])
def test_wait_that_runs_out_is_reported(mm, M):
    """A product whose load never comes ends by its bounded waits; the handle then refuses work."""
    from paper_2608_07971_gb300 import esp, moe
    m = moe.Moe()
    x, w = torch.randn(M, 1024, device="cuda"), torch.randn(300, 1024, device="cuda")
    q = m.quantize_weight(w)
    want = m.linear(x, q)
    m.synchronize()
    lib = moe.load_library()
    esp._check(lib.esp_moe_debug_set_wait_limit(m.h, 20), "set_wait_limit")
    esp._check(lib.esp_moe_debug_hold_load(m.h), "hold_load")
    m.linear(x, q)
    with pytest.raises(esp.EspError) as err:
        m.synchronize()
    assert err.value.status == esp.ESP_ERR_TIMEOUT
    with pytest.raises(esp.EspError) as err:
        m.linear(x, q)
    assert err.value.status == esp.ESP_ERR_STATE
    m.close()
    assert torch.equal(mm.linear(x, q), want)   # another handle works on


def test_wait_that_runs_out_in_the_weight_gradient(mm):
    from paper_2608_07971_gb300 import esp, moe
    for M, N, K in ((900, 300, 500), (300, 2100, 2000)):
        m = moe.Moe()
        x, dy = torch.randn(M, K, device="cuda"), torch.randn(M, N, device="cuda")
        q = m.quantize_weight(torch.randn(N, K, device="cuda"))
        want = m.linear_backward(dy, x, q, need=(False, True))[1]
        m.synchronize()
        lib = moe.load_library()
        esp._check(lib.esp_moe_debug_set_wait_limit(m.h, 20), "set_wait_limit")
        esp._check(lib.esp_moe_debug_hold_load(m.h), "hold_load")
        m.linear_backward(dy, x, q, need=(False, True))
        with pytest.raises(esp.EspError) as err:
            m.synchronize()
        assert err.value.status == esp.ESP_ERR_TIMEOUT
        m.close()
        assert torch.equal(mm.linear_backward(dy, x, q, need=(False, True))[1], want)


def test_capture_on_another_stream(mm):
    """Calls captured on a stream that the handle has not used, then replayed and called directly."""
    z = make_logits(700, 32, "f32", 8)
    want = mm.route(z, 3)
    r = mm.routing(700, 32, 3)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=torch.cuda.Stream()):
        mm.route(z, 3, out=r)
    r.rows.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(r.rows, want.rows) and torch.equal(r.weight, want.weight)
    assert torch.equal(mm.route(z, 3).rows, want.rows)


def test_weight_refusals(mm):
    from paper_2608_07971_gb300 import moe
    u8 = lambda *s: torch.zeros(*s, dtype=torch.uint8, device="cuda")  # noqa: E731
    f32 = lambda *s: torch.zeros(*s, device="cuda")  # noqa: E731
    moe.Weight(2, 10, 8, u8(2, 10, 16), f32(2, 1, 1))
    for q, scale, qt in ((u8(2, 10, 7), f32(2, 1, 1), None), (u8(2, 9, 16), f32(2, 1, 1), None),
                         (u8(2, 10, 16).float(), f32(2, 1, 1), None), (u8(2, 10, 16), f32(2, 1), None),
                         (u8(2, 10, 16), f32(2, 1, 1), u8(2, 7, 16)), (u8(2, 10, 32)[:, :, ::2], f32(2, 1, 1), None)):
        with pytest.raises(ValueError):
            moe.Weight(2, 10, 8, q, scale, qt)
    from paper_2608_07971_gb300 import esp
    with pytest.raises(esp.EspError):   # rows of codes not a multiple of 16 bytes apart
        mm.linear(f32(3, 8), moe.Weight(1, 10, 8, u8(1, 10, 8), f32(1, 1, 1)))
    with pytest.raises(ValueError):
        mm.quantize_weight(torch.randn(8, 10, device="cuda").t())


@pytest.mark.parametrize("T,E,k,N,K,dt", [(3000, 5, 4, 1040, 1408, "bf16"), (2100, 1, 8, 300, 2050, "f16"),
                                          (9000, 40, 3, 1000, 640, "f32")])
def test_rows_picked_after_rounding(mm, T, E, k, N, K, dt):
    """Many rows for each token: they are rounded once and copied, with the results of rows picked before."""
    g = torch.Generator(device="cuda").manual_seed(T)
    x = torch.randn(T, K, generator=g, device="cuda").to(DT[dt])
    q = mm.quantize_weight(torch.randn(E, N, K, generator=g, device="cuda") / math.sqrt(K))
    M = T * k
    rows = torch.randint(0, T, (M,), generator=g, device="cuda").int()
    cut = torch.sort(torch.randint(0, M + 1, (E - 1,), generator=g, device="cuda"))[0].int()
    offsets = torch.cat([cut.new_zeros(1), cut, cut.new_full((1,), M - 7)]).int().sort()[0]
    rows[5], rows[M // 2] = -1, T          # read zeros
    out = torch.full((M, N), 3.0, dtype=DT[dt], device="cuda")
    mm.linear(x, q, offsets=offsets, rows=rows, out=out)
    assert mm.last_launch_count() == 3
    zero = torch.cat([x, torch.zeros(1, K, dtype=x.dtype, device="cuda")])
    picked = zero[torch.where((rows < 0) | (rows >= T), torch.full_like(rows, T), rows).long()]
    want = torch.full((M, N), 3.0, dtype=DT[dt], device="cuda")
    mm.linear(picked, q, offsets=offsets, out=want)
    assert mm.last_launch_count() == 2
    assert torch.equal(out, want) and bool((out[M - 7:] == 3).all())
    mm.synchronize()


@pytest.mark.parametrize("B,T", [(1, 5), (31, 100), (33, 400), (1100, 3000), (2500, 2500)])
def test_balance_over_many_sequences(mm, B, T):
    """Sequences found by searches of different depth, empty ones among them, tokens before and after all."""
    rng = np.random.default_rng(B)
    z = make_logits(T, 6, "f32", B)
    idx = mo.choose(host(z), 2)
    seq = np.sort(rng.integers(1, T - 1, B + 1)).astype(np.int32)
    di, ds = dev(idx.astype(np.int32)), dev(seq)
    b = mm.balance(z, di, seq_offsets=ds)
    loss, counts, share, tokens = mo.balance(host(z), idx, "softmax", seq)
    assert np.array_equal(host(b.counts), counts) and np.array_equal(host(b.tokens), tokens)
    c = const(z) + T * U
    close(b.share, share, c * share)
    close(b.loss, loss, 4 * c * (loss + 1.0))
    d = np.array([1.0, 0.5], np.float32)
    got = mm.route_backward(z, di, balance=b, seq_offsets=ds, dloss=dev(d))
    want = mo.balance_grad(host(z), idx, "softmax", d, seq)
    n, used = max(tokens.sum(), 1), max((tokens > 0).sum(), 1)
    least = tokens[tokens > 0].min() if used and tokens.any() else 1
    size = 6.0 / (least * used) + 2 * 0.5 * (np.abs(host(z)).max() + 2) / n
    close(got, want, c * size)
