"""The losses' gradient, each element against its own fp64 terms, and every gradient against differences at every point.

Bound of an element, u = 2^-24, c = C u the relative error of a softmax (tests/test_moe_gpu.py: C = 8 R + 200), with the
oracle's r, coefficient k_e = g0 E counts / (k n n), dot = sum k r, and for the logit loss p, lse and g1 = 2 dloss / n:
  r (k_e - dot): r and dot are within c and c + 50 u of their own size, k_e within 6 u: 3 c r (k_e + dot) in all
  times sigmoid(-z), within c: 4 c
  g1 lse p: lse is within 2 c (1 + |lse|), p within c: 4 c |g1| (1 + |lse|) p
and then the rounding of the result's type. Each test also shows that a gradient without either loss is out of bounds.
"""

import numpy as np
import pytest

from oracle import moe_oracle as mo
from tests.test_moe_gpu import BALANCES, DT, UNIT, U, Gate, close, const, dev, host, make_logits

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


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


def bound_of(z, idx, gate, dloss, seq):
    """The element's bound before the type's rounding, from the oracle's terms."""
    zc = mo._clean(z).astype(np.float64)
    T, E = zc.shape
    k = idx.shape[1]
    seq = np.asarray([0, T] if seq is None else seq)
    _, counts, _, tokens = mo.balance(z, idx, gate, seq)
    used, n = max((tokens > 0).sum(), 1), max(tokens.sum(), 1)
    out = np.zeros((T, E))
    for b in range(len(seq) - 1):
        live = np.arange(seq[b], seq[b + 1])
        live = live[idx[live, 0] >= 0]
        if len(live) == 0:
            continue
        coef = dloss[0] * E * counts[b] / (k * tokens[b]) / (tokens[b] * used)
        r = mo.softmax(mo._values(zc[live], gate))
        size = r * (np.abs(coef) + (np.abs(coef) * r).sum(-1, keepdims=True))
        if gate == "sigmoid":
            size = size * mo.sigmoid(-zc[live])
        lse = mo.logsumexp(zc[live])[:, None]
        out[live] = size + 2 * np.abs(dloss[1]) / n * (1 + np.abs(lse)) * mo.softmax(zc[live])
    return out


def outside(got, want, bound, dt):
    rel, absolute = UNIT[dt]
    return np.abs(got - want) > bound + rel * np.abs(want) + rel * bound + absolute


MANY = [(5, 6, 2, "f32", "softmax", [0, 5], False), (400, 6, 2, "f32", "sigmoid", 33, False),
        (3000, 6, 2, "bf16", "softmax", 1100, False), (2500, 20, 3, "f32", "softmax", 2500, True)]


@pytest.mark.parametrize("T,E,k,dt,gate,seq,masked", BALANCES + MANY)
def test_losses_gradient_by_element(mm, T, E, k, dt, gate, seq, masked):
    rng = np.random.default_rng(T + E)
    if isinstance(seq, int):   # so many sequences, empty ones among them, tokens before and after all
        seq = np.sort(rng.integers(1, T, seq + 1)).tolist()
    z = make_logits(T, E, dt, E, masked)
    if masked:
        z = torch.where(torch.isinf(z) & (z > 0), torch.zeros_like(z), z)
        z = torch.where(z == torch.finfo(z.dtype).min, torch.full_like(z, -30.0), z)
    idx = mo.choose(host(z), k, None, rng.random(T) < 0.8 if masked else None)
    di, ds = dev(idx.astype(np.int32)), None if seq is None else dev(np.asarray(seq, np.int32))
    b = mm.balance(z, di, gate=Gate(gate), seq_offsets=ds)
    d = np.array([3.0, 0.25], np.float32) * (2.0 ** 12 if dt == "f16" else 1.0)   # a program in fp16 scales its loss
    want = mo.balance_grad(host(z), idx, gate, d, seq)
    bound = 4 * const(z) * bound_of(host(z), idx, gate, d, seq)
    close(mm.route_backward(z, di, gate=Gate(gate), balance=b, seq_offsets=ds, dloss=dev(d)), want, bound, dt)
    # what the bounds can tell: a gradient without one of the losses is outside at most elements that are not zero
    for part in ((0.0, 1.0), (1.0, 0.0)):
        less = mo.balance_grad(host(z), idx, gate, d * np.array(part, np.float32), seq)
        assert outside(less, want, bound, dt).sum() > 0.8 * np.count_nonzero(want) > 0


def test_every_gradient_against_differences_at_every_point(mm):
    """Logits at least 0.4 apart within a token, so that no step of 2^-4 changes a choice: each gate's weights and both
    losses. Step error h^2 / 6 times a third derivative of at most 4; the fp32 value, of size 20, is within 400 u of
    itself, twice, over 2 h."""
    T, E, k, h = 8, 10, 3, 2.0 ** -4
    rng = np.random.default_rng(4)
    z = dev(np.stack([rng.permutation(np.linspace(-2.2, 2.2, E)) for _ in range(T)]) + rng.uniform(-0.02, 0.02, (T, E)),
            "f32")
    g = dev(rng.normal(size=(T, k)).astype(np.float32))
    seq, dl = dev(np.asarray([0, 3, 8], np.int32)), dev(np.asarray([2.0, 0.5], np.float32))
    lim = 4 * h * h / 6 + 20 * 400 * U / (2 * h)
    for gate in (Gate("softmax"), Gate("sigmoid"), Gate("softmax", False), Gate("sigmoid", False)):
        idx = mm.route(z, k, gate=gate).idx
        b = mm.balance(z, idx, gate=gate, seq_offsets=seq)
        dz = host(mm.route_backward(z, idx, gate=gate, dweight=g, balance=b, seq_offsets=seq, dloss=dl))

        def value(v):
            r = mm.route(v, k, gate=gate)
            assert torch.equal(r.idx, idx)
            lo = mm.balance(v, idx, gate=gate, seq_offsets=seq).loss
            return float((r.weight.double() * g.double()).sum() + (lo.double() * dl.double()).sum())

        points = 0
        for t in range(T):
            for e in range(E):
                f = []
                for s in (-h, h):
                    v = z.clone()
                    v[t, e] += s
                    f.append(value(v))
                assert abs((f[1] - f[0]) / (2 * h) - dz[t, e]) < lim
                points += 1
        assert points == T * E and np.abs(dz).max() > 10 * lim
