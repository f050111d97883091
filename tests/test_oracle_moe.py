"""The expert layer's oracle (oracle/moe_oracle.py) against hand values and difference quotients (CPU)."""

import numpy as np
import pytest

from oracle import moe_oracle as mo


def logits(T, E, seed=0):
    return np.random.default_rng(seed).normal(size=(T, E)).astype(np.float32)


def numeric(f, z, h=1e-3):
    """Central differences of f in every element of z; f's own error is fp64, the step's is h^2."""
    g = np.zeros(z.shape)
    for i in np.ndindex(z.shape):
        a, b = z.copy(), z.copy()
        a[i] += h
        b[i] -= h
        g[i] = (f(a) - f(b)) / (float(a[i]) - float(b[i]))
    return g


def test_choice_by_hand():
    z = np.array([[1.0, 2.0, 2.0, -np.inf], [0.0, -0.0, np.nan, 1.0], [-np.inf] * 4], np.float32)
    assert mo.choose(z, 3).tolist() == [[1, 2, 0], [3, 0, 1], [-1, -1, -1]]
    assert mo.choose(z, 2, prices=np.array([0, 1.5, 0, 0], np.float32)).tolist() == [[2, 0], [3, 0], [-1, -1]]
    assert mo.choose(z, 1, valid=np.array([False, True, True])).tolist() == [[-1], [3], [-1]]


def test_plan_by_hand():
    counts, offsets, rows, pos = mo.plan(np.array([[2, 0], [0, -1], [2, 1]]), 3)
    assert counts.tolist() == [2, 1, 2] and offsets.tolist() == [0, 2, 3, 5]
    assert rows.tolist() == [0, 1, 2, 0, 2, -1] and pos.tolist() == [[3, 0], [1, -1], [4, 2]]


@pytest.mark.parametrize("gate", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [True, False])
def test_gate_gradient_against_differences(gate, renorm):
    z = logits(4, 6)
    idx = mo.choose(z, 3)
    idx[1, 2], idx[2] = -1, -1
    g = np.random.default_rng(1).normal(size=idx.shape)
    f = lambda v: (mo.gate_weight(v, idx, gate, renorm, 1.5) * g).sum()  # noqa: E731
    got = mo.gate_weight_grad(z, idx, gate, renorm, 1.5, g)
    assert np.abs(got - numeric(f, z)).max() < 1e-5
    assert not got[2].any()


@pytest.mark.parametrize("gate", ["softmax", "sigmoid"])
def test_balance_gradient_against_differences(gate):
    z = logits(9, 5, 2)
    idx = mo.choose(z, 2)
    idx[3], idx[5:7] = -1, -1
    seq = [0, 4, 4, 5, 7, 9]
    d = np.array([0.7, 0.3])
    f = lambda v: (mo.balance(v, idx, gate, seq)[0] * d).sum()  # noqa: E731
    assert np.abs(mo.balance_grad(z, idx, gate, d, seq) - numeric(f, z)).max() < 1e-5


def test_balance_of_even_use_is_one():
    z = np.zeros((8, 4), np.float32)
    loss, counts, share, tokens = mo.balance(z, np.arange(8)[:, None] % 4, "softmax")
    assert loss == pytest.approx([1.0, np.log(4.0) ** 2]) and (counts == 2).all() and tokens.tolist() == [8]


def test_price_step():
    assert mo.step_prices([0.0, 0.5, 0.0], [4, 0, 2], 0.1, 1.0) == pytest.approx([0.1, 0.4, 0.0])
    assert mo.step_prices([0.3], [0], 0.1, 1.0) == pytest.approx([0.3])


def test_e4m3_values():
    every = [(-1) ** s * (m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
             for s in (0, 1) for e in range(16) for m in range(8) if not (e == 15 and m == 7)]
    assert (mo.e4m3(every) == every).all() and max(every) == 448.0
    assert mo.e4m3([17.0, 19.0, 1000.0, 2.0 ** -10, 3 * 2.0 ** -10]).tolist() == [16.0, 20.0, 448.0, 0.0, 2.0 ** -8]


def test_blocks():
    x = np.zeros((2, 130), np.float32)
    x[0, :128], x[0, 128:], x[1, 3] = 448.0, [2.0, -1.0], np.inf
    codes, scales = mo.quantize_rows(x)
    assert scales[0].tolist() == [1.0, np.float32(2.0) / np.float32(448.0)]
    assert codes[0, 128:].tolist() == [448.0, -224.0]
    assert np.isnan(scales[1, 0]) and not codes[1].any()


def test_combine_gradient_against_differences():
    rng = np.random.default_rng(3)
    y, pos, w, d = rng.normal(size=(5, 3)), np.array([[4, 0], [-1, 2]]), rng.normal(size=(2, 2)), rng.normal(size=(2, 3))
    dy, dw = mo.combine_grad(d, y, pos, w)
    assert np.abs(dy - numeric(lambda v: (mo.combine(v, pos, w) * d).sum(), y)).max() < 1e-8
    assert np.abs(dw - numeric(lambda v: (mo.combine(y, pos, v) * d).sum(), w)).max() < 1e-8


def test_choice_reads_infinite_logits_as_they_are():
    big, inf = np.finfo(np.float32).max, np.inf
    z = np.array([[big, inf], [inf, inf], [0.0, inf]], np.float32)
    assert mo.choose(z, 1).tolist() == [[1], [0], [1]]
    assert mo.choose(z, 2, prices=np.array([1e38, inf], np.float32)).tolist() == [[0, -1], [0, -1], [0, -1]]
    assert mo.choose(z, 2, prices=np.array([1e38, 1e38], np.float32)).tolist() == [[1, 0], [0, 1], [1, 0]]
