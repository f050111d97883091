"""Copies and pickles of the expert layer's gates, weights and results (CPU: no kernel runs)."""

import copy
import dataclasses
import pickle

import pytest

torch = pytest.importorskip("torch")

from paper_2608_07971_gb300 import moe  # noqa: E402

WAYS = [copy.copy, copy.deepcopy, lambda v: pickle.loads(pickle.dumps(v))]


def weight():
    return moe.Weight(2, 10, 20, torch.arange(2 * 10 * 32).view(2, 10, 32).to(torch.uint8), torch.rand(2, 1, 1),
                      torch.ones(2, 20, 16, dtype=torch.uint8))


@pytest.mark.parametrize("way", WAYS)
def test_gate(way):
    for g in (moe.Gate(), moe.Gate("sigmoid", False, 2.5)):
        c = way(g)
        assert c == g and (c._c.kind, c._c.renorm, c._c.scale) == (g._c.kind, g._c.renorm, g._c.scale)
    assert dataclasses.replace(moe.Gate(), scale=3.0)._c.scale == 3.0


@pytest.mark.parametrize("way", WAYS)
def test_weight(way):
    w = weight()
    c = way(w)
    assert torch.equal(c.q, w.q) and torch.equal(c.scale, w.scale) and torch.equal(c.qt, w.qt)
    c._arg()
    assert (c._c.q, c._c.qt, c._c.scale) == (c.q.data_ptr(), c.qt.data_ptr(), c.scale.data_ptr())
    assert (c._c.E, c._c.N, c._c.K, c._c.ld, c._c.ldt) == (2, 10, 20, 32, 16)
    assert (c.q.data_ptr() == w.q.data_ptr()) == (way is copy.copy)


@pytest.mark.parametrize("way", WAYS)
def test_results_are_checked_anew(way):
    """A result that was loaded, to another device perhaps, is not taken as one that the handle made."""
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    r = moe.Routing(i32(4, 2), torch.zeros(4, 2), torch.zeros(8, dtype=torch.int64), i32(8), i32(4, 2), i32(9))
    b = moe.Balance(torch.zeros(2), torch.zeros(1, 8, dtype=torch.int64), torch.zeros(1, 8), i32(1).long())
    object.__setattr__(r, "checked", (0, 4, 8, 2))
    object.__setattr__(b, "checked", (0, 1, 8))
    for v in (r, b):
        c = way(v)
        assert c.checked is None and v.checked is not None
        for f in dataclasses.fields(v):
            if f.init:
                assert torch.equal(getattr(c, f.name), getattr(v, f.name))
