"""Results and weights that a program hands back to the expert layer's calls: what was changed is checked and used."""

import dataclasses

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def moe():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2608_07971_gb300 import build, moe
    build.build()
    return moe


@pytest.fixture(scope="module")
def m(moe):
    h = moe.Moe()
    yield h
    h.synchronize()
    h.close()


def i32(*shape):
    return torch.zeros(shape, dtype=torch.int32, device="cuda")


def test_replaced_results_are_checked(moe, m):
    z = torch.randn(40, 8, device="cuda")
    r, b = m.routing(40, 8, 2), m.balancing(1, 8)
    m.route(z, 2, out=r)
    # larger than needed, so that nothing is written out of bounds where the check is missing
    for change in (dict(idx=i32(50, 2)), dict(rows=i32(100)), dict(pos=i32(40, 3)), dict(offsets=i32(10)),
                   dict(counts=torch.zeros(9, dtype=torch.int64, device="cuda")),
                   dict(weight=torch.zeros(40, 2, dtype=torch.float64, device="cuda")), dict(rows=i32(80).long())):
        with pytest.raises(ValueError):
            m.route(z, 2, out=dataclasses.replace(r, **change))
    for change in (dict(loss=torch.zeros(3, device="cuda")), dict(share=torch.zeros(2, 8, device="cuda")),
                   dict(tokens=torch.zeros(2, dtype=torch.int64, device="cuda"))):
        with pytest.raises(ValueError):
            m.balance(z, r.idx, out=dataclasses.replace(b, **change))
    m.balance(z, r.idx, out=b)
    with pytest.raises(ValueError):
        m.route_backward(z, r.idx, balance=dataclasses.replace(b, counts=torch.zeros(1, 9, dtype=torch.int64, device="cuda")),
                         dloss=torch.ones(2, device="cuda"))
    # good replacements are taken
    spare = dataclasses.replace(r, rows=i32(80))
    assert m.route(z, 2, out=spare) is spare and torch.equal(spare.rows, r.rows)


def test_parts_of_a_plan_are_refused(moe, m):
    """A plan is whole or left out, also where there are no tokens and nothing but offsets would be written."""
    z, r = torch.randn(0, 8, device="cuda"), m.routing(0, 8, 2)
    for change in (dict(rows=None, offsets=i32(20)), dict(rows=None, pos=None, offsets=i32(20)), dict(pos=None)):
        with pytest.raises(ValueError):
            m.route(z, 2, out=dataclasses.replace(r, **change))
    assert m.route(z, 2, out=dataclasses.replace(r, rows=None, pos=None, offsets=None)).rows is None


def test_changed_weights_are_used(moe, m):
    """Tensors assigned to a weight's fields, or moved under them, are what the next call reads or writes."""
    g = torch.Generator(device="cuda").manual_seed(0)
    w = [torch.randn(2, 48, 160, generator=g, device="cuda") for _ in range(3)]
    x, dy = torch.randn(7, 160, generator=g, device="cuda"), torch.randn(7, 48, generator=g, device="cuda")
    off = torch.tensor([0, 3, 7], device="cuda").int()
    a, b, c = (m.quantize_weight(v, transposed=True) for v in w)
    kept = (a.q, a.scale, a.qt)   # the memory before stays there
    a.q, a.scale, a.qt = b.q, b.scale, b.qt
    assert torch.equal(m.linear(x, a, offsets=off), m.linear(x, b, offsets=off))
    assert torch.equal(m.linear_backward(dy, x, a, offsets=off)[0], m.linear_backward(dy, x, b, offsets=off)[0])
    a.q.data = c.q.clone()
    a.scale.data = c.scale.clone()
    assert torch.equal(m.linear(x, a, offsets=off), m.linear(x, c, offsets=off))
    a.q, a.scale, a.qt = kept
    m.quantize_weight(w[2], transposed=True, out=a)
    assert torch.equal(kept[0], c.q) and torch.equal(kept[2], c.qt) and torch.equal(kept[1], c.scale)
    a.qt = None
    with pytest.raises(ValueError):
        m.linear_backward(dy, x, a, offsets=off)
    a.q = torch.zeros(2, 40, 160, dtype=torch.uint8, device="cuda")
    with pytest.raises(ValueError):
        m.linear(x, a, offsets=off)
