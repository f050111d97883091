"""Gated experts trained with the library's calls (examples/priced_experts.py: GatedExperts): a step's gradients agree with
autograd, and a step runs."""

import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ex():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2608_07971_gb300 import build
    build.build()
    spec = importlib.util.spec_from_file_location("priced_experts", os.path.join(ROOT, "examples", "priced_experts.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def test_gradients_of_a_step(ex):
    m = ex.Moe()
    layer = ex.GatedExperts(m, 96, 80, 6, k=2, seed=3)
    x = ex.tokens(150, 96, "cuda")
    dout = torch.randn(150, 96, device="cuda").bfloat16()
    _, (logits, r, kept, y) = layer.forward(x, keep=True)
    got = layer.gradients(x, dout, logits, r, kept, y)

    v = [t.double().requires_grad_() for t in (layer.wr, layer.blocks.inner, layer.blocks.outer)]
    xd = x.double()
    p = torch.softmax(torch.gather(xd @ v[0].t(), 1, r.idx.long()), -1)
    total = 0.0
    for e in range(6):
        t, j = torch.nonzero(r.idx == e, as_tuple=True)
        q = xd[t] @ v[1][e].t()
        ye = (torch.nn.functional.silu(q[:, :80]) * q[:, 80:]) @ v[2][e].t()
        total = total + torch.zeros_like(xd).index_add(0, t, ye * p[t, j][:, None])
    total.backward(dout.double())
    # at most 8 roundings to bf16 (2^-8) of what the sums are made of, which have terms of either sign: 2 percent
    for a, b in zip(got, v):
        assert a.dtype is torch.float32 and float((a.double() - b.grad).norm() / b.grad.norm()) < 0.02
    m.synchronize()
    m.close()


def test_steps_run(ex):
    m = ex.Moe()
    torch.manual_seed(0)
    layer = ex.GatedExperts(m, 128, 192, 8, k=2)
    for _ in range(3):
        x = ex.tokens(512, 128, "cuda")
        loss, norm, heavy = layer.train_step(x, x + torch.tanh(x))
        assert torch.isfinite(loss) and torch.isfinite(norm) and norm > 0 and heavy >= 1.0
    assert torch.equal(layer.blocks.inner, layer.inner.bfloat16()) and torch.equal(layer.blocks.outer, layer.outer.bfloat16())
    m.synchronize()
    m.close()
