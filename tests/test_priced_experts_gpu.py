"""The expert layer's calls together, as examples/priced_experts.py runs them: the loss falls, prices level the
load, a step's gradients agree with autograd on the same rounded values, a served token equals the layer's."""

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


def test_training_and_serving(ex):
    m = ex.Moe()
    torch.manual_seed(0)
    layer = ex.PricedExperts(m, 256, 512, 16, k=2)
    mix = torch.randn(256, 256, device="cuda") / 16
    losses, loads = [], []
    for _ in range(60):
        x = ex.tokens(1024, 256, "cuda")
        loss, _, heavy = layer.train_step(x, x + torch.tanh(x.float() @ mix).bfloat16())
        losses.append(loss.item())
        loads.append(heavy.item())
    assert losses[-1] < 0.6 * losses[0]
    assert loads[0] > 1.8 and max(loads[-5:]) < 0.8 * loads[0]
    for tokens in (1, 5):
        serve = ex.Server(layer, tokens)
        for _ in range(3):
            x = torch.randn(tokens, 256, device="cuda").bfloat16()
            assert torch.equal(serve(x), layer.forward(x)[0])
    m.synchronize()
    m.close()


def test_step_against_autograd(ex):
    """Products on values that 8 bits hold exactly (so rounding changes nothing): the layer's output and the
    router's and experts' gradients against autograd in fp64."""
    m = ex.Moe()
    T, H, F, E, k = 96, 128, 128, 4, 2
    g = torch.Generator(device="cuda").manual_seed(3)
    pick = lambda *s: torch.randint(-2, 3, s, generator=g, device="cuda").float()  # noqa: E731
    x, w1, dy = pick(T, H), pick(E, F, H) / 8, pick(T * k, F) / 4
    x[:, 0], w1[:, 0, 0] = 2.0, 0.25          # the largest magnitude of every block: scales are powers of two / 448 * 448
    logits = torch.randn(T, E, generator=g, device="cuda")
    r = m.route(logits, k)
    q = m.quantize_weight(w1, transposed=True)
    h = m.linear(x, q, offsets=r.offsets, rows=r.rows)
    out = m.combine(h, r.pos, r.weight)
    dout = torch.randn(T, F, generator=g, device="cuda")
    dh, dweight = m.combine_backward(dout, h, r.pos, r.weight)
    dlogits = m.route_backward(logits, r.idx, dweight=dweight)

    z = logits.double().requires_grad_(True)
    xd, wd = x.double().requires_grad_(True), w1.double().requires_grad_(True)
    idx = r.idx.long()
    weight = torch.softmax(torch.gather(z, 1, idx), -1)
    rows = torch.einsum("th,tkfh->tkf", xd, wd[idx])
    (torch.einsum("tk,tkf->tf", weight, rows) * dout.double()).sum().backward()
    # fp32 sums of 128 terms of size up to 4 and of 2 rows of size up to 40
    assert (out.double() - torch.einsum("tk,tkf->tf", weight, rows)).abs().max() < 1e-4
    assert (dlogits.double() - z.grad).abs().max() < 1e-3
    # the products' gradients round the rows' gradients to 8 bits: a relative 2^-4 of each term at most
    dx, dw = m.linear_backward(dh, x, q, offsets=r.offsets, rows=r.rows)
    slots = m.combine(dx, r.pos)
    bound = torch.einsum("tk,tf,tkfh->th", weight, dout.double().abs(), wd[idx].abs()) / 16
    assert bool(((slots.double() - xd.grad).abs() <= bound + 1e-3).all())
    onehot = torch.nn.functional.one_hot(idx, E).double() * weight[:, :, None]
    bound = torch.einsum("tke,tf,th->efh", onehot, dout.double().abs(), xd.abs()) / 16
    # a block of 128 rows keeps a relative 2^-4 of its terms or an absolute 2^-10 of its largest one
    small = dout.abs().max().double() * 2.0 * T * k * 2.0 ** -10
    assert bool(((dw.double() - wd.grad).abs() <= bound + small).all())
    m.close()
