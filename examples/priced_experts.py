"""A sparse layer of experts whose load is levelled by shadow prices: trained for some steps, then served.

Tokens take their experts as jobs take configurations in the solver: greatest value minus price, the demand summed,
the prices stepped by excess demand (Eq. price_update in capacity fractions). The layer is

    out = x + combine(W2 silu(W1 x_rows)),  rows and weights from the router's logits z = x Wr^T

with 8-bit products; gradients come from the library's calls, the elementwise parts from torch. Run it with
``python examples/priced_experts.py`` on a GB300 (random data: it learns to reproduce a fixed random map).
"""

from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2608_07971_gb300.moe import Gate, Moe  # noqa: E402


class PricedExperts:
    """Router, prices and two products per expert; fp32 master weights, bf16 rows."""

    def __init__(self, m: Moe, hidden: int, inner: int, experts: int, k: int, seed: int = 0):
        g = torch.Generator(device=m.device).manual_seed(seed)
        rand = lambda *s: torch.randn(*s, generator=g, device=m.device)  # noqa: E731
        self.m, self.k, self.gate = m, k, Gate("softmax", renorm=True)
        self.wr = rand(experts, hidden) * hidden ** -0.5
        # some experts start out popular: the first feature is a constant 1
        self.wr[:, 0] += torch.linspace(2.0, 0.0, experts, device=m.device)
        self.w1 = rand(experts, inner, hidden) * hidden ** -0.5
        self.w2 = rand(experts, hidden, inner) * inner ** -0.5
        self.prices = torch.zeros(experts, device=m.device)
        self.q1 = m.empty_weight(experts, inner, hidden, transposed=True)
        self.q2 = m.empty_weight(experts, hidden, inner, transposed=True)
        self.quantize()

    def quantize(self):
        self.m.quantize_weight(self.w1, out=self.q1)
        self.m.quantize_weight(self.w2, out=self.q2)

    def forward(self, x):
        m = self.m
        logits = x.float() @ self.wr.t()
        r = m.route(logits, self.k, gate=self.gate, prices=self.prices)
        h = m.linear(x, self.q1, offsets=r.offsets, rows=r.rows)
        s = torch.nn.functional.silu(h.float()).to(x.dtype)
        y = m.linear(s, self.q2, offsets=r.offsets)
        return x + m.combine(y, r.pos, r.weight), (logits, r, h, s, y)

    def train_step(self, x, target, lr: float = 0.05, balance: float = 0.01, eta: float = 0.1):
        """One step on mean (out - target)^2 plus the balance loss; returns (loss, balance loss, heaviest load /
        mean load)."""
        m, T = self.m, x.shape[0]
        out, (logits, r, h, s, y) = self.forward(x)
        diff = (out - target).float()
        loss = (diff * diff).mean()
        b = m.balance(logits, r.idx, gate=self.gate)

        dout = (2.0 / diff.numel() * diff).to(x.dtype)
        dy, dweight = m.combine_backward(dout, y, r.pos, r.weight)
        ds, dw2 = m.linear_backward(dy, s, self.q2, offsets=r.offsets)
        hf = h.float()
        sig = torch.sigmoid(hf)
        dh = (ds.float() * sig * (1.0 + hf * (1.0 - sig))).to(x.dtype)
        _, dw1 = m.linear_backward(dh, x, self.q1, offsets=r.offsets, rows=r.rows, need=(False, True))
        dl = torch.tensor([balance, 0.0], device=m.device)
        dlogits = m.route_backward(logits, r.idx, gate=self.gate, dweight=dweight, balance=b, dloss=dl)
        dwr = dlogits.t() @ x.float()

        step = lr * x.numel() ** 0.5
        for w, d in ((self.wr, dwr), (self.w1, dw1), (self.w2, dw2)):
            w.sub_(step * d)
        self.quantize()
        m.step_prices(self.prices, r.counts, eta)
        heavy = r.counts.max().float() * r.counts.numel() / (T * self.k)
        return loss, b.loss[0], heavy


class Server:
    """The trained layer for a fixed number of tokens in flight, captured in a CUDA graph."""

    def __init__(self, layer: PricedExperts, tokens: int):
        m, self.layer = layer.m, layer
        E, hidden, k = layer.wr.shape[0], layer.wr.shape[1], layer.k
        self.x = torch.zeros(tokens, hidden, dtype=torch.bfloat16, device=m.device)
        self.r = m.routing(tokens, E, k)
        self.h = torch.empty(tokens * k, layer.q1.N, dtype=torch.bfloat16, device=m.device)
        self.y = torch.empty(tokens * k, hidden, dtype=torch.bfloat16, device=m.device)
        self.out = torch.empty_like(self.x)
        stream = torch.cuda.Stream(m.device)
        stream.wait_stream(torch.cuda.current_stream(m.device))
        with torch.cuda.stream(stream):
            self._step()   # work space is there before the capture
        torch.cuda.current_stream(m.device).wait_stream(stream)
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph, stream=stream):
            self._step()

    def _step(self):
        m, la = self.layer.m, self.layer
        m.route(self.x.float() @ la.wr.t(), la.k, gate=la.gate, prices=la.prices, out=self.r)
        m.linear(self.x, la.q1, offsets=self.r.offsets, rows=self.r.rows, out=self.h)
        s = torch.nn.functional.silu(self.h.float()).to(self.h.dtype)
        m.linear(s, la.q2, offsets=self.r.offsets, out=self.y)
        m.combine(self.y, self.r.pos, self.r.weight, out=self.out)

    def __call__(self, x):
        self.x.copy_(x)
        self.graph.replay()
        return x + self.out


def tokens(n: int, hidden: int, device):
    """Random rows whose first feature is 1."""
    x = torch.randn(n, hidden, device=device)
    x[:, 0] = 1.0
    return x.bfloat16()


def main():
    m = Moe()
    torch.manual_seed(0)
    hidden, experts = 256, 16
    layer = PricedExperts(m, hidden, 512, experts, k=2)
    mix = torch.randn(hidden, hidden, device=m.device) * hidden ** -0.5
    for i in range(60):
        x = tokens(2048, hidden, m.device)
        loss, bal, heavy = layer.train_step(x, x + torch.tanh(x.float() @ mix).bfloat16())
        if i % 10 == 0 or i == 59:
            print(f"step {i:3d}  loss {loss.item():.4f}  balance {bal.item():.3f}  heaviest expert {heavy.item():.2f} x mean")
    server = Server(layer, 1)
    x = tokens(1, hidden, m.device)
    a, b = server(x), layer.forward(x)[0]
    print("served token equals the layer's:", bool(torch.equal(a, b)))
    m.synchronize()
    m.close()


if __name__ == "__main__":
    main()
