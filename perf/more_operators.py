"""Timed cases of the expert layer's 16-bit training path: gated feed-forward blocks, and the gradients' norm and clipping.

A case is a dict of plain sizes and options. ``listed()`` holds the named cases, ``draw(rng)`` one more of the
same ranges. ``prepare`` makes the inputs on the GPU from the seed, ``run`` is one pass: the framework's calls
where ``own`` is true, else the same in elementary 32-bit torch operations. ``exact`` is the definition in 64 bits.

Kinds:
  block   gated feed-forward blocks, one for each expert (or a single dense one): a row x of expert e becomes
          y = O_e (act(G_e x) * (U_e x)), with G and U stacked as ``inner`` (E, 2 F, H) and O as ``outer`` (E, H, F). Rows are
          gathered from the tokens by expert; rows past the last expert's (padding tokens chose nothing) stay as
          they were. With ``train`` also the gradients of the rows and of both weights at dy.
  clip    many gradient tensors at once: g' = scale * g (the inverse of a loss scale), norm = the 2-norm of all g'
          together, and g' * min(1, max_norm / norm). Where the norm is not finite g' is returned unclipped, and the norm
          tells the program to skip its step.
"""

import math
import random

import torch

own = False

DEV = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def listed():
    return [
        # serving, one token through a dense block: the weights' bytes count
        dict(name="block_token", kind="block", T=1, E=1, k=1, H=4096, F=8192, dtype="bf16", act="silu", padded=False,
             train=False),
        # serving, 16 tokens in flight over 64 experts: a row or two for each
        dict(name="block_decode", kind="block", T=16, E=64, k=6, H=4096, F=2048, dtype="bf16", act="silu", padded=False,
             train=False),
        # a ragged training step of odd sizes, padding tokens among the rows
        dict(name="block_odd", kind="block", T=1001, E=5, k=2, H=2050, F=999, dtype="f16", act="gelu", padded=True,
             train=True),
        # one dense block over a long prompt
        dict(name="block_dense", kind="block", T=8192, E=1, k=1, H=4096, F=8192, dtype="bf16", act="gelu_tanh",
             padded=False, train=False),
        # a prompt's experts: 65536 gathered rows over 64 experts of uneven load
        dict(name="block_prefill", kind="block", T=8192, E=64, k=8, H=2048, F=1024, dtype="bf16", act="silu", padded=False,
             train=False),
        # a training step of 16 experts
        dict(name="block_train", kind="block", T=8192, E=16, k=2, H=4096, F=2048, dtype="bf16", act="silu", padded=False,
             train=True),
        # gradients of a router and of small blocks: only latency counts
        dict(name="clip_small", kind="clip", tensors=7, total=300_000, dtype="f32", mixed=False, packed=False,
             max_norm=1.0, scale=1.0, bad=False),
        # a packed buffer's slices of odd sizes, scaled losses
        dict(name="clip_odd", kind="clip", tensors=37, total=9_999_991, dtype="f16", mixed=True, packed=True,
             max_norm=1.0, scale=2.0 ** -10, bad=False),
        # one expert layer's gradients: 16-bit weights, a 32-bit router
        dict(name="clip_layer", kind="clip", tensors=5, total=402_900_000, dtype="bf16", mixed=True, packed=False,
             max_norm=1.0, scale=1.0, bad=False),
        # a whole model's
        dict(name="clip_model", kind="clip", tensors=60, total=2_000_000_000, dtype="bf16", mixed=True, packed=False,
             max_norm=1.0, scale=1.0, bad=False),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    if rng.random() < 0.3:
        tensors = _log(rng, 1, 60)
        total = _log(rng, max(tensors, 10), 2_000_000_000)
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        return dict(kind="clip", tensors=tensors, total=total // 2 if dtype == "f32" else total, dtype=dtype,
                    mixed=rng.random() < 0.5, packed=rng.random() < 0.4, max_norm=rng.choice([0.5, 1.0, 1e9]),
                    scale=2.0 ** -12 if dtype == "f16" else 1.0, bad=rng.random() < 0.1)
    E = rng.choice([1, 1, _log(rng, 2, 64), _log(rng, 2, 64)])
    k = 1 if E == 1 else rng.randint(1, min(8, E))
    train = rng.random() < 0.45
    T, H, F = _log(rng, 1, 8192), _log(rng, 32, 4096), _log(rng, 32, 8192)
    most = 18 * 16384 * 4096 * 2048 // (3 if train else 1)
    while 6 * T * k * H * F > most or E * H * F > 64 * 4096 * 2048 // (2 if train else 1):
        if T * k > 4096:
            T = (T + 1) // 2
        else:
            F = (F + 1) // 2
    return dict(kind="block", T=T, E=E, k=k, H=H, F=F, dtype=rng.choice(["bf16", "bf16", "f16"]),
                act=rng.choice(["silu", "silu", "gelu", "gelu_tanh", "relu"]), padded=E > 1 and rng.random() < 0.3, train=train)


# ---- inputs


def _plan(idx, E):
    """Rows sorted by expert, within an expert by token: (rows, offsets, counts); -1 past the last expert's."""
    T, k = idx.shape
    key = torch.where(idx < 0, torch.full_like(idx, E), idx).reshape(-1)
    skey, order = torch.sort(key, stable=True)
    rows = torch.where(skey < E, order // k, torch.full_like(order, -1)).int()
    counts = torch.zeros(E + 1, dtype=torch.int64, device=DEV).index_add_(0, key, torch.ones_like(key))[:E]
    offsets = torch.zeros(E + 1, dtype=torch.int32, device=DEV)
    offsets[1:] = torch.cumsum(counts, 0)
    return rows, offsets, counts


def _sizes(case):
    """Elements of the tensors: uneven, their sum the total."""
    n, total = case["tensors"], case["total"]
    r = random.Random(1000 * n + total % 997)
    w = [math.exp(r.uniform(0.0, 6.0)) for _ in range(n)]
    sizes = [max(1, int((total - n) * v / sum(w))) for v in w]
    sizes[-1] += max(0, total - sum(sizes))
    return sizes


def _tensors(case):
    """(type, elements) of every tensor; with ``mixed`` one in four is 32-bit and small."""
    sizes, dt = _sizes(case), DTYPES[case["dtype"]]
    if not case["mixed"]:
        return [(dt, n) for n in sizes]
    return [(torch.float32, max(1, n // 64)) if i % 4 == 1 else (dt, n) for i, n in enumerate(sizes)]


def _empty(spec, packed):
    """Tensors of these types and sizes: each its own, or consecutive slices of one buffer for each type."""
    if not packed:
        return [torch.empty(n, dtype=dt, device=DEV) for dt, n in spec]
    out, at = [], {}
    room = {dt: torch.empty(sum(n for d, n in spec if d is dt), dtype=dt, device=DEV) for dt in {d for d, _ in spec}}
    for dt, n in spec:
        a = at.get(dt, 0)
        out.append(room[dt][a:a + n])
        at[dt] = a + n
    return out


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    st = dict(case=case)
    if own:
        from paper_2608_07971_gb300 import moe
        st["moe"] = m = moe.Moe()
    if case["kind"] == "clip":
        spec = _tensors(case)
        st["grads"] = _empty(spec, case["packed"])
        for t in st["grads"]:
            # a tensor's own size of gradients, times the loss scale
            size = math.exp(-3.0 * float(torch.rand((), generator=g, device=DEV))) * 1e-2 / case["scale"]
            t.normal_(generator=g).mul_(size)
        if case["bad"]:
            st["grads"][-1][-1] = math.inf
        if own:
            st["out"] = _empty(spec, case["packed"])
            st["list"] = m.gradients(st["grads"], out=st["out"])
        return st
    T, E, k, H, F, dt = case["T"], case["E"], case["k"], case["H"], case["F"], DTYPES[case["dtype"]]
    M = T * k
    # activations with a few loud columns
    loud = 1.0 + 7.0 * (torch.rand(H, generator=g, device=DEV) < 0.01)
    st["x"] = (torch.randn(T, H, generator=g, device=DEV) * loud).to(dt)
    st["rows"], st["offsets"], st["sizes"] = None, None, [M]
    if E > 1:
        z = torch.randn(T, E, generator=g, device=DEV) + 0.7 * torch.randn(E, generator=g, device=DEV)
        idx = torch.sort(z, dim=-1, descending=True, stable=True)[1][:, :k]
        if case["padded"]:
            idx = torch.where(torch.rand(T, 1, generator=g, device=DEV) < 0.1, torch.full_like(idx, -1), idx)
        st["rows"], st["offsets"], counts = _plan(idx, E)
        st["sizes"] = counts.tolist()
    inner = torch.empty(E, 2 * F, H, dtype=dt, device=DEV)
    outer = torch.empty(E, H, F, dtype=dt, device=DEV)
    for e in range(E):
        inner[e] = torch.randn(2 * F, H, generator=g, device=DEV) * H ** -0.5
        outer[e] = torch.randn(H, F, generator=g, device=DEV) * F ** -0.5
    if case["train"]:
        # a program that trains in f16 scales its loss
        st["dy"] = (torch.randn(M, H, generator=g, device=DEV) * (0.25 if case["dtype"] == "f16" else 1e-3)).to(dt)
    if own:
        st["weight"] = m.gated_weight(inner, outer, case["act"])
        st["y"] = torch.zeros(M, H, dtype=dt, device=DEV)
        if case["train"]:
            st["kept"] = m.keep(M, st["weight"])
            st["grad"] = (torch.zeros(M, H, dtype=dt, device=DEV), torch.empty(E, 2 * F, H, dtype=dt, device=DEV),
                          torch.empty(E, H, F, dtype=dt, device=DEV))
    else:
        st["inner"], st["outer"] = inner, outer
    return st


# ---- plain forms


def _act(g, kind):
    """The activation and its derivative."""
    if kind == "silu":
        s = 1.0 / (1.0 + torch.exp(-g))
        return g * s, s * (1.0 + g * (1.0 - s))
    if kind == "gelu":
        c = 0.5 * (1.0 + torch.erf(g * math.sqrt(0.5)))
        return g * c, c + g * torch.exp(-0.5 * g * g) * (2.0 * math.pi) ** -0.5
    if kind == "gelu_tanh":
        a = math.sqrt(2.0 / math.pi)
        t = torch.tanh(a * (g + 0.044715 * g * g * g))
        return 0.5 * g * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * g * (1.0 - t * t) * a * (1.0 + 3.0 * 0.044715 * g * g)
    return torch.clamp(g, min=0.0), (g > 0.0).float()


def _expert(st, e, a, b):
    """Expert e's rows [a, b): (y, dx, dinner, douter), the gradients None without training."""
    c, dt = st["case"], st["x"].dtype
    F = c["F"]
    x = (st["x"] if st["rows"] is None else st["x"][st["rows"][a:b].long()]).float()
    w, o = st["inner"][e].float(), st["outer"][e].float()
    p = x @ w.t()
    g, u = p[:, :F], p[:, F:]
    act, slope = _act(g, c["act"])
    h = act * u
    y = (h @ o.t()).to(dt)
    if not c["train"]:
        return y, None, None, None
    d = st["dy"][a:b].float()
    dh = d @ o
    dp = torch.cat([dh * u * slope, dh * act], 1)
    return y, (dp @ w).to(dt), (dp.t() @ x).to(dt), (d.t() @ h).to(dt)


def _run_block(st):
    c, dt, sizes = st["case"], st["x"].dtype, st["sizes"]
    ends = [sum(sizes[:e + 1]) for e in range(len(sizes))]
    parts = [_expert(st, e, b - n, b) for e, (b, n) in enumerate(zip(ends, sizes))]
    left = torch.zeros(c["T"] * c["k"] - ends[-1], c["H"], dtype=dt, device=DEV)   # rows of no expert
    out = dict(y=torch.cat([p[0] for p in parts] + [left]))
    if c["train"]:
        out.update(dx=torch.cat([p[1] for p in parts] + [left]), dinner=torch.stack([p[2] for p in parts]),
                   douter=torch.stack([p[3] for p in parts]))
    return out


def _square(t):
    f = t.float()
    return torch.sum(f * f)


def _run_clip(st):
    c = st["case"]
    scaled = c["scale"] * torch.sqrt(torch.sum(torch.stack([_square(t) for t in st["grads"]]).double()))
    finite = torch.isfinite(scaled)
    less = torch.clamp(c["max_norm"] / torch.clamp(scaled, min=1e-300), max=1.0)
    factor = (c["scale"] * torch.where(finite, less, torch.ones_like(less))).float()
    return dict(norm=scaled.float(), grads=[(t.float() * factor).to(t.dtype) for t in st["grads"]])


def _run_own(st):
    c, m = st["case"], st["moe"]
    if c["kind"] == "clip":
        norm = m.clip(st["list"], c["max_norm"], scale=c["scale"])
        return dict(norm=norm, grads=st["out"])
    w, plan = st["weight"], dict(offsets=st["offsets"], rows=st["rows"])
    if not c["train"]:
        return dict(y=m.feed_forward(st["x"], w, out=st["y"], **plan))
    y = m.feed_forward(st["x"], w, out=st["y"], keep=st["kept"], **plan)
    dx, dinner, douter = m.feed_forward_backward(st["dy"], st["x"], w, st["kept"], out=st["grad"], **plan)
    return dict(y=y, dx=dx, dinner=dinner, douter=douter)


def run(state):
    if own:
        return _run_own(state)
    return _run_clip(state) if state["case"]["kind"] == "clip" else _run_block(state)


def work(case):
    c = case
    if c["kind"] == "clip":
        n = [(4 if dt is torch.float32 else 2, k) for dt, k in _tensors(c)]
        return dict(bytes=sum(2 * s * k for s, k in n) + 4, flops=sum(3 * k for _, k in n))
    T, E, k, H, F = c["T"], c["E"], c["k"], c["H"], c["F"]
    M = T * k * (0.9 if c["padded"] else 1.0)
    used = min(E, M)
    b = 2 * (T * H + M * H + used * 3 * F * H) + (4 * T * k + 4 * E if E > 1 else 0)
    if c["train"]:
        b += 2 * (2 * M * H + E * 3 * F * H)
    return dict(bytes=b, flops=(18 if c["train"] else 6) * M * H * F)


# ---- the definition in 64 bits


def _exact_act(g, kind):
    if kind == "silu":
        return torch.nn.functional.silu(g)
    if kind == "gelu":
        return torch.nn.functional.gelu(g)
    if kind == "gelu_tanh":
        return torch.nn.functional.gelu(g, approximate="tanh")
    return torch.relu(g)


def exact(case, seed):
    c = case
    if c["kind"] == "block" and work(c)["flops"] > 1e13:
        return None   # too long in 64 bits
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    if c["kind"] == "clip":
        wide = [t.double() * c["scale"] for t in st["grads"]]
        norm = sum(float(t.square().sum()) for t in wide) ** 0.5
        by = c["max_norm"] / norm if c["max_norm"] < norm < math.inf else 1.0
        return dict(norm=torch.tensor(norm, dtype=torch.float64), grads=[t.mul_(by) for t in wide])
    T, E, k, H, F = c["T"], c["E"], c["k"], c["H"], c["F"]
    y = torch.zeros(T * k, H, dtype=torch.float64, device=DEV)
    dx = torch.zeros_like(y)
    dinner, douter = [], []
    a = 0
    for e, n in enumerate(st["sizes"]):
        pick = slice(a, a + n) if st["rows"] is None else st["rows"][a:a + n].long()
        x, w, o = (t.double().requires_grad_(c["train"]) for t in (st["x"][pick], st["inner"][e], st["outer"][e]))
        out = torch.nn.functional.linear(
            _exact_act(torch.nn.functional.linear(x, w[:F]), c["act"]) * torch.nn.functional.linear(x, w[F:]), o)
        y[a:a + n] = out.detach()
        if c["train"]:
            dx[a:a + n], dw, do = torch.autograd.grad(out, (x, w, o), st["dy"][a:a + n].double())
            dinner.append(dw)
            douter.append(do)
        a += n
    if not c["train"]:
        return dict(y=y)
    return dict(y=y, dx=dx, dinner=torch.stack(dinner), douter=torch.stack(douter))
