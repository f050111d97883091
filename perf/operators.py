"""Timed cases of the price-routed expert layer: what a program with a sparse layer of experts asks of it.

A case is a dict of plain sizes and options. ``listed()`` holds the named cases, ``draw(rng)`` one more of the
same ranges. ``prepare`` makes the inputs on the GPU from the seed, ``run`` is one pass: the framework's calls
where ``own`` is true, else the same in elementary 32-bit torch operations. ``exact`` is the definition in 64 bits.

Kinds:
  route     every token takes the k experts of greatest logit minus price (ties to the lowest index), its gate
            weights, the experts' counts and the plan that sorts the rows by expert; with ``train`` also the
            gradient of the logits
  balance   the balance and logit losses of a routing, per-expert counts and shares for each sequence, and the
            gradient of both losses
  combine   the experts' output rows, weighted and summed back into their tokens; with ``train`` both gradients
  product   rows of 16-bit activations, gathered by expert, times 8-bit weights with a scale for each block of
            128 x 128, the activations rounded to 8 bits with a scale for each 128 of a row; with ``train`` the
            weights' rounding and both gradients too

An 8-bit block holds a = max(max |x|, 2^-100), the scale a / 448 and the codes e4m3(x * (448 / a)), each step one
32-bit rounding; a block with a value that is not finite has the scale NaN.
"""

import math

import torch

own = False

DEV = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BLOCK = 128


def listed():
    return [
        # serving, one token: the router of one layer between two products; only latency counts
        dict(name="route_token", kind="route", T=1, E=64, k=6, dtype="f32", gate="softmax", renorm=True,
             prices=True, masked=False, train=False),
        # a ragged batch in flight: padding rows, closed experts, an odd number of experts, sigmoid gate
        dict(name="route_odd", kind="route", T=1537, E=134, k=5, dtype="f16", gate="sigmoid", renorm=True,
             prices=True, masked=True, train=False),
        # a training step's router: many tokens, forward and gradient
        dict(name="route_train", kind="route", T=16384, E=256, k=8, dtype="bf16", gate="softmax", renorm=False,
             prices=True, masked=False, train=True),
        # losses of a small odd batch, one sequence, sigmoid gate, 32-bit logits
        dict(name="balance_odd", kind="balance", T=1021, E=61, k=3, B=1, dtype="f32", gate="sigmoid",
             masked=True),
        # losses of a training step, balanced within each of 16 sequences of uneven length
        dict(name="balance_train", kind="balance", T=16384, E=256, k=8, B=16, dtype="bf16", gate="softmax",
             masked=False),
        # serving, one token: its experts' rows summed
        dict(name="combine_token", kind="combine", T=1, E=64, k=6, H=2048, dtype="bf16", train=False),
        # a training step: the layer's output and both gradients
        dict(name="combine_train", kind="combine", T=8192, E=64, k=8, H=4096, dtype="bf16", train=True),
        # serving: 16 tokens in flight, few rows for each expert, so the weights' bytes count
        dict(name="product_decode", kind="product", T=16, E=64, k=6, N=2048, K=4096, dtype="bf16", train=False),
        # one dense layer of odd sizes
        dict(name="product_odd", kind="product", T=1001, E=1, k=1, N=1999, K=2050, dtype="f16", train=False),
        # one large dense layer
        dict(name="product_dense", kind="product", T=8192, E=1, k=1, N=8192, K=4096, dtype="bf16", train=False),
        # a prompt's experts: 65536 gathered rows over 64 experts of uneven load
        dict(name="product_prefill", kind="product", T=8192, E=64, k=8, N=4096, K=2048, dtype="bf16", train=False),
        # a training step of 16 experts: weights rounded, the product, the gradients of rows and weights
        dict(name="product_train", kind="product", T=8192, E=16, k=2, N=2048, K=4096, dtype="bf16", train=True),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    kind = rng.choice(["route", "balance", "combine", "product", "product"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if kind == "route":
        E = _log(rng, 4, 256)
        return dict(kind=kind, T=_log(rng, 1, 16384), E=E, k=rng.randint(1, min(8, E)), dtype=dtype,
                    gate=rng.choice(["softmax", "sigmoid"]), renorm=rng.random() < 0.6,
                    prices=rng.random() < 0.6, masked=rng.random() < 0.4, train=rng.random() < 0.5)
    if kind == "balance":
        E = _log(rng, 4, 256)
        T = _log(rng, 16, 16384)
        return dict(kind=kind, T=T, E=E, k=rng.randint(1, min(8, E)), B=_log(rng, 1, min(16, T)), dtype=dtype,
                    gate=rng.choice(["softmax", "sigmoid"]), masked=rng.random() < 0.4)
    if kind == "combine":
        E = _log(rng, 8, 64)
        return dict(kind=kind, T=_log(rng, 1, 8192), E=E, k=rng.randint(1, 8), H=_log(rng, 64, 4096), dtype=dtype,
                    train=rng.random() < 0.5)
    E = rng.choice([1, _log(rng, 2, 64)])
    k = 1 if E == 1 else rng.randint(1, min(8, E))
    train = rng.random() < 0.35
    T, N, K = _log(rng, 1, 8192), _log(rng, 64, 8192), _log(rng, 64, 4096)
    cap = 2 * 65536 * 4096 * 2048 // (3 if train else 1)
    while 2 * T * k * N * K > cap or E * N * K > 64 * 4096 * 2048 // (2 if train else 1):
        if T * k > 4096:
            T = (T + 1) // 2
        else:
            N = (N + 1) // 2
    return dict(kind=kind, T=T, E=E, k=k, N=N, K=K, dtype=dtype, train=train)


# ---- inputs


def _logits(case, g):
    """Logits of T tokens: an expert's popularity, a token's taste."""
    T, E = case["T"], case["E"]
    z = torch.randn(T, E, generator=g, device=DEV) + 0.7 * torch.randn(E, generator=g, device=DEV)
    return z


def _choose(score, k):
    """The k greatest, descending, ties to the lowest index."""
    return torch.sort(score, dim=-1, descending=True, stable=True)[1][:, :k]


def _plan(idx, E):
    """Rows sorted by expert in the order of their slots: (rows, pos, offsets, counts)."""
    T, k = idx.shape
    flat = idx.reshape(-1).long()
    key = torch.where(flat < 0, torch.full_like(flat, E), flat)
    skey, order = torch.sort(key, stable=True)
    ok = skey < E
    rows = torch.where(ok, order // k, torch.full_like(order, -1)).int()
    pos = torch.empty_like(flat)
    pos[order] = torch.where(ok, torch.arange(T * k, device=idx.device), torch.full_like(order, -1))
    counts = torch.sum(key[:, None] == torch.arange(E, device=idx.device), dim=0) if T * k * E <= 1 << 26 else \
        torch.zeros(E + 1, dtype=torch.int64, device=idx.device).index_add_(0, key, torch.ones_like(key))[:E]
    offsets = torch.zeros(E + 1, dtype=torch.int32, device=idx.device)
    offsets[1:] = torch.cumsum(counts, 0)
    return rows, pos.reshape(T, k).int(), offsets, counts


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    kind, T, E, k, dt = case["kind"], case["T"], case["E"], case["k"], DTYPES[case["dtype"]]
    st = dict(case=case)
    if own:
        from paper_2608_07971_gb300 import moe
        st["moe"] = moe.Moe()
    if kind == "route":
        z = _logits(case, g).to(dt)
        st["valid"] = None
        if case["masked"]:
            # closed experts by -inf and by the type's lowest value, a row with every expert closed, padding rows
            closed = torch.rand(T, E, generator=g, device=DEV) < 0.05
            z = torch.where(closed, torch.full_like(z, -math.inf), z)
            z = torch.where(torch.rand(T, E, generator=g, device=DEV) < 0.01, torch.full_like(z, torch.finfo(dt).min), z)
            z = torch.where(torch.rand(T, 1, generator=g, device=DEV) < 0.01, torch.full_like(z, -math.inf), z)
            st["valid"] = torch.rand(T, generator=g, device=DEV) >= 0.1
        st["logits"] = z
        st["prices"] = None
        if case["prices"]:
            st["prices"] = torch.clamp(0.5 * torch.randn(E, generator=g, device=DEV), min=0.0)
        st["dweight"] = torch.randn(T, k, generator=g, device=DEV)
        if own:
            gate = moe.Gate(case["gate"], renorm=case["renorm"], scale=2.5)
            st["gate"], st["out"] = gate, st["moe"].routing(T, E, k)
            st["dlogits"] = torch.empty_like(z)
    elif kind == "balance":
        z = _logits(case, g).to(dt)
        score = z.float() - 0.3 * torch.rand(E, generator=g, device=DEV)
        if case["masked"]:
            # experts closed to some tokens; a row keeps those that it took
            closed = torch.rand(T, E, generator=g, device=DEV) < 0.1
            closed.scatter_(1, _choose(score, k), False)
            z = torch.where(closed, torch.full_like(z, -math.inf), z)
        idx = _choose(score, k)
        # rows that chose nothing: padding
        idx = torch.where(torch.rand(T, 1, generator=g, device=DEV) < 0.05, torch.full_like(idx, -1), idx).int()
        st["logits"], st["idx"] = z, idx
        B = case["B"]
        cut = torch.sort(torch.randperm(T - 1, generator=g, device=DEV)[:B - 1] + 1)[0] if T > 1 else \
            torch.zeros(0, dtype=torch.int64, device=DEV)
        st["seq"] = torch.cat([torch.zeros(1, dtype=torch.int64, device=DEV), cut,
                               torch.full((1,), T, dtype=torch.int64, device=DEV)]).int()
        # gradients of the weighted losses; a program that trains in f16 scales its loss
        st["dloss"] = torch.tensor([0.01, 0.001], device=DEV) * (65536.0 if case["dtype"] == "f16" else 1.0)
        if own:
            st["gate"] = moe.Gate(case["gate"])
            st["out"], st["dlogits"] = st["moe"].balancing(B, E), torch.empty_like(z)
    elif kind == "combine":
        H = case["H"]
        idx = _choose(_logits(case, g), k).int()
        _, st["pos"], _, _ = _plan(idx, E)
        w = torch.rand(T, k, generator=g, device=DEV) + 0.05
        st["weight"] = w / w.sum(-1, keepdim=True)
        st["y"] = torch.randn(T * k, H, generator=g, device=DEV).to(dt)
        st["dout"] = torch.randn(T, H, generator=g, device=DEV).to(dt) if case["train"] else None
        if own:
            st["out"] = torch.empty(T, H, dtype=dt, device=DEV)
            if case["train"]:
                st["dy"], st["dw"] = torch.empty_like(st["y"]), torch.empty_like(st["weight"])
    else:
        N, K, M = case["N"], case["K"], T * k
        # activations with a few loud columns
        loud = 1.0 + 15.0 * (torch.rand(K, generator=g, device=DEV) < 0.01)
        st["x"] = (torch.randn(T, K, generator=g, device=DEV) * loud).to(dt)
        st["rows"], st["offsets"], st["sizes"] = None, None, [M]
        if E > 1:
            rows, _, offsets, counts = _plan(_choose(_logits(case, g), k).int(), E)
            st["rows"], st["offsets"], st["sizes"] = rows, offsets, counts.tolist()
        w = torch.empty(E, N, K, dtype=dt, device=DEV)
        for e in range(E):
            w[e] = torch.randn(N, K, generator=g, device=DEV) * (K ** -0.5)
        if case["train"]:
            st["w"] = w
            st["dy"] = (torch.randn(M, N, generator=g, device=DEV) * 1e-3).to(dt)
        else:
            # a served model's weights: codes and scales
            codes = torch.empty(E, N, K, dtype=torch.float8_e4m3fn, device=DEV)
            scale = torch.empty(E, -(-N // BLOCK), -(-K // BLOCK), device=DEV)
            for e in range(E):
                codes[e], scale[e] = _quantize_weight(w[e].float())
            st["codes"], st["scale"] = codes, scale
        if own:
            m = st["moe"]
            st["y"] = torch.empty(M, N, dtype=dt, device=DEV)
            if case["train"]:
                st["weight"] = m.empty_weight(E, N, K, transposed=True)
                st["dx"] = torch.empty(M, K, dtype=dt, device=DEV)
                st["dw"] = torch.empty(E, N, K, device=DEV)
            else:
                st["weight"] = m.load_weight(st.pop("codes"), st.pop("scale"))
    return st


# ---- plain forms


def _amax_scale(amax):
    a = torch.clamp(amax, min=2.0 ** -100)
    bad = ~torch.isfinite(amax)
    scale = torch.where(bad, torch.full_like(a, math.nan), a / 448.0)
    inv = torch.where(bad, torch.zeros_like(a), torch.full_like(a, 448.0) / a)
    return scale, inv


def _codes(x, inv):
    return torch.clamp(x * inv, -448.0, 448.0).to(torch.float8_e4m3fn)


def _quantize_weight(w):
    """Codes and the scale of every 128 x 128 block of a 32-bit matrix."""
    N, K = w.shape
    p = torch.nn.functional.pad(w, (0, -K % BLOCK, 0, -N % BLOCK))
    p = p.reshape(p.shape[0] // BLOCK, BLOCK, p.shape[1] // BLOCK, BLOCK)
    scale, inv = _amax_scale(p.abs().amax(dim=(1, 3)))
    q = _codes(p, inv[:, None, :, None]).reshape(p.shape[0] * BLOCK, p.shape[2] * BLOCK)
    return q[:N, :K], scale


def _spread(scale, N, K):
    return scale.repeat_interleave(BLOCK, 0)[:N].repeat_interleave(BLOCK, 1)[:, :K]


def _round_rows(x):
    """x rounded to 8 bits with a scale for each 128 of a row, as 32-bit values."""
    M, K = x.shape
    p = torch.nn.functional.pad(x, (0, -K % BLOCK)).reshape(M, -1, BLOCK)
    scale, inv = _amax_scale(p.abs().amax(-1, keepdim=True))
    return (_codes(p, inv).float() * scale).reshape(M, -1)[:, :K]


def _run_route(st):
    c, z = st["case"], st["logits"].float()
    T, E, k = c["T"], c["E"], c["k"]
    profit = z if st["prices"] is None else z - st["prices"]
    if st["valid"] is not None:
        profit = torch.where(st["valid"][:, None], profit, torch.full_like(profit, -math.inf))
    idx = _choose(profit, k)
    took = torch.gather(profit, 1, idx) > -math.inf
    zs = torch.gather(z, 1, idx)
    ninf = torch.full_like(zs, -math.inf)
    live = took[:, :1]
    a = z if c["gate"] == "softmax" else torch.nn.functional.logsigmoid(z)
    if c["renorm"]:
        ac = torch.where(took, torch.gather(a, 1, idx), ninf)
        e = torch.exp(ac - torch.where(live, ac.amax(-1, keepdim=True), torch.zeros_like(ac[:, :1])))
        p = e / torch.where(live, e.sum(-1, keepdim=True), torch.ones_like(e[:, :1]))
    elif c["gate"] == "softmax":
        m = torch.where(live, z.amax(-1, keepdim=True), torch.zeros_like(z[:, :1]))
        ez = torch.exp(z - m)
        s = ez / torch.where(live, ez.sum(-1, keepdim=True), torch.ones_like(m))
        p = torch.where(took, torch.gather(s, 1, idx), torch.zeros_like(zs))
    else:
        p = torch.where(took, 1.0 / (1.0 + torch.exp(-zs)), torch.zeros_like(zs))
    weight = 2.5 * p
    out_idx = torch.where(took, idx, torch.full_like(idx, -1)).int()
    rows, pos, offsets, counts = _plan(out_idx, E)
    out = dict(idx=out_idx, weight=weight, counts=counts, rows=rows, pos=pos, offsets=offsets)
    if c["train"]:
        gw = torch.where(took, 2.5 * st["dweight"], torch.zeros_like(zs))
        if c["renorm"]:
            d = p * (gw - torch.sum(gw * p, -1, keepdim=True))
            if c["gate"] == "sigmoid":
                d = d / (1.0 + torch.exp(zs))
            d = torch.where(took, d, torch.zeros_like(d))
            dz = torch.zeros_like(z).scatter_(1, idx, d)
        elif c["gate"] == "softmax":
            gz = torch.zeros_like(z).scatter_(1, idx, gw)
            dz = torch.where(live, s * (gz - torch.sum(gw * p, -1, keepdim=True)), torch.zeros_like(z))
        else:
            d = torch.where(took, gw * p * (1.0 - p), torch.zeros_like(p))
            dz = torch.zeros_like(z).scatter_(1, idx, d)
        out["dlogits"] = dz.to(st["logits"].dtype)
    return out


def _run_balance(st):
    c, z, idx = st["case"], st["logits"].float(), st["idx"]
    T, E, k, B = c["T"], c["E"], c["k"], c["B"]
    live = idx[:, 0] >= 0
    seg = torch.sum(torch.arange(T, device=DEV)[:, None] >= st["seq"][None, 1:B].long(), dim=1) if B > 1 else \
        torch.zeros(T, dtype=torch.int64, device=DEV)
    m = z.amax(-1, keepdim=True)
    ez = torch.exp(z - m)
    sz = ez.sum(-1, keepdim=True)
    lse = (m + torch.log(sz))[:, 0]
    soft = ez / sz
    if c["gate"] == "softmax":
        r = soft
    else:
        sig = 1.0 / (1.0 + torch.exp(-z))
        r = sig / sig.sum(-1, keepdim=True)
    livef = live.float()
    tokens = torch.zeros(B, dtype=torch.int64, device=DEV).index_add_(0, seg, live.long())
    hit = torch.zeros(B, E + 1, dtype=torch.int64, device=DEV)
    key = (seg[:, None] * (E + 1) + torch.where(idx < 0, torch.full_like(idx, E), idx).long()).reshape(-1)
    hit.view(-1).index_add_(0, key, torch.ones_like(key))
    counts = hit[:, :E].contiguous()
    n = torch.clamp(tokens, min=1).float()
    share = torch.stack([torch.sum((r * livef[:, None])[a:b], 0) for a, b in st_bounds(st)]) / n[:, None]
    f = counts.float() / (k * n[:, None])
    full = torch.clamp((tokens > 0).sum(), min=1).float()
    total = torch.clamp(tokens.sum(), min=1).float()
    loss = torch.stack([E * torch.sum(f * share) / full, torch.sum(livef * lse * lse) / total])
    coef = (st["dloss"][0] * E * f / (n[:, None] * full))[seg]
    d = r * (coef - torch.sum(coef * r, -1, keepdim=True))
    if c["gate"] == "sigmoid":
        d = d * (1.0 - sig)
    d = d + (st["dloss"][1] * 2.0 / total) * lse[:, None] * soft
    dz = torch.where(live[:, None], d, torch.zeros_like(d)).to(st["logits"].dtype)
    return dict(loss=loss, counts=counts, share=share, tokens=tokens, dlogits=dz)


def st_bounds(st):
    """The sequences' (start, end) on the host, as the program that packed them knows them."""
    if "bounds" not in st:
        s = st["seq"].tolist()
        st["bounds"] = list(zip(s[:-1], s[1:]))
    return st["bounds"]


def _run_combine(st):
    c, dt = st["case"], DTYPES[st["case"]["dtype"]]
    y = st["y"].float()
    picked = y[st["pos"].long().reshape(-1)].reshape(c["T"], c["k"], c["H"])
    out = dict(out=torch.sum(picked * st["weight"][:, :, None], 1).to(dt))
    if c["train"]:
        d = st["dout"].float()
        out["dweight"] = torch.sum(picked * d[:, None, :], -1)
        dy = torch.empty_like(st["y"])
        dy[st["pos"].long().reshape(-1)] = (st["weight"][:, :, None] * d[:, None, :]).reshape(-1, c["H"]).to(dt)
        out["dy"] = dy
    return out


def _run_product(st):
    c, dt = st["case"], DTYPES[st["case"]["dtype"]]
    E, N, K, M = c["E"], c["N"], c["K"], c["T"] * c["k"]
    x = st["x"].float()
    xs = _round_rows(x)
    if st["rows"] is not None:
        xs = xs[st["rows"].long()]
    y = torch.empty(M, N, dtype=dt, device=DEV)
    if c["train"]:
        xg = x if st["rows"] is None else x[st["rows"].long()]
        dy = st["dy"].float()
        dys = _round_rows(dy)
        dx, dw = torch.empty(M, K, dtype=dt, device=DEV), torch.zeros(E, N, K, device=DEV)
    a = 0
    for e, n in enumerate(st["sizes"]):
        b = a + n
        if n > 0:
            q, s = _quantize_weight(st["w"][e].float()) if c["train"] else (st["codes"][e], st["scale"][e])
            w = q.float() * _spread(s, N, K)
            y[a:b] = (xs[a:b] @ w.t()).to(dt)
            if c["train"]:
                dx[a:b] = (dys[a:b] @ w).to(dt)
                dw[e] = _round_rows(dy[a:b].t()) @ _round_rows(xg[a:b].t()).t()
        a = b
    return dict(y=y, dx=dx, dw=dw) if c["train"] else dict(y=y)


def _run_own(st):
    c, m = st["case"], st["moe"]
    if c["kind"] == "route":
        r = m.route(st["logits"], c["k"], gate=st["gate"], prices=st["prices"], valid=st["valid"], out=st["out"])
        out = dict(idx=r.idx, weight=r.weight, counts=r.counts, rows=r.rows, pos=r.pos, offsets=r.offsets)
        if c["train"]:
            out["dlogits"] = m.route_backward(st["logits"], r.idx, gate=st["gate"], dweight=st["dweight"],
                                              out=st["dlogits"])
        return out
    if c["kind"] == "balance":
        b = m.balance(st["logits"], st["idx"], gate=st["gate"], seq_offsets=st["seq"], out=st["out"])
        dz = m.route_backward(st["logits"], st["idx"], gate=st["gate"], balance=b, seq_offsets=st["seq"],
                              dloss=st["dloss"], out=st["dlogits"])
        return dict(loss=b.loss, counts=b.counts, share=b.share, tokens=b.tokens, dlogits=dz)
    if c["kind"] == "combine":
        out = dict(out=m.combine(st["y"], st["pos"], st["weight"], out=st["out"]))
        if c["train"]:
            out["dy"], out["dweight"] = m.combine_backward(st["dout"], st["y"], st["pos"], st["weight"],
                                                           out=(st["dy"], st["dw"]))
        return out
    if c["train"]:
        m.quantize_weight(st["w"], out=st["weight"])
    y = m.linear(st["x"], st["weight"], offsets=st["offsets"], rows=st["rows"], out=st["y"])
    if not c["train"]:
        return dict(y=y)
    dx, dw = m.linear_backward(st["dy"], st["x"], st["weight"], offsets=st["offsets"], rows=st["rows"],
                               out=(st["dx"], st["dw"]))
    return dict(y=y, dx=dx, dw=dw)


def run(state):
    if own:
        return _run_own(state)
    return {"route": _run_route, "balance": _run_balance, "combine": _run_combine,
            "product": _run_product}[state["case"]["kind"]](state)


def work(case):
    c, size = case, 4 if case["dtype"] == "f32" else 2
    T, E, k = c["T"], c["E"], c["k"]
    if c["kind"] == "route":
        # logits, prices, padding marks; choices, weights, rows, places, counts, offsets; gradient
        b = size * T * E + (4 * E if c["prices"] else 0) + (T if c["masked"] else 0) + 16 * T * k + 12 * E + 4
        f = 4 * T * E
        if c["train"]:
            b, f = b + 4 * T * k + size * T * E, f + 4 * T * E
        return dict(bytes=b, flops=f)
    if c["kind"] == "balance":
        return dict(bytes=2 * size * T * E + 4 * T * k + 12 * c["B"] * E, flops=12 * T * E)
    if c["kind"] == "combine":
        H = c["H"]
        b, f = size * (T * k * H + T * H) + 8 * T * k, 2 * T * k * H
        if c["train"]:
            b, f = b + size * (T * H + T * k * H) + 4 * T * k, f + 3 * T * k * H
        return dict(bytes=b, flops=f)
    N, K, M = c["N"], c["K"], T * k
    used = min(E, M)
    b = size * (T * K + M * N) + used * N * K * (size if c["train"] else 1)
    if c["train"]:
        b += size * (M * N + M * K) + 4 * E * N * K
    return dict(bytes=b, flops=2 * M * N * K * (3 if c["train"] else 1))


# ---- the definition in 64 bits


def _exact_codes(v):
    """Nearest e4m3 value (ties to even), by the spacing of the value's binade."""
    _, e = torch.frexp(v)
    step = torch.ldexp(torch.ones_like(v), torch.clamp(e - 1, min=-6) - 3)
    return torch.clamp(torch.round(v / step) * step, -448.0, 448.0)


def _exact_round(x, amax):
    """Values that the 8-bit blocks stand for; amax spreads over x. Scale, its inverse and the scaled value are
    32-bit numbers by definition."""
    a = torch.clamp(amax, min=2.0 ** -100)
    f32 = lambda v: v.float().double()  # noqa: E731
    scale = torch.where(torch.isfinite(amax), f32(a / 448.0), torch.full_like(a, math.nan))
    return _exact_codes(f32(x * f32(448.0 / a))) * scale


def _exact_rows(x):
    out = torch.empty_like(x)
    for j in range(0, x.shape[1], BLOCK):
        b = x[:, j:j + BLOCK]
        out[:, j:j + BLOCK] = _exact_round(b, b.abs().amax(1, keepdim=True))
    return out


def _exact_weight(w):
    out = torch.empty_like(w)
    for i in range(0, w.shape[0], BLOCK):
        r = w[i:i + BLOCK]
        for j in range(0, r.shape[1], BLOCK):
            b = r[:, j:j + BLOCK]
            out[i:i + BLOCK, j:j + BLOCK] = _exact_round(b, b.abs().amax())
    return out


def _exact_gate(z, gate):
    """(probabilities over the experts, gate value of every expert)"""
    if gate == "softmax":
        p = torch.softmax(z, -1)
        return p, p
    s = torch.sigmoid(z)
    return s / s.sum(-1, keepdim=True), s


def exact(case, seed):
    c = case
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    if c["kind"] == "route":
        z32 = st["logits"].float()
        profit = z32 if st["prices"] is None else z32 - st["prices"]   # 32-bit by definition
        T, E, k = c["T"], c["E"], c["k"]
        ok = profit > -math.inf
        if st["valid"] is not None:
            ok &= st["valid"][:, None]
        z = z32.double()
        idx = torch.full((T, k), -1, dtype=torch.int64, device=DEV)
        left, rng = torch.where(ok, profit.double(), torch.full_like(z, -math.inf)), torch.arange(T, device=DEV)
        for j in range(k):
            best = left.amax(-1)
            first = torch.where(left == best[:, None], torch.arange(E, device=DEV), E).amin(-1)
            idx[:, j] = torch.where(best > -math.inf, first, torch.full_like(first, -1))
            left[rng, first] = -math.inf
        took = idx >= 0
        zz = z.clone().requires_grad_(c["train"])
        safe = torch.where(took[:, :1], zz, torch.zeros_like(zz))      # rows that chose nothing
        at = torch.clamp(idx, min=0)
        if c["renorm"]:
            a = safe if c["gate"] == "softmax" else torch.nn.functional.logsigmoid(safe)
            chosen = torch.where(took, torch.gather(a, 1, at), torch.full_like(at, -math.inf, dtype=torch.float64))
            chosen = torch.where(took[:, :1], chosen, torch.zeros_like(chosen))
            p = torch.softmax(chosen, -1)
        else:
            p = torch.gather(_exact_gate(safe, c["gate"])[1], 1, at)
        weight = 2.5 * torch.where(took, p, torch.zeros_like(p))
        rows, pos, offsets, counts = _plan(idx, E)
        out = dict(idx=idx.int(), weight=weight.detach(), counts=counts, rows=rows, pos=pos, offsets=offsets)
        if c["train"]:
            (weight * st["dweight"].double()).sum().backward()
            out["dlogits"] = torch.nan_to_num(zz.grad, nan=0.0)
        return out
    if c["kind"] == "balance":
        z = st["logits"].double().requires_grad_(True)
        E, k, B = c["E"], c["k"], c["B"]
        live = st["idx"][:, 0] >= 0
        r, _ = _exact_gate(z, c["gate"])
        counts, share, tokens, parts = [], [], [], []
        for a, b in st_bounds(st):
            on = live[a:b]
            n = int(on.sum())
            cnt = torch.sum(st["idx"][a:b].reshape(-1, 1) == torch.arange(E, device=DEV), 0)
            P = r[a:b][on].sum(0) / max(n, 1)
            counts.append(cnt), share.append(P), tokens.append(n)
            if n:
                parts.append(E * torch.sum(cnt.double() / (k * n) * P))
        bal = torch.stack(parts).mean() if parts else z.sum() * 0.0
        lse = torch.logsumexp(z[live], -1)
        zl = (lse * lse).sum() / max(int(live.sum()), 1)
        (st["dloss"][0].double() * bal + st["dloss"][1].double() * zl).backward()
        return dict(loss=torch.stack([bal, zl]).detach(), counts=torch.stack(counts),
                    share=torch.stack(share).detach(), tokens=torch.tensor(tokens, device=DEV), dlogits=z.grad)
    if c["kind"] == "combine":
        T, k, H = c["T"], c["k"], c["H"]
        pos, y = st["pos"].long(), st["y"]
        w = st["weight"].double()
        out = torch.zeros(T, H, dtype=torch.float64, device=DEV)
        for j in range(k):
            out += w[:, j:j + 1] * y[pos[:, j]].double()
        res = dict(out=out)
        if c["train"]:
            d = st["dout"].double()
            dy, dw = torch.zeros(T * k, H, dtype=torch.float64, device=DEV), torch.zeros_like(w)
            for j in range(k):
                dy[pos[:, j]] = w[:, j:j + 1] * d
                dw[:, j] = torch.sum(y[pos[:, j]].double() * d, -1)
            res["dy"], res["dweight"] = dy, dw
        return res
    E, N, K, M = c["E"], c["N"], c["K"], c["T"] * c["k"]
    x = st["x"].double()
    xr = _exact_rows(x)
    y = torch.empty(M, N, dtype=torch.float64, device=DEV)
    if c["train"]:
        dy = st["dy"].double()
        dyr = _exact_rows(dy)
        dx = torch.empty(M, K, dtype=torch.float64, device=DEV)
        dw = torch.zeros(E, N, K, dtype=torch.float64, device=DEV)
    a = 0
    for e, n in enumerate(st["sizes"]):
        b = a + n
        if n:
            pick = slice(a, b) if st["rows"] is None else st["rows"][a:b].long()
            if c["train"]:
                w = _exact_weight(st["w"][e].double())
            else:
                w = st["codes"][e].double() * _spread(st["scale"][e].double(), N, K)
            y[a:b] = xr[pick] @ w.t()
            if c["train"]:
                dx[a:b] = dyr[a:b] @ w
                dw[e] = _exact_rows(dy[a:b].t().contiguous()) @ _exact_rows(x[pick].t().contiguous()).t()
        a = b
    return dict(y=y, dx=dx, dw=dw) if c["train"] else dict(y=y)
