"""Oracle of the price-routed expert layer (include/esp_moe.h) in numpy fp64: the choice at prices, the gate
weights, the plan, the losses, the 8-bit products and every gradient's formula.

TEST INFRASTRUCTURE: only tests/ may import this module. It imports nothing from the library.

The choice compares fp32 differences (logit - price), and a block's scale and codes are chains of fp32
roundings by definition, so those steps are numpy float32 here; everything else is fp64.
"""

from __future__ import annotations

import numpy as np

BLOCK = 128


def _clean(z):
    z = np.asarray(z, np.float32)
    z = np.where(np.isnan(z), np.float32(-np.inf), z)
    return np.minimum(z, np.finfo(np.float32).max)


def choose(logits, k, prices=None, valid=None):
    """(T, k) int: experts of greatest fp32 profit, descending, ties to the lower index; -1: none left."""
    z = np.asarray(logits, np.float32)
    T, E = z.shape
    out = np.full((T, k), -1, np.int64)
    with np.errstate(invalid="ignore", over="ignore"):
        profit = z if prices is None else (z - np.asarray(prices, np.float32)).astype(np.float32)
    for t in range(T):
        if valid is not None and not valid[t]:
            continue
        order = sorted((e for e in range(E) if profit[t, e] > -np.inf), key=lambda e: (-float(profit[t, e]), e))
        out[t, :min(k, len(order))] = order[:k]
    return out


def softmax(a):
    a = np.asarray(a, np.float64)
    m = np.max(a, -1, keepdims=True)
    m = np.where(np.isfinite(m), m, 0.0)
    e = np.exp(a - m)
    s = e.sum(-1, keepdims=True)
    return e / np.where(s > 0, s, 1.0)


def logsumexp(a):
    a = np.asarray(a, np.float64)
    m = np.max(a, -1)
    return m + np.log(np.exp(a - m[..., None]).sum(-1))


def sigmoid(z):
    z = np.asarray(z, np.float64)
    e = np.exp(-np.abs(z))
    return np.where(z >= 0, 1.0 / (1.0 + e), e / (1.0 + e))


def log_sigmoid(z):
    z = np.asarray(z, np.float64)
    return np.minimum(z, 0.0) - np.log1p(np.exp(-np.abs(z)))


def _values(z, gate):
    return log_sigmoid(z) if gate == "sigmoid" else z


def gate_weight(logits, idx, gate, renorm, scale):
    z = _clean(logits).astype(np.float64)
    took = idx >= 0
    zc = np.where(took, np.take_along_axis(z, np.maximum(idx, 0), 1), 0.0)
    if renorm:
        p = softmax(np.where(took, _values(zc, gate), -np.inf))
    elif gate == "softmax":
        p = np.take_along_axis(softmax(z), np.maximum(idx, 0), 1)
    else:
        p = sigmoid(zc)
    return scale * np.where(took, p, 0.0)


def gate_weight_grad(logits, idx, gate, renorm, scale, dweight):
    """Gradient of sum(weight * dweight) in the logits."""
    z = _clean(logits).astype(np.float64)
    T, E = z.shape
    took = idx >= 0
    g = np.where(took, scale * np.asarray(dweight, np.float64), 0.0)
    zc = np.where(took, np.take_along_axis(z, np.maximum(idx, 0), 1), 0.0)
    p = np.where(took, gate_weight(logits, idx, gate, renorm, 1.0), 0.0)
    d = np.zeros((T, E))
    rows = np.arange(T)[:, None]
    if renorm:
        dj = p * (g - (g * p).sum(-1, keepdims=True))
        if gate == "sigmoid":
            dj = dj * sigmoid(-zc)
    elif gate == "softmax":
        s = softmax(z)
        np.add.at(d, (np.broadcast_to(rows, idx.shape)[took], idx[took]), g[took])
        d = s * (d - (g * p).sum(-1, keepdims=True))
        d[~took[:, 0]] = 0.0
        return d
    else:
        dj = g * p * sigmoid(-zc)
    np.add.at(d, (np.broadcast_to(rows, idx.shape)[took], idx[took]), dj[took])
    return d


def plan(idx, E):
    """(counts, offsets, rows, pos): slots by expert, in order."""
    T, k = idx.shape
    counts = np.bincount(idx[idx >= 0].ravel(), minlength=E).astype(np.int64)
    offsets = np.concatenate([[0], np.cumsum(counts)])
    rows, pos = np.full(T * k, -1, np.int64), np.full((T, k), -1, np.int64)
    at = offsets[:-1].copy()
    for t in range(T):
        for j in range(k):
            e = idx[t, j]
            if e >= 0:
                rows[at[e]], pos[t, j] = t, at[e]
                at[e] += 1
    return counts, offsets, rows, pos


def balance(logits, idx, gate, seq=None):
    """(loss (2,), counts (B, E), share (B, E), tokens (B,))."""
    z = _clean(logits).astype(np.float64)
    T, E = z.shape
    k = idx.shape[1]
    seq = np.asarray([0, T] if seq is None else seq)
    B = len(seq) - 1
    counts, share, tokens = np.zeros((B, E), np.int64), np.zeros((B, E)), np.zeros(B, np.int64)
    lse2, per = 0.0, []
    for b in range(B):
        live = np.arange(seq[b], seq[b + 1])
        live = live[idx[live, 0] >= 0]
        tokens[b] = len(live)
        if len(live) == 0:
            continue
        ch = idx[live]
        counts[b] = np.bincount(ch[ch >= 0].ravel(), minlength=E)
        share[b] = softmax(_values(z[live], gate)).mean(0)
        per.append(E * (counts[b] / (k * len(live)) * share[b]).sum())
        lse2 += (logsumexp(z[live]) ** 2).sum()
    n = tokens.sum()
    return np.array([np.mean(per) if per else 0.0, lse2 / n if n else 0.0]), counts, share, tokens


def balance_grad(logits, idx, gate, dloss, seq=None):
    z = _clean(logits).astype(np.float64)
    T, E = z.shape
    k = idx.shape[1]
    seq = np.asarray([0, T] if seq is None else seq)
    _, counts, _, tokens = balance(logits, idx, gate, seq)
    used, n = max((tokens > 0).sum(), 1), max(tokens.sum(), 1)
    d = np.zeros((T, E))
    for b in range(len(seq) - 1):
        for t in range(seq[b], seq[b + 1]):
            if idx[t, 0] < 0:
                continue
            c = dloss[0] * E * counts[b] / (k * tokens[b]) / (tokens[b] * used)
            r = softmax(_values(z[t], gate))
            dz = r * (c - (c * r).sum())
            if gate == "sigmoid":
                dz = dz * sigmoid(-z[t])
            d[t] = dz + dloss[1] * 2.0 * logsumexp(z[t]) / n * softmax(z[t])
    return d


def step_prices(prices, counts, eta, slack):
    counts = np.asarray(counts, np.float64)
    if counts.sum() == 0:
        return np.asarray(prices, np.float64)
    cap = slack * counts.sum() / len(counts)
    return np.maximum(0.0, np.asarray(prices, np.float64) + eta * (counts - cap) / cap)


# ---- 8-bit blocks


def e4m3(x):
    """Nearest e4m3 value, ties to even, saturated at 448 (3 fraction bits, exponents -6 .. 8, subnormals)."""
    x = np.asarray(x, np.float64)
    _, e = np.frexp(x)
    step = np.ldexp(1.0, np.maximum(e - 1, -6) - 3)
    return np.clip(np.rint(x / step) * step, -448.0, 448.0)


def block_scale(amax):
    """(scale, inverse) of blocks with these greatest magnitudes, fp32 chains by definition."""
    amax = np.asarray(amax, np.float32)
    a = np.maximum(amax, np.float32(2.0 ** -100))
    bad = ~np.isfinite(amax)
    with np.errstate(invalid="ignore"):
        scale = np.where(bad, np.float32(np.nan), a / np.float32(448.0)).astype(np.float32)
        inv = np.where(bad, np.float32(0.0), np.float32(448.0) / a).astype(np.float32)
    return scale, inv


def _codes(x, inv):
    x = np.where(np.isfinite(x), x, np.float32(0.0)).astype(np.float32)
    return e4m3((x * inv).astype(np.float32))


def quantize_rows(x):
    """(codes as values (M, K), scales (M, ceil(K / 128)))."""
    x = np.asarray(x, np.float32)
    M, K = x.shape
    nb = -(-K // BLOCK)
    codes, scales = np.zeros((M, K)), np.zeros((M, nb), np.float32)
    for b in range(nb):
        p = x[:, b * BLOCK:(b + 1) * BLOCK]
        s, inv = block_scale(np.abs(p).max(1))
        codes[:, b * BLOCK:(b + 1) * BLOCK] = _codes(p, inv[:, None])
        scales[:, b] = s
    return codes, scales


def quantize_weight(w):
    """(codes as values (N, K), scales (ceil(N / 128), ceil(K / 128)))."""
    w = np.asarray(w, np.float32)
    N, K = w.shape
    codes, scales = np.zeros((N, K)), np.zeros((-(-N // BLOCK), -(-K // BLOCK)), np.float32)
    for i in range(scales.shape[0]):
        for j in range(scales.shape[1]):
            at = np.s_[i * BLOCK:(i + 1) * BLOCK, j * BLOCK:(j + 1) * BLOCK]
            s, inv = block_scale(np.abs(w[at]).max())
            codes[at], scales[i, j] = _codes(w[at], inv), s
    return codes, scales


def spread_rows(codes, scales):
    return codes * np.repeat(scales.astype(np.float64), BLOCK, 1)[:, :codes.shape[1]]


def spread_weight(codes, scales):
    s = np.repeat(np.repeat(scales.astype(np.float64), BLOCK, 0), BLOCK, 1)
    return codes * s[:codes.shape[0], :codes.shape[1]]


def linear(x, weights, offsets, rows=None):
    """(y, magnitude): weights is a list of (codes, scales); magnitude is the same sum over absolute values.
    Rows outside every expert are NaN."""
    xr = spread_rows(*quantize_rows(x))
    if rows is not None:
        xr = xr[np.maximum(rows, 0)]
    M, N = xr.shape[0], weights[0][0].shape[0]
    y, mag = np.full((M, N), np.nan), np.full((M, N), np.nan)
    for e, w in enumerate(weights):
        a, b = offsets[e], offsets[e + 1]
        wd = spread_weight(*w)
        y[a:b] = xr[a:b] @ wd.T
        mag[a:b] = np.abs(xr[a:b]) @ np.abs(wd).T
    return y, mag


def linear_backward(dy, x, weights, offsets, rows=None):
    """(dx, |dx|, dw, |dw|)."""
    dyr = spread_rows(*quantize_rows(dy))
    xg = np.asarray(x, np.float32) if rows is None else np.asarray(x, np.float32)[np.maximum(rows, 0)]
    N, K = weights[0][0].shape
    dx, mx = np.full((dyr.shape[0], K), np.nan), np.full((dyr.shape[0], K), np.nan)
    dw, mw = np.zeros((len(weights), N, K)), np.zeros((len(weights), N, K))
    for e, w in enumerate(weights):
        a, b = offsets[e], offsets[e + 1]
        wd = spread_weight(*w)
        dx[a:b], mx[a:b] = dyr[a:b] @ wd, np.abs(dyr[a:b]) @ np.abs(wd)
        if b > a:
            u = spread_rows(*quantize_rows(np.asarray(dy, np.float32)[a:b].T))
            v = spread_rows(*quantize_rows(xg[a:b].T))
            dw[e], mw[e] = u @ v.T, np.abs(u) @ np.abs(v).T
    return dx, mx, dw, mw


def combine(y, pos, weight=None):
    y = np.asarray(y, np.float64)
    w = np.ones(pos.shape) if weight is None else np.asarray(weight, np.float64)
    picked = np.where((pos >= 0)[:, :, None], y[np.maximum(pos, 0)], 0.0)
    return (picked * w[:, :, None]).sum(1)


def combine_grad(dout, y, pos, weight=None):
    """(dy with zeros in rows without a place, dweight)."""
    y, d = np.asarray(y, np.float64), np.asarray(dout, np.float64)
    w = np.ones(pos.shape) if weight is None else np.asarray(weight, np.float64)
    dy, dw = np.zeros_like(y), np.zeros(pos.shape)
    for t in range(pos.shape[0]):
        for j in range(pos.shape[1]):
            if pos[t, j] >= 0:
                dy[pos[t, j]] = w[t, j] * d[t]
                dw[t, j] = d[t] @ y[pos[t, j]]
    return dy, dw
