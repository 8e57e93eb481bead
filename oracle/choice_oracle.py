"""Reference of the row-wise choices: draws from rows of scores, experts of rows, and their gradients.

Whole-number results follow the definition step by step: float32 scores scaled and raised with one
rounding a step (numpy rounds every float32 operation), then integers of any size.  Real-valued
results are float64.  Shares no code with the library.
"""
import math

import numpy as np

F = np.float32
LOG2E = F(1.4426950408889634)
COEF = [F(c) for c in (1.0, 0.693147, 0.24022242, 0.055507336, 0.009671513, 0.0013264727)]
MASKED = F(-np.inf)


def clean(scores):
    """float32 scores with NaN masked and -0 made +0."""
    x = np.asarray(scores, dtype=F)
    return np.where(np.isnan(x), MASKED, x + F(0))


def _split(t):
    """(p, e): 2^t as p 2^e."""
    with np.errstate(invalid="ignore"):
        e = np.rint(t)
        f = t - e
        p = np.full_like(f, COEF[5])
        for c in COEF[4::-1]:
            p = p * f + c
    assert p.dtype == F
    return p, e


def _below(x, m, scale):
    with np.errstate(invalid="ignore", over="ignore"):
        return np.where(x == m, F(0), (x - m) * scale).astype(F)


def fixed_weights(x, scale):
    """The integer weights of one cleaned row."""
    x = np.asarray(x, F)
    if x.size == 0 or x.max() == MASKED:
        return np.zeros(x.size, np.int64)
    t = _below(x, x.max(), F(scale))
    p, e = _split(t)
    out = np.zeros(x.size, np.int64)
    live = (x > MASKED) & (e >= -41)
    m = (p[live].astype(np.float64) * 2.0**24).astype(np.int64)  # exact
    down = (-e[live]).astype(np.int64)
    out[live] = (((m << 17) >> down) + 1) >> 1
    return out


def sample_row(scores, word, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(id, natural log of its probability, kept entries as indices) of one row."""
    x = clean(scores)
    T, p, mp = F(temperature), F(top_p), F(min_p)
    greedy = not T > 0
    with np.errstate(over="ignore"):
        scale = F(1) if greedy else LOG2E / T
    w = fixed_weights(x, scale)
    least = max(1, int(float(min(mp, F(1))) * 2**40)) if mp > 0 else 1
    order = sorted(np.flatnonzero(w >= least).tolist(), key=lambda i: (-float(x[i]), i))
    if greedy:
        order = order[:1]
    elif top_k > 0:
        order = order[:top_k]
    if p < 1:
        total = sum(int(w[i]) for i in order)
        target = max(1, total * int(float(max(p, F(0))) * 2**31) >> 31)
        short, before = [], 0
        for i in order:
            if before >= target:
                break
            short.append(i)
            before += int(w[i])
        order = short
    keep = sorted(order)
    total = sum(int(w[i]) for i in keep)
    if total == 0:
        return -1, -math.inf, []
    at = (int(word) & (2**64 - 1)) * total >> 64
    for i in keep:
        if at < int(w[i]):
            return i, math.log1p((int(w[i]) - total) / total), keep
        at -= int(w[i])
    raise AssertionError("unreachable")


def sample_probs(scores, temperature, keep):
    """float64 probabilities of the kept entries by the textbook formula."""
    x = clean(scores).astype(np.float64)[keep]
    q = np.exp((x - x.max()) / float(F(temperature)))
    return q / q.sum()


def route_scores(logits, kind):
    """(float32 scores, masked) of rows of logits, with the definition's rounding."""
    x = clean(logits)
    masked = x == MASKED
    if kind == "sigmoid":
        with np.errstate(over="ignore"):
            t = -(np.abs(x) * LOG2E)
        p, e = _split(t)
        live = e >= -126
        v = np.where(live, np.where(live, p, F(0)) * np.exp2(np.where(live, e, 0).astype(F)), F(0)).astype(F)
        s = np.where(x >= 0, F(1), v) / (F(1) + v)
    else:
        s = np.zeros_like(x)
        for r in range(x.shape[0]):
            m = x[r].max()
            if m == MASKED:
                continue
            z = int(fixed_weights(x[r], LOG2E).sum())
            inv = F(1) / (F(z) * F(2.0**-40))
            p, e = _split(_below(x[r], m, LOG2E))
            live = e >= -126
            s[r] = np.where(live, np.where(live, p, F(0)) * np.exp2(np.where(live, e, 0).astype(F)), F(0)).astype(F) * inv
    assert s.dtype == F
    return np.where(masked, F(0), s), masked


def route(logits, k, kind, bias=None, groups=1, top_groups=1, group_best=2, renorm=True, scale=1.0):
    """(experts, float64 weights) with the experts chosen by the float32 definition."""
    s, masked = route_scores(logits, kind)
    rows, E = s.shape
    experts = np.full((rows, k), -1, np.int64)
    weights = np.zeros((rows, k))
    size = E // groups
    for r in range(rows):
        c = s[r] if bias is None else s[r] + np.asarray(bias, F)
        ok = ~masked[r] & ~np.isnan(c) & (c != MASKED)
        if groups > 1:
            best = []
            for g in range(groups):
                inside = sorted((c[i] for i in range(g * size, (g + 1) * size) if ok[i]), reverse=True)[:group_best]
                if inside:
                    best.append((-float(inside[0] + inside[1] if len(inside) > 1 else inside[0]), g))
            take = {g for _, g in sorted(best)[:top_groups]}
            ok &= np.array([i // size in take for i in range(E)])
        chosen = sorted(np.flatnonzero(ok).tolist(), key=lambda i: (-float(c[i]), i))[:k]
        experts[r, : len(chosen)] = chosen
        v = s[r, chosen].astype(np.float64)
        if renorm:
            v = v / v.sum() if v.sum() > 0 else np.zeros_like(v)
        weights[r, : len(chosen)] = v * float(F(scale))
    return experts, weights


def scores64(logits, kind):
    x = clean(logits).astype(np.float64)
    if kind == "sigmoid":
        e = np.exp(-np.abs(x))
        return np.where(x == -np.inf, 0.0, np.where(x >= 0, 1.0, e) / (1 + e))
    m = x.max(1, keepdims=True)
    e = np.exp(x - np.where(m == -np.inf, 0, m))
    z = e.sum(1, keepdims=True)
    return e / np.where(z > 0, z, 1)


def weights64(logits, experts, kind, renorm, scale):
    """The weights of fixed experts as a function of the logits, in float64."""
    s = scores64(logits, kind)
    v = np.where(experts >= 0, np.take_along_axis(s, np.maximum(experts, 0), 1), 0.0)
    if renorm:
        d = v.sum(1, keepdims=True)
        v = v / np.where(d > 0, d, 1)
    return v * scale


def route_gradient(logits, experts, dweights, kind, renorm, scale):
    """d/dlogits of sum(dweights * weights64), by the chain rule in float64."""
    s = scores64(logits, kind)
    at = np.maximum(experts, 0)
    v = np.where(experts >= 0, np.take_along_axis(s, at, 1), 0.0)
    g = np.where(experts >= 0, np.asarray(dweights, np.float64) * scale, 0.0)
    if renorm:
        d = v.sum(1, keepdims=True)
        d1 = np.where(d > 0, d, 1)
        g = np.where((experts >= 0) & (d > 0), (g - (g * v / d1).sum(1, keepdims=True)) / d1, 0.0)
    ds = np.zeros_like(s)
    for j in range(experts.shape[1]):
        r = np.flatnonzero(experts[:, j] >= 0)
        ds[r, experts[r, j]] += g[r, j]
    if kind == "sigmoid":
        return ds * s * (1 - s)
    return s * (ds - (ds * s).sum(1, keepdims=True))


def plan(experts, n_experts):
    """(offsets, order, slot) by sorting (expert, pair number)."""
    flat = np.asarray(experts).reshape(-1)
    pairs = sorted((int(e), i) for i, e in enumerate(flat) if 0 <= e < n_experts)
    order = np.full(flat.size, -1, np.int64)
    slot = np.full(flat.size, -1, np.int64)
    for s, (_, i) in enumerate(pairs):
        order[s], slot[i] = i, s
    offsets = np.array([sum(1 for e, _ in pairs if e < b) for b in range(n_experts + 1)])
    return offsets, order, slot.reshape(np.shape(experts))


def combine(y, slot, weights=None):
    y = np.asarray(y, np.float64)
    out = np.zeros((slot.shape[0], y.shape[1]))
    for j in range(slot.shape[1]):
        w = 1.0 if weights is None else np.asarray(weights, np.float64)[:, j, None]
        out += np.where(slot[:, j, None] >= 0, w * y[np.maximum(slot[:, j], 0)], 0.0)
    return out


def combine_gradient(dout, y, slot, weights):
    dout, y = np.asarray(dout, np.float64), np.asarray(y, np.float64)
    dy, dw = np.zeros_like(y), np.zeros(slot.shape)
    for t in range(slot.shape[0]):
        for j in range(slot.shape[1]):
            if slot[t, j] >= 0:
                dy[slot[t, j]] = float(weights[t, j]) * dout[t]
                dw[t, j] = dout[t] @ y[slot[t, j]]
    return dy, dw
