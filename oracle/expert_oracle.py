"""Float64 restatement of the operators of training and answering (test infrastructure only): given
entries of rows of scores, the gated feed-forward block of experts, dropout, and their gradients."""
import math

import numpy as np

from oracle.erc_oracle import philox4x32_10


def score_row(l, i, temperature=1.0, k=0):
    """(logp, entropy, (m, ln Z), top_ids, top_logp) of a row of scores, as read (float32 values)."""
    l = np.asarray(l, np.float64)
    l = np.where(np.isnan(l), -np.inf, l) + 0.0
    n = l.size
    none = np.full(k, -1, np.int64), np.full(k, -np.inf)
    given = 0 <= i < n
    if n == 0 or l.max() == -np.inf:
        return (-math.inf if given else 0.0), 0.0, (-math.inf, -math.inf), *none
    m = l.max()
    t = np.full(n, -np.inf)
    live = l > -np.inf
    t[l == m] = 0.0
    if m < np.inf:
        rest = live & (l < m)
        t[rest] = (l[rest] - m) / temperature
    e = np.exp(t)
    z = e.sum()
    log_p = t - math.log(z)
    entropy = math.log(z) - (e[e > 0] * t[e > 0]).sum() / z
    by = np.lexsort((np.arange(n), -l))[:k]
    by = by[live[by]]
    none[0][: by.size], none[1][: by.size] = by, log_p[by]
    # a finite score beside an infinite maximum is unmasked, with probability 0
    return (log_p[i] if given else 0.0), entropy, (m, math.log(z)), *none


def score_row_backward(l, i, dlogp, dentropy, temperature=1.0):
    l = np.asarray(l, np.float64)
    l = np.where(np.isnan(l), -np.inf, l)
    n = l.size
    if n == 0 or l.max() == -np.inf:
        return np.zeros(n)
    m = l.max()
    with np.errstate(invalid="ignore"):
        t = np.where(l == m, 0.0, (l - m) / temperature)
    log_p = t - math.log(np.exp(t).sum())
    p = np.exp(log_p)
    live = p > 0
    entropy = -(p[live] * log_p[live]).sum()
    g = dlogp if 0 <= i < n and l[i] > -np.inf else 0.0
    out = np.zeros(n)
    out[live] = -p[live] * (g + dentropy * (log_p[live] + entropy))
    if g:
        out[i] += g
    return out / temperature


def act_both(a, act):
    """(act(a), act'(a)); act 0: silu, 1: gelu, 2: relu"""
    a = np.asarray(a, np.float64)
    if act == 2:
        return np.maximum(a, 0.0), (a > 0).astype(np.float64)
    if act == 0:
        q = 1.0 / (1.0 + np.exp(-a))
        return a * q, q * (1.0 + a * (1.0 - q))
    q = 0.5 * (1.0 + np.array([math.erf(v) for v in (a / math.sqrt(2.0)).ravel()]).reshape(a.shape))
    return a * q, q + a * np.exp(-0.5 * a * a) / math.sqrt(2.0 * math.pi)


def ffn(x, offsets, w_in, w_out, act):
    """(y, pre) of rows in expert order; zeros behind offsets[-1]."""
    x, w_in, w_out = (np.asarray(v, np.float64) for v in (x, w_in, w_out))
    inner = w_out.shape[2]
    y, pre = np.zeros((x.shape[0], w_out.shape[1])), np.zeros((x.shape[0], 2 * inner))
    for e in range(w_in.shape[0]):
        s = slice(int(offsets[e]), int(offsets[e + 1]))
        pre[s] = x[s] @ w_in[e].T
        y[s] = (act_both(pre[s, :inner], act)[0] * pre[s, inner:]) @ w_out[e].T
    return y, pre


def ffn_backward(dy, x, pre, offsets, w_in, w_out, act):
    """(dx, dw_in, dw_out) from the stored pre."""
    dy, x, pre, w_in, w_out = (np.asarray(v, np.float64) for v in (dy, x, pre, w_in, w_out))
    inner = w_out.shape[2]
    dx, dw_in, dw_out = np.zeros_like(x), np.zeros_like(w_in), np.zeros_like(w_out)
    for e in range(w_in.shape[0]):
        s = slice(int(offsets[e]), int(offsets[e + 1]))
        a, b = pre[s, :inner], pre[s, inner:]
        value, slope = act_both(a, act)
        dh = dy[s] @ w_out[e]
        dpre = np.concatenate([dh * b * slope, dh * value], 1)
        dx[s], dw_in[e], dw_out[e] = dpre @ w_in[e], dpre.T @ x[s], dy[s].T @ (value * b)
    return dx, dw_in, dw_out


def dropout_keep(count, p, key, first=0):
    """Which of `count` entries stay; first: a multiple of 4."""
    at = first // 4 + np.arange((count + 3) // 4, dtype=np.uint64)
    words = philox4x32_10((at & np.uint64(0xFFFFFFFF), at >> np.uint64(32), np.uint64(0x44524F50), np.uint64(0)),
                          (key & 0xFFFFFFFF, (key >> 32) & 0xFFFFFFFF))
    return (np.stack(np.broadcast_arrays(*words), 1).astype(np.uint64) >= int(p * 2.0**32)).ravel()[:count]


def dropout(x, p, key, residual=None, first=0):
    """float32 results before the last rounding, every step rounded to float32 as the library does."""
    x = np.asarray(x, np.float32)
    scale = np.float32(1.0 / (1.0 - p)) if p < 1 else np.float32(0)
    keep = dropout_keep(x.size, p, key, first).reshape(x.shape)
    with np.errstate(invalid="ignore"):
        out = np.where(keep, x * scale, np.float32(0))
    return out if residual is None else out + np.asarray(residual, np.float32)
