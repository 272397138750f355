"""Plain numpy fp64 definitions of the operators on packed sequences: norms of heads with
the position rotation, linear attention with a decay a head (whole sequences and a single
row), attention to the states of an encoder, the gated recurrence with its gradients, the
norm with a residual's addition, the product with its epilogue.  A row at a time, a sequence
at a time; nothing is blocked, fused or approximated.

Rows of all sequences stand back to back; sequence b has the rows offsets[b] ..
offsets[b + 1] - 1.  Rows of no sequence stay as `out` has them (NaN here)."""
from __future__ import annotations

import math

import numpy as np


def qk_norm(x, gain, eps, positions=None, rot_dim=0, rot_base=10000.0):
    """x [N, H, D] -> each head over sqrt(mean of squares + eps), times gain [D] (None: 1),
    the pairs (i, i + rot_dim / 2) turned by positions * rot_base^(-2 i / rot_dim)."""
    x = np.asarray(x, np.float64)
    y = x / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps)
    if gain is not None:
        y = y * np.asarray(gain, np.float64)
    h = rot_dim // 2
    if h:
        out = y.copy()
        for i in range(h):
            a = np.asarray(positions, np.float64) * float(rot_base) ** (-2.0 * i / rot_dim)
            c, s = np.cos(a)[:, None], np.sin(a)[:, None]
            out[..., i] = y[..., i] * c - y[..., i + h] * s
            out[..., i + h] = y[..., i] * s + y[..., i + h] * c
        y = out
    return y


def linear_attention(q, k, v, log_decay, offsets, scale=1.0, reverse=False, state_in=None):
    """S <- exp(g) S + k v^T, o = scale S^T q along each sequence: (out [N, H, V], states
    [B, H, K, V] after each sequence)."""
    q, k, v, g = (np.asarray(t, np.float64) for t in (q, k, v, log_decay))
    N, H, K = q.shape
    V = v.shape[2]
    B = len(offsets) - 1
    out = np.full((N, H, V), np.nan)
    states = np.zeros((B, H, K, V)) if state_in is None else np.array(state_in, np.float64)
    for b in range(B):
        S = states[b]
        rows = range(int(offsets[b]), int(offsets[b + 1]))
        for t in (reversed(rows) if reverse else rows):
            S = np.exp(g[t])[:, None, None] * S + k[t][:, :, None] * v[t][:, None, :]
            out[t] = scale * np.einsum("hkv,hk->hv", S, q[t])
        states[b] = S
    return out, states


def linear_attention_step(q, k, v, log_decay, state, scale=1.0):
    """One row a sequence: (out [B, H, V], states [B, H, K, V])."""
    B = q.shape[0]
    return linear_attention(q, k, v, log_decay, np.arange(B + 1), scale, False, state)


def cross_attention(q, k, v, q_offsets, kv_offsets, scale):
    """softmax(scale q k^T) v, the queries of a sequence over its states; zeros where there
    are none.  q [Nq, Hq, D], k, v [Nk, Hk, D]: head h reads head h // (Hq / Hk)."""
    q, k, v = (np.asarray(t, np.float64) for t in (q, k, v))
    out = np.full(q.shape, np.nan)
    G = q.shape[1] // k.shape[1]
    for b in range(len(q_offsets) - 1):
        qs = slice(int(q_offsets[b]), int(q_offsets[b + 1]))
        ks = slice(int(kv_offsets[b]), int(kv_offsets[b + 1]))
        if ks.stop <= ks.start:
            out[qs] = 0.0
            continue
        for h in range(q.shape[1]):
            s = scale * q[qs, h] @ k[ks, h // G].T
            p = np.exp(s - s.max(axis=1, keepdims=True))
            out[qs, h] = (p / p.sum(axis=1, keepdims=True)) @ v[ks, h // G]
    return out


def logistic(x):
    """1 / (1 + exp(-x)), accurate near 0 too."""
    x = np.asarray(x, np.float64)
    e = np.exp(-np.abs(x))
    return np.where(x >= 0, 1.0, e) / (1.0 + e)


def gated_scan(p, n, offsets, reverse=False, state_in=None):
    """h <- h + sigma(p) (n - h) along each sequence: (out [N, C], states [B, C] after each)."""
    p, n = np.asarray(p, np.float64), np.asarray(n, np.float64)
    z = logistic(p)
    B = len(offsets) - 1
    out = np.full(n.shape, np.nan)
    states = np.zeros((B, n.shape[1])) if state_in is None else np.array(state_in, np.float64)
    for b in range(B):
        h = states[b]
        rows = range(int(offsets[b]), int(offsets[b + 1]))
        for t in (reversed(rows) if reverse else rows):
            h = h + z[t] * (n[t] - h)
            out[t] = h
        states[b] = h
    return out, states


def gated_scan_backward(p, n, offsets, d_out, reverse=False, state_in=None, d_state_out=None):
    """Gradients of p, n [N, C] and of the first states [B, C]."""
    p, n, g = (np.asarray(t, np.float64) for t in (p, n, d_out))
    z, w = logistic(p), logistic(-p)
    B, C = len(offsets) - 1, n.shape[1]
    dp, dn = np.full(n.shape, np.nan), np.full(n.shape, np.nan)
    h, _ = gated_scan(p, n, offsets, reverse, state_in)
    first = np.zeros((B, C)) if state_in is None else np.asarray(state_in, np.float64)
    d0 = np.zeros((B, C)) if d_state_out is None else np.array(d_state_out, np.float64)
    for b in range(B):
        rows = list(range(int(offsets[b]), int(offsets[b + 1])))
        if reverse:
            rows.reverse()
        d = d0[b]
        for i in range(len(rows) - 1, -1, -1):
            t = rows[i]
            before = h[rows[i - 1]] if i > 0 else first[b]
            d = d + g[t]
            dn[t] = z[t] * d
            dp[t] = z[t] * w[t] * (n[t] - before) * d
            d = w[t] * d
        d0[b] = d
    return dp, dn, d0


def e4m3(x):
    """The nearest values of the 8-bit type (halves to even), for |x| <= 448."""
    x = np.asarray(x, np.float64)
    with np.errstate(divide="ignore", invalid="ignore"):
        step = np.exp2(np.maximum(np.floor(np.log2(np.abs(x))), -6) - 3)
    return np.where(np.abs(x) > 0, np.round(x / step) * step, x)


def add_norm(x, delta, gain, eps):
    """(s, y): s = x + delta (None: x), y = s over sqrt(mean of squares + eps), times gain."""
    s = np.asarray(x, np.float64) + (0.0 if delta is None else np.asarray(delta, np.float64))
    y = s / np.sqrt(np.mean(s * s, axis=-1, keepdims=True) + eps)
    return s, y if gain is None else y * np.asarray(gain, np.float64)


def product(x, weight, bias=None, activation="none", gate=None, residual=None):
    """residual + act(x W^T + bias) * sigma(gate); None: left out."""
    y = np.asarray(x, np.float64) @ np.asarray(weight, np.float64).T
    if bias is not None:
        y = y + np.asarray(bias, np.float64)
    if activation == "relu":
        y = np.maximum(y, 0.0)
    elif activation == "silu":
        y = y * logistic(y)
    elif activation == "gelu":
        y = y * 0.5 * np.vectorize(math.erfc, otypes=[float])(-y / math.sqrt(2.0))
    if gate is not None:
        y = y * logistic(gate)
    return y if residual is None else y + np.asarray(residual, np.float64)
