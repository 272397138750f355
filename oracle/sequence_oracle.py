"""Plain numpy fp64 definitions of the operators on packed sequences: norms of heads with
the position rotation, linear attention with a decay a head (whole sequences and a single
row), attention to the states of an encoder.  A row at a time, a sequence at a time;
nothing is blocked, fused or approximated.

Rows of all sequences stand back to back; sequence b has the rows offsets[b] ..
offsets[b + 1] - 1.  Rows of no sequence stay as `out` has them (NaN here)."""
from __future__ import annotations

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
