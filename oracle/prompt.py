"""Oracle of a recurrent layer's prompt pass in plain fp64 numpy: packed
sequences token by token, straight from the definitions of include/sla.h."""
from __future__ import annotations

import numpy as np


def prefill(state, q, k, v, alpha, beta, starts, family="gdn"):
    """(out [T][H][dv], state_out [B][H][dk][dv]) of sla_prefill.  q, k [T][Hk][dk],
    v [T][H][dv]; state [B][H][dk][dv] or None.  Rows of no sequence come back as NaN."""
    T, H, dv = v.shape
    B, dk, group = len(starts) - 1, q.shape[2], H // q.shape[1]
    S = np.zeros((B, H, dk, dv)) if state is None else np.array(state, np.float64)
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    out = np.full((T, H, dv), np.nan)
    for b in range(B):
        for t in range(starts[b], starts[b + 1]):
            kt, qt = np.repeat(k[t], group, 0), np.repeat(q[t], group, 0)
            u = v[t]
            if family != "deltanet":
                S[b] *= np.asarray(alpha, np.float64)[t][:, None, None]
            if family != "decay":
                u = np.asarray(beta, np.float64)[t][:, None] * (u - np.einsum("hk,hkv->hv", kt, S[b]))
            S[b] += kt[:, :, None] * u[:, None, :]
            out[t] = np.einsum("hk,hkv->hv", qt, S[b])
    return out, S


def conv(state, x, weight, bias, starts, silu=True):
    """(y [T][D], state_out [B][K-1][D]) of sla_conv_prefill; rows of no sequence NaN."""
    T, D = x.shape
    B, K = len(starts) - 1, weight.shape[1]
    w = np.asarray(weight, np.float64)
    y, new = np.full((T, D), np.nan), np.zeros((B, K - 1, D))
    for b in range(B):
        old = np.zeros((K - 1, D)) if state is None else np.asarray(state[b], np.float64)
        line = np.concatenate([old, np.asarray(x[starts[b]:starts[b + 1]], np.float64)])
        n = starts[b + 1] - starts[b]
        for t in range(n):
            s = (line[t:t + K] * w.T).sum(0) + (0 if bias is None else np.asarray(bias, np.float64))
            y[starts[b] + t] = s / (1 + np.exp(-s)) if silu else s
        new[b] = line[n:]
    return y, new


def inputs(q, k, a, b, a_log, dt_bias, q_scale, eps, repeat=1):
    """(q_out, k_out, alpha, beta) of sla_recurrent_inputs (None for an absent gate)."""
    unit = lambda x: np.repeat(x / np.sqrt((x * x).sum(-1, keepdims=True) + eps), repeat, 1)
    q, k = (np.asarray(x, np.float64) for x in (q, k))
    alpha = beta = None
    if a is not None:
        x = np.asarray(a, np.float64) + (0 if dt_bias is None else np.asarray(dt_bias, np.float64))
        alpha = np.exp(-np.exp(np.asarray(a_log, np.float64)) * np.logaddexp(0, x))
    if b is not None:
        beta = 1 / (1 + np.exp(-np.asarray(b, np.float64)))
    return q_scale * unit(q), unit(k), alpha, beta


def gated_norm(x, z, weight, eps, gate):
    """y of sla_gated_norm."""
    x = np.asarray(x, np.float64)
    y = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    if weight is not None:
        y = y * np.asarray(weight, np.float64)
    if gate != "none":
        z = np.asarray(z, np.float64)
        with np.errstate(over="ignore"):
            s = 1 / (1 + np.exp(-z))
        y = y * (z * s if gate == "silu" else s)
    return y
