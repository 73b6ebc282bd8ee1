"""TEST INFRASTRUCTURE ONLY: fp64 definitions of the operators of state space language models, as plain NumPy, step by step.  Like the
rest of the oracle it shares no code with the CUDA package and takes and returns float64 arrays holding the exact values of the
stored tensors."""
from __future__ import annotations

import numpy as np


def _ends(lengths, T, B):
    return [T] * B if lengths is None else [min(max(int(n), 0), T) for n in lengths]


def _logistic(x):
    e = np.exp(-np.abs(x))
    return np.where(x >= 0, 1 / (1 + e), e / (1 + e))


def _silu(x):
    """x sigmoid(x) and its slope."""
    p, q = _logistic(x), _logistic(-x)
    return x * p, p * (1 + x * q)


# ---- short causal convolution ----
def causal_conv(x, w, b, before, lengths, silu):
    """x (T,B,D), w (K,D), b (D) or None, before (K-1,B,D) or None -> y (T,B,D), after (K-1,B,D)."""
    T, B, D = x.shape
    K = w.shape[0]
    y, after = np.zeros((T, B, D)), np.zeros((K - 1, B, D))
    for i, end in enumerate(_ends(lengths, T, B)):
        line = np.concatenate([np.zeros((K - 1, D)) if before is None else before[:, i], x[:end, i]])
        for t in range(end):
            s = np.zeros(D) if b is None else b.copy()
            for k in range(K):
                s = s + w[k] * line[t + k]
            y[t, i] = _silu(s)[0] if silu else s
        after[:, i] = line[end:end + K - 1]
    return y, after


def causal_conv_grad(x, w, b, before, lengths, silu, dy, dafter):
    """-> dx (T,B,D), dw (K,D), db (D), dbefore (K-1,B,D)."""
    T, B, D = x.shape
    K = w.shape[0]
    dx, dw, db, dbefore = np.zeros((T, B, D)), np.zeros((K, D)), np.zeros(D), np.zeros((K - 1, B, D))
    for i, end in enumerate(_ends(lengths, T, B)):
        line = np.concatenate([np.zeros((K - 1, D)) if before is None else before[:, i], x[:end, i]])
        dline = np.zeros_like(line)
        if dafter is not None:
            dline[end:end + K - 1] += dafter[:, i]
        for t in range(end):
            s = np.zeros(D) if b is None else b.copy()
            for k in range(K):
                s = s + w[k] * line[t + k]
            g = dy[t, i] * (_silu(s)[1] if silu else 1.0)
            db += g
            for k in range(K):
                dw[k] += g * line[t + k]
                dline[t + k] += g * w[k]
        dbefore[:, i] = dline[:K - 1]
        dx[:end, i] = dline[K - 1:]
    return dx, dw, db, dbefore


# ---- selective scan ----
def _steps(delta, delta_bias, softplus):
    raw = delta if delta_bias is None else delta + delta_bias
    return raw, (np.logaddexp(raw, 0.0) if softplus else raw)


def _sizes(x):
    return None if x is None else np.abs(x)


def selective_scan(u, delta, a, b, c, d, z, delta_bias, h0, lengths, softplus, span=None, sizes=False):
    """u, delta, z (T,B,D), a (D,N), b, c (T,B,N), d, delta_bias (D), h0 (B,D,N); d, z, delta_bias, h0 may be None
    -> y (T,B,D), h_final (B,D,N), and with `span` the states before every span-th step (ceil(T/span),B,D,N).
    With `sizes` every term of every sum enters with its absolute value: what rounding errors are measured against."""
    if sizes:
        u, b, c, d, h0 = (_sizes(v) for v in (u, b, c, d, h0))
    T, B, D = u.shape
    N = a.shape[1]
    _, step = _steps(delta, delta_bias, softplus)
    y, h_final = np.zeros((T, B, D)), np.zeros((B, D, N)) if h0 is None else h0.copy()
    states = np.zeros((-(-T // span) if span else 0, B, D, N))
    for i, end in enumerate(_ends(lengths, T, B)):
        h = h_final[i]
        for t in range(T):
            if span and t % span == 0:
                states[t // span, i] = h
            if t >= end:
                continue
            h = np.exp(step[t, i][:, None] * a) * h + (step[t, i] * u[t, i])[:, None] * b[t, i]
            y[t, i] = h @ c[t, i] + (0.0 if d is None else d * u[t, i])
            if z is not None:
                y[t, i] *= np.abs(_silu(z[t, i])[0]) if sizes else _silu(z[t, i])[0]
        h_final[i] = h
    return (y, h_final, states) if span else (y, h_final)


def selective_scan_grad(u, delta, a, b, c, d, z, delta_bias, h0, lengths, softplus, dy, dh_final, sizes=False):
    """-> dict of du, ddelta, da, db, dc, dd, dz, ddelta_bias, dh0; `sizes` as above."""
    if sizes:
        u, b, c, d, h0, dy, dh_final = (_sizes(v) for v in (u, b, c, d, h0, dy, dh_final))
    T, B, D = u.shape
    N = a.shape[1]
    raw, step = _steps(delta, delta_bias, softplus)
    o = dict(du=np.zeros((T, B, D)), ddelta=np.zeros((T, B, D)), da=np.zeros((D, N)), db=np.zeros((T, B, N)), dc=np.zeros((T, B, N)),
             dd=np.zeros(D), dz=np.zeros((T, B, D)), ddelta_bias=np.zeros(D), dh0=np.zeros((B, D, N)))
    for i, end in enumerate(_ends(lengths, T, B)):
        h = [np.zeros((D, N)) if h0 is None else h0[i]]
        for t in range(end):
            h.append(np.exp(step[t, i][:, None] * a) * h[-1] + (step[t, i] * u[t, i])[:, None] * b[t, i])
        G = np.zeros((D, N)) if dh_final is None else dh_final[i].copy()
        for t in range(end - 1, -1, -1):
            e = dy[t, i]
            if z is not None:
                plain = h[t + 1] @ c[t, i] + (0.0 if d is None else d * u[t, i])
                gate, slope = (np.abs(v) if sizes else v for v in _silu(z[t, i]))
                o["dz"][t, i] = e * plain * slope
                e = e * gate
            g = e[:, None] * c[t, i] + G
            G = np.exp(step[t, i][:, None] * a) * g
            along, left = g @ b[t, i], G * h[t]
            o["dc"][t, i] = e @ h[t + 1]
            o["db"][t, i] = (step[t, i] * u[t, i]) @ g
            o["du"][t, i] = along * step[t, i] + (0.0 if d is None else e * d)
            o["dd"] += e * u[t, i]
            o["da"] += left * step[t, i][:, None]
            s = along * u[t, i] + np.sum(left * (np.abs(a) if sizes else a), axis=1)
            o["ddelta"][t, i] = s * (_logistic(raw[t, i]) if softplus else 1.0)
        o["dh0"][i] = G
    o["ddelta_bias"] = o["ddelta"].sum(axis=(0, 1))
    return o


# ---- log-probabilities from the head's operands ----
def linear_logprob(x, w, tokens, temperature):
    """x (N,K), w (K,V) -> logp, lse (N,)."""
    N, V = x.shape[0], w.shape[1]
    logp, lse = np.zeros(N), np.zeros(N)
    for i in range(N):
        with np.errstate(invalid="ignore"):
            z = (x[i] @ w) / temperature
        if np.any(np.isnan(z)) or np.any(np.isposinf(z)):
            lse[i] = np.nan
        elif np.all(np.isneginf(z)):
            lse[i] = -np.inf
        else:
            lse[i] = z.max() + np.log(np.exp(z - z.max()).sum())
        if 0 <= tokens[i] < V:
            logp[i] = -np.inf if np.isneginf(lse[i]) else z[tokens[i]] - lse[i]
    return logp, lse


def linear_logprob_grad(x, w, tokens, temperature, lse, dlogp, sizes=False):
    """-> dx (N,K), dw (K,V); rows without a token, or without a class that can occur, have no part in either.  With `sizes` every
    term enters with its absolute value, the one and the probability of a token each."""
    dx, dw = np.zeros(x.shape), np.zeros(w.shape)
    for i in range(x.shape[0]):
        if not 0 <= tokens[i] < w.shape[1] or np.isneginf(lse[i]):
            continue
        dz = -dlogp[i] * np.exp((x[i] @ w) / temperature - lse[i])
        if sizes:
            dz = np.abs(dz)
        dz[tokens[i]] += abs(dlogp[i]) if sizes else dlogp[i]
        dz /= temperature
        dx[i] = np.abs(w) @ dz if sizes else w @ dz
        dw += np.outer(np.abs(x[i]), dz) if sizes else np.outer(x[i], dz)
    return dx, dw
