"""TEST INFRASTRUCTURE ONLY: fp64 definitions of the operators of recurrent language models, as plain NumPy, step by step and
row by row.  Like the rest of the oracle it shares no code with the CUDA package and takes and returns float64 arrays holding
the exact values of the stored tensors."""
from __future__ import annotations

import numpy as np

GATE_GIVEN, GATE_SIGMOID, GATE_MIX = 0, 1, 2


def _sigmoid(x):
    """(sigmoid(x), 1 - sigmoid(x)) without cancellation."""
    e = np.exp(-np.abs(x))
    large, small = 1 / (1 + e), e / (1 + e)
    return np.where(x >= 0, large, small), np.where(x >= 0, small, large)


def _coefficients(f, u, gate):
    """a, the factor of u in b, and 1 - a."""
    if gate == GATE_GIVEN:
        return f, np.ones_like(f), None
    a, s = _sigmoid(f)
    return a, (s if gate == GATE_MIX else np.ones_like(f)), s


def _ends(lengths, T, B):
    return [T] * B if lengths is None else [min(max(int(n), 0), T) for n in lengths]


def gated_recurrence(f, u, h0, lengths, gate):
    """f, u (T,B,D), h0 (B,D) -> h_all (T,B,D), h_final (B,D)."""
    T, B, D = f.shape
    h_all, h_final = np.zeros((T, B, D)), np.array(h0, dtype=np.float64)
    for b, end in enumerate(_ends(lengths, T, B)):
        h = h0[b].astype(np.float64)
        for t in range(end):
            a, i, _ = _coefficients(f[t, b], u[t, b], gate)
            h = a * h + i * u[t, b]
            h_all[t, b] = h
        h_final[b] = h
    return h_all, h_final


def gated_recurrence_grad(f, u, h0, lengths, gate, h_all, dh_all, dh_final):
    """-> df, du (T,B,D), dh0 (B,D), from the saved h_all."""
    T, B, D = f.shape
    df, du, dh0 = np.zeros((T, B, D)), np.zeros((T, B, D)), np.array(dh_final, dtype=np.float64)
    for b, end in enumerate(_ends(lengths, T, B)):
        carry = dh_final[b].astype(np.float64)
        for t in range(end - 1, -1, -1):
            a, i, s = _coefficients(f[t, b], u[t, b], gate)
            before = h_all[t - 1, b] if t > 0 else h0[b]
            g = dh_all[t, b] + carry
            da = g * before - (g * u[t, b] if gate == GATE_MIX else 0.0)
            df[t, b] = da if gate == GATE_GIVEN else da * a * s
            du[t, b] = g * i
            carry = a * g
        dh0[b] = carry
    return df, du, dh0


def token_logprob(scores, tokens, temperature, top=0):
    """scores (N,V), tokens (N,) or None -> dict of logp, entropy, lse (N,), top_ids, top_logp (N,top)."""
    N, V = scores.shape
    out = dict(logp=np.zeros(N), entropy=np.zeros(N), lse=np.zeros(N), top_ids=np.zeros((N, top), np.int64), top_logp=np.zeros((N, top)))
    for i in range(N):
        z = scores[i] / temperature
        if np.all(np.isneginf(z)):
            lp = np.full(V, -np.inf)
            out["lse"][i] = -np.inf
        elif np.any(np.isnan(z)) or np.any(np.isposinf(z)):
            lp = np.full(V, np.nan)
            out["lse"][i] = out["entropy"][i] = np.nan
        else:
            m = z.max()
            log_s = np.log(np.exp(z - m).sum())
            out["lse"][i] = m + log_s
            lp = (z - m) - log_s                          # not z - lse: at |m| = 3e38 even fp64 has no room for log_s beside m
            live = ~np.isneginf(lp)
            out["entropy"][i] = -np.sum(np.exp(lp[live]) * lp[live])
        if tokens is not None and 0 <= tokens[i] < V:
            out["logp"][i] = lp[tokens[i]]
        rank = np.where(np.isnan(scores[i]), np.inf, scores[i])
        order = np.lexsort((np.arange(V), -rank, ~np.isnan(scores[i])))   # NaN first, then the larger score, then the lower id
        out["top_ids"][i] = order[:top]
        out["top_logp"][i] = lp[order[:top]]
    return out


def token_logprob_grad(scores, tokens, temperature, lse, entropy, dlogp, dentropy):
    N, V = scores.shape
    d = np.zeros((N, V))
    for i in range(N):
        if np.isneginf(lse[i]):
            continue
        lp = scores[i] / temperature - lse[i]
        p = np.exp(lp)
        if 0 <= tokens[i] < V:
            d[i] -= dlogp[i] * p
            d[i, tokens[i]] += dlogp[i]
        if dentropy is not None:
            live = p > 0
            d[i, live] -= dentropy[i] * p[live] * (lp[live] + entropy[i])
        d[i] /= temperature
    return d


def orthogonalize(x, steps, coefficients, eps, scale):
    """x (..,M,N): each matrix over its norm, then `steps` times q(X X^T) X with q(A) = a I + b A + c A A."""
    a, b, c = coefficients
    y = np.zeros(x.shape)
    for k in np.ndindex(*x.shape[:-2]):
        m = x[k] / (np.sqrt(np.sum(x[k] ** 2)) + eps)
        for _ in range(steps):
            g = m @ m.T
            m = a * m + (b * g + c * (g @ g)) @ m
        y[k] = scale * m
    return y
