"""Definitions in fp64 of the operators around the decode step: log-probabilities of given tokens
with their gradient, embedding rows with theirs, gradient norm and clipping.

Logits are float32 arrays or uint16 bit patterns of bfloat16, as in `sv_oracle`.
"""
from __future__ import annotations

import numpy as np

FLOOR = -(2.0 ** 30)               # entries with z log2(e) / T below it carry no mass
BAD_ROW, BAD_TOKEN = 1, 16


def values(z):
    """Stored numbers as float64 (uint16: bfloat16 bit patterns)."""
    if z.dtype == np.uint16:
        z = (z.astype(np.uint32) << 16).view(np.float32)
    return z.astype(np.float64)


def to_bf16(x):
    """float64 -> float64 holding the nearest bfloat16 (ties to even), through float32 as the kernels do."""
    u = np.asarray(x, dtype=np.float32).view(np.uint32)
    r = ((u + 0x7FFF + ((u >> 16) & 1)) >> 16 << 16).astype(np.uint32)
    return np.where(np.isnan(x), np.nan, r.view(np.float32)).astype(np.float64)


def within(got, ref, tol, bf16):
    """Whether stored results are ref to within tol before their one rounding to bfloat16 (if any)."""
    lo, hi = ref - tol, ref + tol
    if bf16:
        lo, hi = to_bf16(lo), to_bf16(hi)
    return (got >= lo) & (got <= hi)


def log_probs(z, T):
    """(log p, lse) of one row of stored logits; lse is NaN for a bad row."""
    z = values(z)
    y = z / T
    has = y * np.log2(np.e) >= FLOOR
    if np.isnan(z).any() or np.isposinf(z).any() or not has.any() or (y[has] * np.log2(np.e)).max() > -FLOOR:
        return np.full(z.shape, np.nan), np.nan
    y = np.where(has, y, -np.inf)
    m = y.max()
    lse = m + np.log(np.exp(y - m).sum())
    return y - lse, lse


def entropy_of(lp):
    p = np.exp(lp)
    return -(p * np.where(p > 0, lp, 0.0)).sum()


def token_logprobs(z, tokens, T=1.0, n_top=0):
    """z [N, V] stored logits; tokens [N] (-1: none) or None.  Dict of [N] arrays and top_* [N, n_top]."""
    N, V = z.shape
    out = dict(logprob=np.zeros(N), lse=np.zeros(N), entropy=np.zeros(N), rank=np.zeros(N, np.int64),
               top_token=np.full((N, n_top), -1), top_logprob=np.full((N, n_top), -np.inf),
               flags=np.zeros(N, np.int64))
    for r in range(N):
        t = None if tokens is None else int(tokens[r])
        if t == -1:
            continue
        lp, lse = log_probs(z[r], T)
        if np.isnan(lse):
            for k in ("logprob", "lse", "entropy", "top_logprob"):
                out[k][r] = np.nan
            out["flags"][r] = BAD_ROW
            continue
        out["lse"][r], out["entropy"][r] = lse, entropy_of(lp)
        order = np.lexsort((np.arange(V), -values(z[r])))
        if t is not None and 0 <= t < V:
            out["logprob"][r] = lp[t]
            out["rank"][r] = 1 + int(np.nonzero(order == t)[0][0])
        elif t is not None:
            out["logprob"][r], out["flags"][r] = np.nan, BAD_TOKEN
        best = [v for v in order[:n_top] if lp[v] > -np.inf]
        out["top_token"][r, :len(best)] = best
        out["top_logprob"][r, :len(best)] = lp[best]
    return out


def token_logprobs_grad(z, tokens, g, h=None, T=1.0):
    """Gradient of sum(g logprob + h entropy): dict(logprob, entropy, dz, p) in float64."""
    N, V = z.shape
    out = dict(logprob=np.zeros(N), entropy=np.zeros(N), dz=np.zeros((N, V)), p=np.zeros((N, V)),
               flags=np.zeros(N, np.int64))
    h = np.zeros(N) if h is None else h
    for r in range(N):
        t = int(tokens[r])
        if t == -1:
            continue
        lp, lse = log_probs(z[r], T)
        bad = np.isnan(lse)
        given = 0 <= t < V
        out["flags"][r] = (BAD_ROW if bad else 0) | (0 if given else BAD_TOKEN)
        out["entropy"][r] = np.nan if bad else entropy_of(lp)
        out["logprob"][r] = lp[t] if given else np.nan
        if bad or not given:
            out["dz"][r] = np.nan
            continue
        p = np.exp(lp)
        one = np.zeros(V)
        one[t] = 1.0
        plp = p * np.where(p > 0, lp, 0.0)
        out["dz"][r] = (float(g[r]) * (one - p) - float(h[r]) * (plp + p * out["entropy"][r])) / T
        out["p"][r] = p
    return out


def embedding(table, ids, scale):
    V = table.shape[0]
    out = np.zeros((len(ids), table.shape[1]))
    for i, t in enumerate(ids):
        if 0 <= t < V:
            out[i] = values(table[t]) * scale
    return out


def embedding_grad(grad_out, ids, V, scale, old=None):
    """(gradient, sum of absolute values of what was added, number of rows added)"""
    D = grad_out.shape[1]
    s, a, c = np.zeros((V, D)), np.zeros((V, D)), np.zeros(V, np.int64)
    g = values(grad_out)
    for i, t in enumerate(ids):
        if 0 <= t < V:
            s[t] += g[i]
            a[t] += np.abs(g[i])
            c[t] += 1
    s, a = s * scale, a * abs(scale)
    if old is not None:
        s, a = s + old, a + np.abs(old)
    return s, a, c


def grad_norm(grads):
    return np.sqrt(sum((values(g) ** 2).sum() for g in grads))


def clip_factor(norm, max_norm):
    return min(1.0, max_norm / (norm + 1e-6)) if np.isfinite(norm) else 1.0
