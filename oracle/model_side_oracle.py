"""Definitions in fp64 of the model side of a decode step: rotary positions, a paged cache and its 8-bit form, attention of new
tokens over it, and drawing tokens.  Plain loops over sequences and heads, on float64 arrays."""
from __future__ import annotations

import numpy as np

BAD_PAGE = 256
F8_MAX = 448.0


def frequencies(rot, base=10000.0, scaling=0, factor=1.0, low=1.0, high=32.0, length=0):
    """0 plain, 1 linear, 2 ntk, 3 parts."""
    j = np.arange(rot // 2, dtype=np.float64)
    if scaling == 2 and rot > 2:
        base = base * factor ** (rot / (rot - 2.0))
    f = base ** (-2.0 * j / rot)
    if scaling == 1:
        f = f / factor
    if scaling == 3:
        r = np.clip((length * f / (2.0 * np.pi) - low) / (high - low), 0.0, 1.0)
        f = (1.0 - r) * f / factor + r * f
    return f


def turned(x, positions, freq, pairs=False, amplitude=1.0, inverse=False):
    """x [n, H, D]."""
    rot = 2 * len(freq)
    a_at, b_at = (np.arange(0, rot, 2), np.arange(1, rot, 2)) if pairs else (np.arange(rot // 2), np.arange(rot // 2, rot))
    t = np.asarray(positions, np.float64)[:, None] * freq[None, :] * (-1.0 if inverse else 1.0)
    c, s = amplitude * np.cos(t)[:, None, :], amplitude * np.sin(t)[:, None, :]
    y = x.copy()
    y[..., a_at] = x[..., a_at] * c - x[..., b_at] * s
    y[..., b_at] = x[..., b_at] * c + x[..., a_at] * s
    return y


def scale_of(x):
    """Scale of a head's columns in 8 bits, as float64."""
    top = np.abs(x).max(-1)
    s = np.maximum((top.astype(np.float32) / np.float32(F8_MAX)), np.float32(2.0 ** -126)).astype(np.float64)
    s = np.where(top == 0, 1.0, s)
    return np.where(np.isfinite(x).all(-1), s, np.nan)


def e4m3(code):
    """Values of e4m3 codes (uint8)."""
    c = code.astype(np.int64)
    e, f, sign = (c >> 3) & 15, c & 7, np.where(c & 128, -1.0, 1.0)
    v = np.where(e == 0, f * 2.0 ** -9, (8 + f) * 2.0 ** (e - 10.0))
    return np.where((c & 127) == 127, np.nan, sign * v)


def rows_of(t_offsets, n_rows, B, P):
    """[(row, b, i)] of the new tokens."""
    out = []
    for b in range(B):
        lo, hi = (b * P, b * P + P) if t_offsets is None else (t_offsets[b], t_offsets[b + 1])
        out += [(r, b, r - lo) for r in range(lo, min(hi, lo + P))]
    return out


def place(pages, b, position, page, n_pages):
    """(physical page, place in it), or None."""
    if position < 0 or position // page >= pages.shape[1]:
        return None
    at = pages[b, position // page]
    return (at, position % page) if 0 <= at < n_pages else None


def attention(q, k_cache, v_cache, lengths, pages, t_offsets, P, scale, window=0, first=None):
    """q [n_rows, Hq, D], caches [n_pages, heads, page, D], float64.  (out, lse, flags, wabs, smax) by row: wabs = sum_j w_j |v_j|,
    smax = max_j |scale| sum_d |q_d k_d|; rows of no sequence are NaN, flags -1."""
    n_rows, Hq, D = q.shape
    n_pages, heads, page, _ = k_cache.shape
    out, wabs = np.full((n_rows, Hq, D), np.nan), np.full((n_rows, Hq, D), np.nan)
    lse, smax = np.full((n_rows, Hq), np.nan), np.zeros((n_rows, Hq))
    flags = np.full(n_rows, -1)
    for r, b, i in rows_of(t_offsets, n_rows, len(lengths), P):
        cap = pages.shape[1] * page
        start = lengths[b] if 0 <= lengths[b] <= cap else cap
        p = start + i
        lo = max(0 if first is None else first[b], 0, p - window + 1 if window else 0)
        at = [place(pages, b, j, page, n_pages) for j in range(lo, p + 1)]
        flags[r] = BAD_PAGE if p >= cap or any(a is None for a in at) else 0
        if flags[r]:
            continue
        if not at:
            out[r], lse[r], wabs[r] = 0.0, -np.inf, 0.0
            continue
        pg, sl = np.array([a[0] for a in at]), np.array([a[1] for a in at])
        for h in range(Hq):
            k, v = k_cache[pg, h // (Hq // heads), sl], v_cache[pg, h // (Hq // heads), sl]
            with np.errstate(all="ignore"):
                s = scale * (k @ q[r, h])
                smax[r, h] = abs(scale) * (np.abs(k) @ np.abs(q[r, h])).max()
                if (s == -np.inf).all():
                    out[r, h], lse[r, h], wabs[r, h] = 0.0, -np.inf, 0.0
                    continue
                w = np.exp(s - s.max())
                lse[r, h] = s.max() + np.log(w.sum())
                w = w / w.sum()
                out[r, h], wabs[r, h] = w @ v, w @ np.abs(v)
    return out, lse, flags, wabs, smax


def draw(z, u, T=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, log-probability, margin) of one row of float64 logits; T, top_p, min_p as float32 holds them.  margin: how near a decision
    was to its other outcome, relative to the mass."""
    T, top_p, min_p = (float(np.float32(x)) for x in (T, top_p, min_p))
    y = z * np.log2(np.e) / T
    if np.isnan(z).any() or np.isnan(u) or not (-2.0 ** 30 <= y.max() <= 2.0 ** 30):
        return -1, np.nan, 1.0
    d = (z - z.max()) / T
    w = np.exp(d)
    keep = np.ones(len(z), bool)
    margin = 1.0
    if 0 < top_k < len(z):
        keep &= z >= np.sort(z)[-top_k]
    if top_p < 1.0:
        values = np.unique(z[keep])[::-1]
        mass = np.array([w[keep & (z == v)].sum() for v in values]) if len(values) < 64 else \
            np.bincount(np.searchsorted(-values, -z[keep]), w[keep], len(values))
        run, target = mass.cumsum(), top_p * w[keep].sum()
        n = min(int((run < target).sum()), len(values) - 1)
        margin = min(margin, np.abs(run - target).min() / run[-1])
        keep &= z >= values[n]
    if min_p > 0.0:
        margin = min(margin, np.abs(w[keep & (w < 1.0)] - min_p).min()) if (keep & (w < 1.0)).any() else margin
        keep &= w >= min_p
    w = np.where(keep, w, 0.0)
    u = min(max(u, 0.0), 1.0 - 2.0 ** -53)
    run = w.cumsum()
    t = min(int((run <= u * run[-1]).sum()), int(np.flatnonzero(w)[-1]))
    margin = min(margin, np.abs(run / run[-1] - u).min())
    return t, d[t] - np.log(run[-1]), margin
