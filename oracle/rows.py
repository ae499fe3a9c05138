"""Reference for the operators on rows of logits (TEST INFRASTRUCTURE ONLY): first entries, filtered sampling, distillation.

Plain numpy fp64 on the exact input values, one row at a time; nothing shared with the GPU library.  A row's entries stand in
the order (logit descending, index ascending); NaN and minus infinity are masked.
"""
from __future__ import annotations

import numpy as np

F32_MAX = float(np.finfo(np.float32).max)                     # where scaled logits of unmasked entries stop
REST_IS_NONE = -2.0 ** 28 * np.log(2.0)                       # scaled logits below this are masks: no mass outside a student's entries


def in_order(x: np.ndarray) -> np.ndarray:
    """Indices of the unmasked entries of x [V], in order."""
    there = np.flatnonzero(x > -np.inf)                       # (false for NaN)
    return there[np.argsort(-x[there], kind="stable")]


def lse(z: np.ndarray) -> float:
    z = z[z > -np.inf]
    return float(z.max() + np.log(np.exp(z - z.max()).sum())) if z.size else -np.inf


def top(x: np.ndarray, K: int, inv_temp: float):
    """values [K], index [K], log-sum-exp of x * inv_temp; (-inf, -1) where there are fewer."""
    o = in_order(x)[:K]
    values, index = np.full(K, -np.inf), np.full(K, -1, dtype=np.int64)
    values[:o.size], index[:o.size] = x[o], o
    z = np.where(np.isnan(x), -np.inf, x) * inv_temp
    return values, index, lse(np.where(np.isfinite(x), np.clip(z, -F32_MAX, F32_MAX), z))


def keep(x: np.ndarray, inv_temp: float = 1.0, top_k: int = 0, top_p: float = 1.0, min_p: float = 0.0):
    """(kept indices in order, scaled logits z [V]): top-k, then top-p of their mass, then min-p of the largest probability."""
    if inv_temp > np.float32(1e30):                           # the first entry alone
        inv_temp, top_k = 1.0, 1
    z = np.where(x > -np.inf, np.clip(x * inv_temp, -F32_MAX, F32_MAX), -np.inf)
    o = in_order(x)
    if 1 <= top_k < x.size:
        o = o[:top_k]
    if o.size == 0:
        return o, z
    if top_p < 1.0:
        c = np.cumsum(np.exp(z[o] - z[o[0]]))
        o = o[:1 + int(np.searchsorted(c, top_p * c[-1], side="left"))]
    if min_p > 0.0:
        o = o[np.exp(z[o] - z[o[0]]) >= min(min_p, 1.0)]
    return o, z


def probabilities(x: np.ndarray, **how) -> np.ndarray:
    o, z = keep(x, **how)
    p = np.zeros(x.size)
    if o.size:
        e = np.exp(z[o] - z[o[0]])
        p[o] = e / e.sum()
    return p


def draw(p: np.ndarray, u: float):
    """(token, how far u lies from the nearest border of the tokens' intervals): the first whose cumulative mass exceeds u."""
    c = np.cumsum(p)
    total = c[-1]
    if not total > 0:
        return -1, 1.0
    c = c / total
    with_mass = np.flatnonzero(p > 0)
    at = int(np.searchsorted(c, u, side="right"))
    return (at if at < p.size else int(with_mass[-1])), float(np.abs(c[with_mass] - u).min())


def distill(z: np.ndarray, top_val, top_idx, top_lse, label: int, inv_temp: float, kl_weight: float, ce_weight: float, dloss: float = 1.0):
    """(kl, ce, gradient [V]) of one row; top_lse None: the entries' own soft-max."""
    V = z.size
    s_log = z * inv_temp - lse(z * inv_temp)
    s = np.exp(s_log)
    there = (top_idx >= 0) & (top_idx < V)
    i, t = top_idx[there], top_val[there].astype(np.float64) * inv_temp
    kl, ce, g = 0.0, 0.0, np.zeros(V)
    if i.size:
        log_p = t - (lse(t) if top_lse is None else top_lse)
        p = np.exp(log_p)
        kl = float((p * (log_p - s_log[i])).sum())
        dist = np.zeros(V)
        np.add.at(dist, i, p)
        outside = np.ones(V, dtype=bool)
        outside[i] = False
        g = s * p.sum() - dist
        if top_lse is not None:
            p_rest, rest = 1.0 - p.sum(), np.where(outside, z * inv_temp, -np.inf)
            log_rest = lse(rest)                              # (of the student's mass outside the entries, however small that is)
            if p_rest > 0 and log_rest > REST_IS_NONE:
                kl += float(p_rest * (np.log(p_rest) - log_rest + lse(z * inv_temp)))
                g = s - dist - p_rest * np.exp(rest - log_rest)
            elif p_rest > 4e-5 + 2.0 ** -22 * abs(top_lse):   # (less is what a log-sum-exp in 32 bits leaves)
                kl, g = np.inf, s - dist
        g *= inv_temp
    g = kl_weight * g
    if 0 <= label < V:
        ce = float(lse(z) - z[label])
        d = np.exp(z - lse(z))
        d[label] -= 1.0
        g = g + ce_weight * d
    return kl, ce, g * dloss
