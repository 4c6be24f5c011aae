"""Serving over paged caches in float64, from the formulas: rotary positions, attention of one row per sequence, eviction by weight, log-probabilities."""
import math

import numpy as np


def rope_frequencies(rot, theta=10000.0, scaling="none", factor=1.0, low=1.0, high=4.0, original=8192):
    if scaling == "base":
        theta = theta * factor ** (rot / (rot - 2))
    w = theta ** (-2.0 * np.arange(rot // 2) / rot)
    if scaling in ("none", "base"):
        return w
    if scaling == "linear":
        keep = np.zeros_like(w)
    elif scaling == "bands":
        keep = (original * w / (2 * np.pi) - low) / (high - low)
    else:
        lo, hi = (rot * math.log(original / (n * 2 * np.pi)) / (2 * math.log(theta)) for n in (high, low))
        lo, hi = max(0, math.floor(lo)), min(rot - 1, math.ceil(hi))
        keep = 1 - (np.arange(rot // 2) - lo) / max(hi - lo, 1e-3)
    keep = np.clip(keep, 0, 1)
    return keep * w + (1 - keep) * w / factor


def rotate(x, positions, w, interleaved=False, magnitude=1.0, inverse=False):
    """x [rows, heads, dim] as complex numbers times magnitude * e^(i position w)."""
    r = 2 * len(w)
    a, b = (slice(0, r, 2), slice(1, r, 2)) if interleaved else (slice(0, r // 2), slice(r // 2, r))
    z = (x[..., a] + 1j * x[..., b]) * (magnitude * np.exp((-1j if inverse else 1j) * np.asarray(positions, np.float64)[:, None, None] * w))
    y = np.array(x, np.float64)
    y[..., a], y[..., b] = z.real, z.imag
    return y


def gather(pool, table, length, page_tokens, values=False):
    """One sequence's first `length` slots from pages [page][head][place][dim] (values: [page][head][dim][place]): [heads, length, dim]."""
    pool = pool.swapaxes(2, 3) if values else pool
    n = -(-length // page_tokens)
    return pool[table[:n]].swapaxes(0, 1).reshape(pool.shape[1], n * page_tokens, pool.shape[3])[:, :length]


def attend(q, k, v, scale):
    """q [heads, dim] over k, v [kv_heads, slots, dim]: (out, lse, probabilities [heads, slots], scores)."""
    heads, dim = q.shape
    g = heads // k.shape[0]
    if k.shape[1] == 0:
        return np.zeros((heads, dim)), np.full(heads, -np.inf), np.zeros((heads, 0)), np.zeros((heads, 0))
    s = np.stack([k[h // g] @ q[h] for h in range(heads)]) * scale
    m = s.max(axis=1, keepdims=True)
    e = np.exp(s - m)
    p = e / e.sum(axis=1, keepdims=True)
    return np.stack([p[h] @ v[h // g] for h in range(heads)]), m[:, 0] + np.log(e.sum(axis=1)), p, s


def evict(weights, positions, length, budget, first, recent):
    """One head's slots: the former slot of each that is left (list)."""
    length = min(max(int(length), 0), len(weights))
    if length <= budget:
        return list(range(length))
    newest = max(int(p) for p in positions[:length])

    def order(i):
        p, w = int(positions[i]), float(weights[i])
        if p < first or p > newest - recent:
            return (0, 0.0, i)
        return (2, 0.0, i) if math.isnan(w) else (1, -w, i)
    keep = set(sorted(range(length), key=order)[:budget])
    above = iter(sorted(i for i in keep if i >= budget))
    return [i if i in keep else next(above) for i in range(budget)]


def logprobs(x, temperature=1.0):
    """(log-probabilities [rows, vocab], entropy [rows]) of logits; a row that has no distribution is NaN."""
    with np.errstate(all="ignore"):
        z = np.asarray(x, np.float64) / temperature
        m = z.max(axis=1, keepdims=True)
        e = np.exp(z - m)
        lp = z - m - np.log(e.sum(axis=1, keepdims=True))
        lp[~np.isfinite(m[:, 0])] = np.nan
        p = np.exp(lp)
        return lp, -np.where(p == 0, 0.0, p * lp).sum(axis=1)


def best(row, n):
    """Ids of the n largest of a row, equal ones by the lowest, NaN last."""
    return sorted(range(len(row)), key=lambda i: (1, 0.0, i) if np.isnan(row[i]) else (0, -float(row[i]), i))[:n]
