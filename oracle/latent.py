"""Attention over one shared latent vector a token, absorbed and expanded forms.

TEST INFRASTRUCTURE ONLY (see oracle/__init__.py).

Absorbed: the key of a cached vector c is all of it, its value the first d_latent
elements; row i of the n rows of a sequence of len tokens sees tokens j < len - n
+ i + 1.  Expanded: per-head keys (k_nope, and the rotary part that the heads
share) and values; query i of n sees keys j < m - n + i + 1 of m.  In both
    s_j = scale q . k_j,  lse = log sum_j e^{s_j},  out = sum_j e^{s_j - lse} v_j,
and a row that sees nothing has out 0, lse -inf.
"""
import numpy as np


def attend(q, k, v, scale, limits):
    """q [r][d], k [t][d], v [t][e] float64; row i sees k[:limits[i]].  Returns out [r][e], lse [r], and
    sum_j |p_j v_j| [r][e] (what roundings of the weights scale with)."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    out, mag = np.zeros((len(q), v.shape[1])), np.zeros((len(q), v.shape[1]))
    lse = np.full(len(q), -np.inf)
    for i, n in enumerate(limits):
        n = max(0, min(int(n), len(k)))
        if n == 0:
            continue
        with np.errstate(invalid="ignore", over="ignore"):
            s = scale * (k[:n] @ q[i])
            m = s.max()
            if np.isnan(m) or m == np.inf:
                out[i], lse[i], mag[i] = np.nan, np.nan, np.nan
                continue
            p = np.exp(s - m)
            lse[i] = m + np.log(p.sum())
            p /= p.sum()
            out[i], mag[i] = p @ v[:n], p @ np.abs(v[:n])
    return out, lse, mag


def gather(cache, pages, length):
    """The vectors of one sequence's tokens from its pages, and which of them exist."""
    size = cache.shape[1]
    j = np.arange(length)
    page = np.asarray(pages)[j // size]
    have = (page >= 0) & (page < len(cache))
    return cache[np.where(have, page, 0), j % size], have
