"""Laws over a vocabulary: log-probabilities, and verification of drafted tokens.

TEST INFRASTRUCTURE ONLY (see oracle/__init__.py).

Log-probabilities of a row of logits z / T: lse = log sum_x e^{z_x / T},
log p_x = z_x / T - lse, entropy = -sum_x p_x log p_x, and the largest logits
with equal ones by the lower token.  A row of -inf alone has lse = -inf, entropy
0; a row with a NaN or +inf has no law (NaN).

Verification (Alg. 6 / Alg. 2 with categorical p_j, q_j): ell_j = log q_j(x_j) -
log p_j(x_j), log alpha_j = min(0, log alpha_{j-1} + ell_j),
    v_j = sum_x max(0, alpha_j q_{j+1}(x) - p_{j+1}(x)),
    h_j = v_j / (v_j + 1 - alpha_j) for j < K_b, h_{K_b} = alpha_{K_b},
coins c_j = [eta_j < h_j], tau = 1 + max{j : c_j = 1} (c_0 = 1), alpha_res =
alpha_{tau-1}; token verification has h_j = min(1, e^{ell_j}), tau the first
rejected draft, alpha_res = 1.  The next token is drawn from the law proportional
to max(0, alpha_res q_tau - p_tau) (tau <= K_b) or from q_{K_b+1}, by inversion
of its cumulative sums at u.

Readings: alpha_j = 1 gives h_j = 1; a draft outside the vocabulary or of target
probability 0, or with a row without a law, is rejected; where the residual has
no mass the target's law is drawn from; -1 where that has none either.
"""
import math

import numpy as np

from . import philox


def coin_uniforms(seed, chain, rnd, K):
    """eta_1..eta_K of a chain's round: the COIN stream's uniforms."""
    return np.array([philox.uniform_at(seed, chain, rnd, philox.TAG_COIN, 0, j) for j in range(K)])


def draw_uniform(seed, chain, rnd):
    """The draw's uniform: 52 bits of the first two words of the USAMPLE stream."""
    w = [int(v) for v in philox.words(seed, 0, chain, rnd, philox.TAG_USAMPLE, 0)[:2]]
    return ((w[0] >> 6) * 2.0 ** 26 + (w[1] >> 6) + 0.5) * 2.0 ** -52


def row_law(z, T=1.0):
    """log p of one row in float64 (None: no law), all -inf where the mask leaves nothing."""
    z = np.asarray(z, np.float64)
    if np.isnan(z).any() or np.isposinf(z).any():
        return None
    m = z.max()
    if m == -np.inf:
        return np.full(z.shape, -np.inf)
    d = (z - m) / T
    return d - np.log(np.exp(d).sum())


def logprobs(z, tokens=None, n_top=0, T=1.0):
    """lse, entropy, logprob [n_tok], top_ids, top_logprobs of one row."""
    z = np.asarray(z, np.float64)
    V = z.shape[0]
    tokens = [] if tokens is None else tokens
    lp = row_law(z, T)
    if lp is None:
        nan = float("nan")
        return dict(lse=nan, entropy=nan, logprob=np.full(len(tokens), nan), top_ids=np.full(n_top, -1),
                    top_logprobs=np.full(n_top, nan))
    m = z.max()
    none = m == -np.inf
    lse = -np.inf if none else m / T + np.log(np.exp((z - m) / T).sum())
    p = np.exp(lp)
    order = np.lexsort((np.arange(V), -z))[:n_top]
    ids, top = np.full(n_top, -1), np.full(n_top, -np.inf)
    ids[: len(order)], top[: len(order)] = order, lp[order]
    return dict(lse=lse, entropy=0.0 if none else -float((p[p > 0] * lp[p > 0]).sum()),
                logprob=np.array([lp[t] if 0 <= t < V else -np.inf for t in tokens]), top_ids=ids, top_logprobs=top)


def draw(w, u):
    """The lowest x whose cumulative sum of w exceeds u times the whole."""
    c = np.cumsum(w)
    hit = np.nonzero(c > u * c[-1])[0]
    return int(hit[0]) if len(hit) else int(np.nonzero(w > 0)[0][-1])


def verify_chain(draft, target, x, kb, eta, u, mode="block", T=1.0):
    """One chain: draft [K][V], target [K+1][V] logits, x [K] tokens, eta [K], u.

    Returns dict tau, token, log_alpha_res, ell [kb], h [kb], coins (bitmask), w (the drawn weights or None).
    """
    if kb <= 0:
        return dict(tau=0, token=-1, log_alpha_res=0.0, ell=np.zeros(0), h=np.zeros(0), coins=0, w=None)
    V = len(target[0])
    q = [row_law(target[j], T) for j in range(kb + 1)]
    p = [row_law(draft[j], T) for j in range(kb)]
    ell = np.empty(kb)
    for j in range(kb):
        if q[j] is None or p[j] is None:
            ell[j] = np.nan
            continue
        known = 0 <= x[j] < V
        lq, lp = (q[j][x[j]], p[j][x[j]]) if known else (-np.inf, -np.inf)
        ell[j] = -np.inf if lq == -np.inf else lq - lp
    la = [0.0]
    for j in range(kb):
        e = ell[j] if ell[j] == ell[j] else -np.inf
        la.append(-np.inf if la[-1] == -np.inf else min(0.0, la[-1] + e))
    h = np.empty(kb)
    coins = 0
    for j in range(1, kb + 1):
        if mode == "token":
            e = ell[j - 1]
            h[j - 1] = math.exp(min(0.0, e)) if e == e else 0.0
        elif j == kb:
            h[j - 1] = math.exp(la[j])
        elif la[j] >= 0.0:
            h[j - 1] = 1.0
        elif q[j] is None or p[j] is None:
            h[j - 1] = 0.0
        else:
            v = np.maximum(0.0, np.exp(q[j] + la[j]) - np.exp(p[j])).sum()
            h[j - 1] = v / (v - math.expm1(la[j]))
        if eta[j - 1] < h[j - 1]:
            coins |= 1 << (j - 1)
    if mode == "token":
        tau = next((j for j in range(1, kb + 1) if not coins >> (j - 1) & 1), kb + 1)
        res = 0.0
    else:
        tau = coins.bit_length() + 1
        res = la[tau - 1]
    lq = q[tau - 1]
    lp = p[tau - 1] if tau <= kb else np.full(V, -np.inf)
    if lq is None or lp is None or lq.max() == -np.inf:
        return dict(tau=tau, token=-1, log_alpha_res=res, ell=ell, h=h, coins=coins, w=None)
    w = np.maximum(0.0, np.exp(lq + res) - np.exp(lp))
    if not w.sum() > 0:
        w = np.exp(lq)
    return dict(tau=tau, token=draw(w, u), log_alpha_res=res, ell=ell, h=h, coins=coins, w=w)
