"""Trees of drafted tokens: positions, who sees whom, the rotation, verification, the kept branch.

TEST INFRASTRUCTURE ONLY (see oracle/__init__.py).

Node 0 is the root; parents[i] in [0, i) is node i's parent, any other value none.
Verification walks from the root: a node's children x_0, x_1, .. are tried in order,
    r_0 = q,  x_k accepted if eta < r_k(x_k) / p_k(x_k),  else r_{k+1} = norm(max(0, r_k - p_k)),
p_k the draft law ("iid"), the draft law without x_0 .. x_{k-1} ("distinct") or all on x_k
("given"); where none is accepted the next token is drawn from the last r.
"""
import numpy as np

from .tokens import draw, row_law


def parent_of(parents, i):
    return int(parents[i]) if 0 <= int(parents[i]) < i else -1


def depth(parents, i):
    d = 0
    while parent_of(parents, i) >= 0:
        i, d = parent_of(parents, i), d + 1
    return d


def sees(parents, n):
    """[n][n]: whether node i sees node j (itself and its ancestors)."""
    m = np.eye(n, dtype=bool)
    for i in range(n):
        j = parent_of(parents, i)
        while j >= 0:
            m[i, j] = True
            j = parent_of(parents, j)
    return m


def rotate(x, pos, freq, halves):
    """The pairs of x [..][d] turned by pos * freq."""
    x = np.asarray(x, np.float64)
    a = np.float64(pos) * np.asarray(freq, np.float64)
    half = x.shape[-1] // 2
    u, v = (x[..., :half], x[..., half:]) if halves else (x[..., ::2], x[..., 1::2])
    s, t = u * np.cos(a) - v * np.sin(a), u * np.sin(a) + v * np.cos(a)
    return np.concatenate([s, t], -1) if halves else np.stack([s, t], -1).reshape(x.shape)


def tries(q, p, xs, draws, ell=None):
    """For every child of a node in order: h, and the law that is left if it is rejected.

    q, p: probabilities (p None: given); ell: log q - log p, where that is more than the quotient of the two (both
    may be too small for float64).  Yields (h, ratio r_k / p_k, a, S, r after a rejection); a and S are those of
    r = max(0, q - a p) / S.
    """
    r, p = q.copy(), None if p is None else p.copy()
    a, S, rest, tried = 0.0, 1.0, 1.0, []
    for x in xs:
        known = 0 <= x < len(q)
        if not known or (draws != "iid" and x in tried):
            yield 0.0, 0.0, a, S, r.copy()
            continue
        if p is None:
            ratio, left = r[x], np.where(np.arange(len(q)) == x, 0.0, r)
        else:
            if rest == 0 or (p[x] == 0 and ell is None):
                ratio = np.inf if r[x] > 0 else 0.0
            elif p[x] > 0:
                ratio = r[x] / p[x]
            elif ell[x] == np.inf:
                ratio = np.inf if r.sum() > 0 else 0.0
            else:
                ratio = max(0.0, np.exp(min(ell[x], 700.0)) - a) * rest / S if S > 0 and ell[x] > -np.inf else 0.0
            left = np.maximum(r - p, 0.0)
        if rest > 0:  # (nothing of p is left to be subtracted otherwise)
            a, S, r = a + S / rest, S * left.sum(), left / left.sum() if left.sum() > 0 else left
        tried.append(x)
        yield min(ratio, 1.0), ratio, a, S, r.copy()
        if draws == "distinct":
            p[x] = 0.0
            rest *= p.sum()
            p = p / p.sum() if p.sum() > 0 else p


def verify(draft, target, tokens, parents, n, eta, u, draws, max_children=None, T=1.0):
    """One tree: draft (None: given), target [Q][V] logits, eta[i] the coin of node i, u the draw's uniform.

    Returns dict tau, token, path, accept {node: h}, w (the law that was drawn from, None without one).
    """
    if n <= 0:
        return dict(tau=0, token=-1, path=[], accept={}, w=None)
    path, accept, node = [0], {}, 0
    while True:
        kids = [i for i in range(node + 1, n) if parent_of(parents, i) == node][:max_children]
        lq = row_law(target[node], T)
        lp = row_law(draft[node], T) if draft is not None and kids else np.full(len(target[node]), -np.inf)
        if lq is None or lp is None or lq.max() == -np.inf:
            # no law: every child is rejected, and nothing is left to draw from
            accept.update({i: 0.0 for i in kids})
            return dict(tau=len(path), token=-1, path=path, accept=accept, w=None)
        r = q = np.exp(lq)
        taken = None
        with np.errstate(invalid="ignore"):
            ell = lq - lp
        laws = tries(q, None if draft is None else np.exp(lp), [tokens[k] for k in kids], draws, ell)
        for i, (h, _, _, _, left) in zip(kids, laws):
            accept[i] = h
            if eta[i] < h:
                taken = i
                break
            r = left
        if taken is None:
            w = r if r.sum() > 0 else q
            return dict(tau=len(path), token=draw(w, u), path=path, accept=accept, w=w)
        path.append(taken)
        node = taken


def keep(cache, table, first, path, tau, n):
    """One sequence's accepted branch moved up behind its first `first` tokens (cache [pages][size][d], in place).

    Returns the sequence's new length."""
    size, kept = cache.shape[1], 0

    def at(j):
        page = int(table[j // size]) if 0 <= j < len(table) * size else -1
        return (page, j % size) if 0 <= page < len(cache) else None

    last = -1
    for j in range(min(max(tau, 0), n)):
        v = int(path[j])
        if v <= last or v >= n:
            break
        last, kept = v, kept + 1
        if at(first + v) and at(first + j):
            cache[at(first + j)] = cache[at(first + v)]
    return max(first + kept, 0)
