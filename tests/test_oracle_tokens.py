"""The token oracle against what defines it: enumerated laws on tiny vocabularies.

Block and token verification are lossless: with drafts from p and the residual
draw, the first accepted-or-drawn token follows q_1, and the whole block's law is
that of the target (Alg. 6's and Alg. 2's exactness), checked by summing over
every draft and integrating the uniforms exactly.
"""
import itertools
import math

import numpy as np
import pytest

from oracle import philox, tokens as otok


def _tables(V, K, seed):
    """p and q for every prefix: logits [prefix] -> [V]."""
    g = np.random.default_rng(seed)
    t = {}
    for n in range(K + 1):
        for pre in itertools.product(range(V), repeat=n):
            t[pre] = (g.normal(size=V) * 1.2, g.normal(size=V) * 1.2)
    return t


def _block_law(t, V, K, mode):
    """The law of the first token that a round emits, and of the first two where it emits two or more."""
    one = np.zeros(V)
    for x in itertools.product(range(V), repeat=K):
        draft = [t[x[:j]][0] for j in range(K)]
        target = [t[x[:j]][1] for j in range(K + 1)]
        px = math.exp(sum(otok.row_law(draft[j])[x[j]] for j in range(K)))
        r = otok.verify_chain(draft, target, x, K, np.full(K, 2.0), 0.5, mode)
        h = r["h"]
        for c in itertools.product((0, 1), repeat=K):  # the coins' outcomes, each with its probability
            pc = np.prod([h[j] if c[j] else 1.0 - h[j] for j in range(K)])
            if pc == 0.0:
                continue
            eta = [0.5 * h[j] if c[j] else 0.5 * (1.0 + h[j]) for j in range(K)]
            s = otok.verify_chain(draft, target, x, K, eta, 0.5, mode)
            if s["tau"] > 1:
                one[x[0]] += px * pc
            else:
                one += px * pc * s["w"] / s["w"].sum()
    return one


@pytest.mark.parametrize("mode", ["block", "token"])
@pytest.mark.parametrize("V,K,seed", [(3, 1, 0), (2, 3, 1), (3, 3, 2), (4, 2, 3)])
def test_first_token_follows_the_target(V, K, seed, mode):
    t = _tables(V, K, seed)
    np.testing.assert_allclose(_block_law(t, V, K, mode), np.exp(otok.row_law(t[()][1])), rtol=1e-12)


def test_block_accepts_at_least_as_many():
    V, K = 3, 3
    for seed in range(4):
        t = _tables(V, K, seed)
        mean = {}
        for mode in ("block", "token"):
            mean[mode] = 0.0
            for x in itertools.product(range(V), repeat=K):
                draft = [t[x[:j]][0] for j in range(K)]
                target = [t[x[:j]][1] for j in range(K + 1)]
                px = math.exp(sum(otok.row_law(draft[j])[x[j]] for j in range(K)))
                h = otok.verify_chain(draft, target, x, K, np.full(K, 2.0), 0.5, mode)["h"]
                for c in itertools.product((0, 1), repeat=K):
                    pc = np.prod([h[j] if c[j] else 1.0 - h[j] for j in range(K)])
                    if mode == "block":
                        tau = 1 + max([j + 1 for j in range(K) if c[j]], default=0)
                    else:
                        tau = next((j + 1 for j in range(K) if not c[j]), K + 1)
                    mean[mode] += px * pc * tau
        assert mean["block"] >= mean["token"] - 1e-12


def test_draw_inverts_the_cumulative_sums():
    w = np.array([0.0, 0.25, 0.0, 0.5, 0.25, 0.0])
    assert [otok.draw(w, u) for u in (1e-9, 0.2499, 0.25, 0.7, 0.75, 1 - 1e-12)] == [1, 1, 3, 3, 4, 4]


def test_logprobs_of_degenerate_rows():
    inf = np.inf
    r = otok.logprobs(np.full(4, -inf), [0, 9], 3)
    assert r["lse"] == -inf and r["entropy"] == 0.0 and list(r["top_ids"]) == [0, 1, 2] and (r["logprob"] == -inf).all()
    r = otok.logprobs(np.array([1.0, inf, 0.0]), [0], 2)
    assert math.isnan(r["lse"]) and list(r["top_ids"]) == [-1, -1]
    r = otok.logprobs(np.array([2.0, 1.0, 2.0]), [1, -1], 5)
    assert list(r["top_ids"]) == [0, 2, 1, -1, -1] and r["logprob"][1] == -inf
    r = otok.logprobs(np.zeros(8), [3], 0, T=0.5)
    assert abs(r["entropy"] - math.log(8)) < 1e-14 and abs(r["logprob"][0] + math.log(8)) < 1e-14


def test_uniforms_lie_inside_the_unit_interval():
    for w0, w1 in ((0, 0), (0xFFFFFFFF, 0xFFFFFFFF)):
        u = ((w0 >> 6) * 2.0 ** 26 + (w1 >> 6) + 0.5) * 2.0 ** -52
        assert 0.0 < u < 1.0
    u = np.array([otok.draw_uniform(5, b, r) for b in range(40) for r in range(10)])
    assert 0.0 < u.min() and u.max() < 1.0 and abs(u.mean() - 0.5) < 5 / math.sqrt(12 * u.size)
    e = otok.coin_uniforms(5, 1, 2, 7)
    assert e.shape == (7,) and e[6] == philox.uniform_at(5, 1, 2, philox.TAG_COIN, 0, 6)
