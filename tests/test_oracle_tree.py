"""The tree oracle against what defines it: the next token follows the target's law, whatever
is drafted; the rest after k rejections is max(0, q - a_k p) / S_k; rotations."""
import itertools

import numpy as np
import pytest

from oracle import tree


def _laws(V, seed):
    r = np.random.default_rng(seed)
    return r.dirichlet(np.ones(V) * 0.7), r.dirichlet(np.ones(V) * 0.7)


def _drawn(p, m, draws):
    """All tuples of m children with their probabilities."""
    for xs in itertools.product(range(len(p)), repeat=m):
        if draws == "iid":
            yield xs, np.prod([p[x] for x in xs])
        elif len(set(xs)) == m:
            w, rest = 1.0, 1.0
            for x in xs:
                w *= p[x] / rest
                rest -= p[x]
            yield xs, w


@pytest.mark.parametrize("draws", ["iid", "distinct"])
@pytest.mark.parametrize("m", [1, 2, 3])
def test_the_next_token_follows_the_targets_law(draws, m):
    V = 4
    for seed in range(5):
        q, p = _laws(V, seed)
        law = np.zeros(V)
        for xs, w in _drawn(p, m, draws):
            alive = w
            for x, (h, _, _, _, left) in zip(xs, tree.tries(q, p, xs, draws)):
                law[x] += alive * h
                alive *= 1 - h
            law += alive * left
        assert np.abs(law - q).max() < 1e-12


def test_given_candidates_leave_the_law_whole():
    q, _ = _laws(5, 3)
    for xs in ([2], [2, 0], [4, 1, 1, 0, 9], [0, 1, 2, 3]):
        law, alive = np.zeros(5), 1.0
        for x, (h, _, _, _, left) in zip(xs, tree.tries(q, None, xs, "given")):
            if h > 0:
                law[x] += alive * h
            alive *= 1 - h
        assert np.abs(law + alive * left - q).max() < 1e-12


def test_what_is_left_after_k_independent_tries():
    q, p = _laws(30, 8)
    for h, ratio, a, S, left in tree.tries(q, p, [3] * 5, "iid"):
        w = np.maximum(q - a * p, 0.0)
        assert abs(w.sum() - S) < 1e-12 and np.abs(left - w / w.sum()).max() < 1e-12


def test_draws_without_replacement_share_the_form():
    # a_{k+1} = a_k + S_k / rest_k, for every x that was rejected where its ratio is below 1
    q = np.array([0.05, 0.05, 0.3, 0.2, 0.4])
    p = np.array([0.5, 0.3, 0.1, 0.06, 0.04])
    a, S, rest = 0.0, 1.0, 1.0
    for x, (h, ratio, _, _, left) in zip((0, 1), tree.tries(q, p, (0, 1), "distinct")):
        assert h < 1 and abs(h - max(0.0, q[x] / p[x] - a) * rest / S) < 1e-12
        a += S / rest
        rest -= p[x]
        S = np.maximum(q - a * p, 0.0).sum()
        assert np.abs(left - np.maximum(q - a * p, 0.0) / S).max() < 1e-12


def test_a_walk():
    """Two levels: the first child of the root is refused, the second taken, and its own child refused."""
    V = 3
    target = np.log(np.array([[0.2, 0.5, 0.3], [1, 1, 1], [0.1, 0.1, 0.8], [1, 1, 1]], float))
    draft = np.log(np.array([[0.6, 0.2, 0.2], [1, 1, 1], [0.5, 0.25, 0.25], [1, 1, 1]], float))
    parents, tokens = [-1, 0, 0, 2], [0, 0, 1, 0]
    r = tree.verify(draft, target, tokens, parents, 4, [0, 0.9, 0.5, 0.9], 0.5, "iid")
    # r_1 = (0, 0.3, 0.1) / 0.4, r_1 / p of token 1 is 3.75
    assert r["path"] == [0, 2] and r["tau"] == 2 and abs(r["accept"][1] - 1 / 3) < 1e-12 and r["accept"][2] == 1.0
    assert abs(r["accept"][3] - 0.2) < 1e-12 and np.abs(r["w"] - [0, 0, 1]).max() < 1e-12 and r["token"] == 2
    # at most one child of a node: the root's second is not tried
    r = tree.verify(draft, target, tokens, parents, 4, [0, 0.9, 0.5, 0.9], 0.5, "iid", max_children=1)
    assert r["path"] == [0] and set(r["accept"]) == {1}


def test_nodes_without_a_parent_see_themselves_alone():
    parents = [7, 0, 2, -1, 1, 9]
    m = tree.sees(parents, 6)
    assert [list(np.nonzero(r)[0]) for r in m] == [[0], [0, 1], [2], [3], [0, 1, 4], [5]]
    assert [tree.depth(parents, i) for i in range(6)] == [0, 1, 0, 0, 2, 0]


@pytest.mark.parametrize("halves", [False, True])
def test_rotations_keep_lengths_and_differences_of_positions(halves):
    r = np.random.default_rng(1)
    x, y, f = r.standard_normal(16), r.standard_normal(16), 10000.0 ** (-np.arange(8) / 8)
    a, b = tree.rotate(x, 905, f, halves), tree.rotate(y, 900, f, halves)
    assert abs(np.linalg.norm(a) - np.linalg.norm(x)) < 1e-12
    assert abs(a @ b - tree.rotate(x, 5, f, halves) @ y) < 1e-9
    assert np.abs(tree.rotate(x, 0, f, halves) - x).max() == 0


def test_keep_moves_in_order_and_ends_where_the_path_does_not_rise():
    cache = np.arange(24.0).reshape(3, 4, 2)
    before, table = cache.copy(), [2, 0, -1]
    assert tree.keep(cache, table, 2, [0, 2, 3, -1], 3, 5) == 5
    assert (cache[2, 3] == before[0, 0]).all() and (cache[0, 0] == before[0, 1]).all() and (cache[2, 2] == before[2, 2]).all()
    assert tree.keep(before.copy(), table, 2, [0, 2, 2, 4], 4, 5) == 4
    assert tree.keep(before.copy(), table, 2, [1, 0, 0, 0], 9, 3) == 3
