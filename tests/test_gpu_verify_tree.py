"""sd_verify_tree against the oracle's walk in float64.

The kernels' laws are sums of at most 160 roundings (2^-45 relative), so the ratio r = q/p and a, a sum of
such numbers, are off by 2^-43 (1 + r + a) together, what is left of p by 2^-44 of itself, and S =
sum max(0, q - a p), in which a p is below q and adds up to less than 1, by 2^-44: a try h = (r - a) rest / S by
2^-43 ((1 + r + a) rest + 2 h) / S, and half a step of float32 of itself where it is given out.  A coin nearer
than that to its h would be no test: none is (asserted).  The drawn token's border is off by 2^-42 / S of the
whole.
"""
import numpy as np
import pytest
import torch

from oracle import tree
from paper_2606_13426_amd import _lib

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
DRAWS = {"iid": _lib.SD_TREE_IID, "distinct": _lib.SD_TREE_DISTINCT, "given": _lib.SD_TREE_GIVEN}


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _grown(seed, B, Q, wide):
    r, trees = np.random.default_rng(seed), []
    for _ in range(B):
        has, p = [0] * Q, [-1]
        for i in range(1, Q):
            free = [j for j in range(i) if has[j] < wide]
            p.append(int(free[int(len(free) * r.random() ** 1.5)]))
            has[p[-1]] += 1
        trees.append(p)
    return trees


def _inputs(B, Q, V, wide, draws, t, seed, near=0.6):
    """Laws with a few likely tokens, and candidates as they are drawn in earnest."""
    g = _gen(seed)
    target = torch.randn(B, Q, V, generator=g, device=DEV) * 2
    target[..., :: max(1, V // 7)] += 5
    draft = (target + near * torch.randn(B, Q, V, generator=g, device=DEV)).to(TYPES[t])
    trees = _grown(seed, B, Q, wide)
    tokens, e = torch.zeros(B, Q, dtype=torch.int32), torch.rand(B, Q, V, generator=g, device=DEV)
    score = draft.float() - (torch.log(-torch.log(e.clamp(1e-7, 1 - 1e-7))) if draws != "given" else 0)
    for b in range(B):
        had = [0] * Q
        for i in range(1, Q):
            p = trees[b][i]
            if draws == "iid":
                x = draft[b, p].float() - torch.log(-torch.log(torch.rand(V, generator=g, device=DEV).clamp(1e-7, 1 - 1e-7)))
                tokens[b, i] = int(x.argmax())
            else:
                tokens[b, i] = int(score[b, p].topk(min(V, wide)).indices[had[p] % min(V, wide)])
            had[p] += 1
    un = torch.rand(B, Q, generator=g, device=DEV, dtype=torch.float64)
    return None if draws == "given" else draft, target.to(TYPES[t]), tokens.to(DEV), trees, un


def _check(draft, target, tokens, trees, un, got, draws, rows=None, wide=None, T=1.0, seqs=None):
    B, Q, V = target.shape
    x, tok, u = target.double().cpu().numpy(), tokens.cpu().numpy(), un.cpu().numpy()
    y = None if draft is None else draft.double().cpu().numpy()
    tau, token, path, accept = (got[k].cpu().numpy() for k in ("tau", "token", "path", "accept"))
    for b in range(B) if seqs is None else seqs:
        n = Q if rows is None else min(max(rows[b], 0), Q)
        eta = np.concatenate([[0.0], u[b, :Q - 1]])
        w = tree.verify(None if y is None else y[b], x[b], tok[b], trees[b], n, eta, u[b, Q - 1], draws, wide, T)
        say = (b, w, tau[b], token[b], path[b][:8])
        bound = _bounds(None if y is None else y[b], x[b], tok[b], trees[b], n, w, draws, wide, T)
        for i, h in w["accept"].items():
            assert abs(eta[i] - h) > bound[i], say  # (else another seed)
        assert tau[b] == w["tau"] and list(path[b]) == w["path"] + [-1] * (Q - len(w["path"])), say
        for i in range(Q):
            h = w["accept"].get(i, -1.0)
            assert abs(accept[b, i] - h) <= bound.get(i, 0.0) + 2.0 ** -24 * abs(h), (say, i, accept[b, i], h)
        if token[b] != w["token"]:
            assert w["w"] is not None and token[b] >= 0, say
            c = np.cumsum(w["w"]) / w["w"].sum()
            lo, hi = sorted((token[b], w["token"]))
            assert abs(c[lo] - u[b, Q - 1]) <= bound[None] and w["w"][token[b]] > 0 and c[hi - 1] - c[lo] <= bound[None], say


def _bounds(y, x, tok, parents, n, w, draws, wide, T):
    """How far each tried node's h may be off, and (None) the borders of the last law."""
    out = {None: 2.0 ** -40}
    for node in w["path"]:
        kids = [i for i in w["accept"] if tree.parent_of(parents, i) == node]
        lq = tree.row_law(x[node], T)
        lp = tree.row_law(y[node], T) if y is not None else None
        if lq is None or (y is not None and lp is None) or lq.max() == -np.inf:
            out.update({i: 0.0 for i in kids})
            continue
        a0, S0, rest, q, p = 0.0, 1.0, 1.0, np.exp(lq), None if y is None else np.exp(lp)
        left = None if p is None else p.copy()
        for i, (h, _, a, S, _) in zip(kids, tree.tries(q, p, [tok[k] for k in kids], draws, None if lp is None else lq - lp)):
            known = 0 <= tok[i] < len(q)
            if not known:
                out[i] = 0.0
                continue
            with np.errstate(invalid="ignore", over="ignore"):
                r = q[tok[i]] if p is None else np.exp(lq[tok[i]] - lp[tok[i]])
            if not np.isfinite(r):  # of a draft of no probability: h is 0 or 1 whatever the sums
                out[i], a0, S0 = 0.0, a, S
                continue
            err = 2.0 ** -43 * (1 + r + a0)
            out[i] = 0.0 if h == 0 and r < a0 - err else (err * rest + 2.0 ** -42 * h) / max(S0, 2.0 ** -40)  # (max(0, r - a) is 0)
            a0, S0 = a, S
            if draws == "distinct":
                left[tok[i]] = 0.0
                rest = left.sum()
        out[None] = max(out[None], 2.0 ** -42 / max(S0, 2.0 ** -40))
    return out


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("draws", list(DRAWS))
@pytest.mark.parametrize("B,Q,V,wide", [
    (1, 1, 5, 1), (2, 2, 1, 1), (1, 2, 7, 1), (3, 9, 1000, 3), (5, 64, 4099, 4), (3, 64, 300, 63), (4, 12, 32000, 2), (2, 17, 70001, 1),
    (64, 32, 3001, 4), (2, 7, 9, 6)])
def test_trees(B, Q, V, wide, draws, t):
    draft, target, tokens, trees, un = _inputs(B, Q, V, wide, draws, t, B * 7 + Q)
    got = _lib.sd_verify_tree(draft, target, tokens, _i32(trees), draws=DRAWS[draws], max_children=min(wide, Q), uniforms=un)
    _check(draft, target, tokens, trees, un, got, draws, wide=wide, seqs=None if B < 10 else range(0, B, 5))


@pytest.mark.parametrize("draws", list(DRAWS))
def test_far_drafts_take_many_tries(draws):
    """Drafts that are mostly refused: all rounds of a node run, and its last law is what they leave."""
    for seed in range(6):
        draft, target, tokens, trees, un = _inputs(4, 12, 900, 11, draws, "f32", 40 + seed, near=4.0)
        trees = [[-1] + [0] * 11] * 4
        if draws != "iid":
            score = (draft if draft is not None else target)[:, 0].float()
            tokens[:, 1:] = score.topk(11).indices.to(torch.int32)
        un[:, :11] = 0.6 + 0.4 * un[:, :11]
        got = _lib.sd_verify_tree(draft, target, tokens, _i32(trees), draws=DRAWS[draws], uniforms=un)
        _check(draft, target, tokens, trees, un, got, draws)


@pytest.mark.parametrize("T", [0.25, 3.0, 2.0 ** -60])
@pytest.mark.parametrize("draws", list(DRAWS))
def test_temperatures(T, draws):
    draft, target, tokens, trees, un = _inputs(3, 10, 500, 3, draws, "bf16", 50)
    got = _lib.sd_verify_tree(draft, target, tokens, _i32(trees), draws=DRAWS[draws], uniforms=un, temperature=T)
    _check(draft, target, tokens, trees, un, got, draws, T=T)


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("K,V", [(1, 11), (4, 32000), (9, 50001)])
def test_a_chain_has_the_results_of_token_verification(K, V, t):
    B = 6
    draft, target, tokens, trees, un = _inputs(B, K + 1, V, 1, "iid", t, K)
    kb = _i32([K, max(1, K - 1), K, 0, 99, 1])
    for kw in (dict(uniforms=un), dict(rnd=_i32([3, 0, 9, 9, 2, 1]), seed=77)):
        want = _lib.sd_verify_tokens(draft[:, :K], target, tokens[:, 1:].contiguous(), kb, mode=_lib.SD_TOKEN, **kw)
        got = _lib.sd_verify_tree(draft, target, tokens, _i32([list(range(-1, K))] * B), rows=kb.clamp(max=K) + (kb > 0).int(),
                                  max_children=1, **kw)
        assert torch.equal(want["tau"], got["tau"]) and torch.equal(want["token"], got["token"])
        for b in range(B):
            n = int(want["tau"][b])
            assert got["path"][b].tolist() == list(range(n)) + [-1] * (K + 1 - n)


@pytest.mark.parametrize("draws", list(DRAWS))
def test_trees_that_are_none(draws):
    """Parents of no node, nodes that the root does not reach, rows of no sequence, more children than are tried."""
    B, Q, V = 6, 10, 400
    draft, target, tokens, _, un = _inputs(B, Q, V, 3, draws, "f32", 60)
    trees = [[4, 0, 5, -1, 3, 2 ** 31 - 1, 1, 0, 9, 2], [-2 ** 31, 1, 0, 2, 4, 4, 3, 0, 0, 2], [0] * 10, [-1, 0, 0, 0, 1, 1, 1, 2, 2, 2],
             [-1] + list(range(9)), [-1, 0, 1, 2, 3, 4, 5, 6, 7, 8]]
    rows = [10, 10, 10, 0, 1, -4]
    tokens[0, 1], tokens[1, 2], tokens[2, 3] = V, -1, -2 ** 31  # drafts of no token
    tokens[0, 0] = 2 ** 31 - 1
    for wide in (None, 1, 2, 9):
        got = _lib.sd_verify_tree(draft, target, tokens, _i32(trees), rows=_i32(rows), draws=DRAWS[draws], max_children=wide,
                                  uniforms=un)
        _check(draft, target, tokens, trees, un, got, draws, rows=rows, wide=wide)
    assert got["tau"][3] == 0 and got["token"][3] == -1 and (got["path"][3] == -1).all() and (got["accept"][3] == -1).all()


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("draws", ["distinct", "given", "iid"])
def test_the_same_candidate_twice(draws, t):
    draft, target, tokens, _, un = _inputs(4, 8, 50, 7, draws, t, 70)
    trees = [[-1] + [0] * 7] * 4
    top = target[:, 0].float().topk(3).indices.to(torch.int32)
    tokens[:, 1:] = top[:, [0, 0, 1, 0, 2, 1, 2]]
    un[:, :7] = 0.5 + 0.5 * un[:, :7]
    got = _lib.sd_verify_tree(draft, target, tokens, _i32(trees), draws=DRAWS[draws], uniforms=un)
    _check(draft, target, tokens, trees, un, got, draws)


@pytest.mark.parametrize("draws", list(DRAWS))
@pytest.mark.parametrize("t", list(TYPES))
def test_masks_and_rows_without_a_law(draws, t):
    """Masks that leave one token or none, NaN and +inf, on the walk and off it."""
    B, Q, V = 12, 6, 3000
    draft, target, tokens, _, un = _inputs(B, Q, V, 2, draws, t, 80)
    trees = [[-1, 0, 0, 1, 1, 2]] * B
    none = -float("inf")
    un[:, 0] = 1e-9  # the walk goes to node 1 where that has any chance
    target[0] = none
    target[1, 0], target[1, 0, 7] = none, 0.0  # one token, which nobody drafted
    target[2, 0], target[2, 0, 7], tokens[2, 1] = none, 3.0, 7
    target[3, 1, 5] = float("nan")
    target[4, 3, 2999] = float("inf")
    target[5, 2, 0] = float("nan")  # off the walk
    target[6, 0, ::2] = none
    target[7, 1] = none
    target[8, 0, :] = torch.finfo(target.dtype).min
    target[8, 0, 17], tokens[8, 1], tokens[8, 2] = 1.0, 16, 17
    if draft is not None:
        draft[6, 0, 1::2] = none  # nothing in common with the target
        tokens[6, 1], tokens[6, 2] = 4, 8
        draft[7, 0, tokens[7, 1].long()] = none  # a draft of draft probability 0
        draft[9, 1, 11] = float("nan")
        draft[10, 1] = none
        draft[11, 2, 3] = float("inf")  # off the walk
    got = _lib.sd_verify_tree(draft, target, tokens, _i32(trees), draws=DRAWS[draws], uniforms=un)
    _check(draft, target, tokens, trees, un, got, draws)
    assert got["token"][0] == -1 and got["token"][1] == 7 and got["token"][3] == -1


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("off", [0, 1, 3])
def test_equal_laws_accept_and_leave_nothing(off, t):
    """Draft rows that hold the target's values, also at other places of a 16-byte vector: h = 1 whatever the coin."""
    B, Q, V = 3, 5, 20003
    _, target, tokens, _, un = _inputs(B, Q, V, 2, "iid", t, 90)
    trees = [[-1, 0, 0, 1, 1]] * B
    draft = torch.empty(B, Q, V + 8, device=DEV, dtype=target.dtype)[..., off:off + V]
    draft.copy_(target)
    un[:, :4] = 1 - 1e-15
    got = _lib.sd_verify_tree(draft, target, tokens, _i32(trees), uniforms=un)
    assert got["path"].tolist() == [[0, 1, 3, -1, -1]] * B and (got["accept"][:, [1, 3]] == 1).all()


def test_drafts_that_leave_next_to_nothing_of_their_law():
    """Draws without replacement from a law that is all one token but 1e-17: the rest is summed, not subtracted."""
    B, Q, V = 4, 4, 300
    g = _gen(95)
    target = torch.randn(B, Q, V, generator=g, device=DEV)
    draft = torch.randn(B, Q, V, generator=g, device=DEV)
    draft[:, 0, 9] = 47.0
    tokens = _i32([[0, 9, 30 + b, 60 + b] for b in range(B)])
    un = torch.rand(B, Q, generator=g, device=DEV, dtype=torch.float64)
    un[:, 0] = 0.9
    trees = [[-1, 0, 0, 0]] * B
    got = _lib.sd_verify_tree(draft, target, tokens, _i32(trees), draws=_lib.SD_TREE_DISTINCT, uniforms=un)
    _check(draft, target, tokens, trees, un, got, "distinct")


def test_views_rounds_and_given_outputs():
    """Strided rows, the generator's coins, outputs given; equal calls have equal bits."""
    B, Q, V = 5, 12, 1001
    draft, target, tokens, trees, _ = _inputs(B, Q, V, 3, "distinct", "bf16", 100)
    wide = torch.zeros(B, Q + 2, V + 5, device=DEV, dtype=target.dtype)
    wide[:, 1:Q + 1, 3:V + 3] = target
    rnd = _i32([5, 0, 2 ** 31 - 1, 7, 7])
    call = lambda t, **kw: _lib.sd_verify_tree(draft, t, tokens, _i32(trees), draws=_lib.SD_TREE_DISTINCT, **kw)  # noqa: E731
    want = call(target, rnd=rnd, seed=9)
    got = call(wide[:, 1:Q + 1, 3:V + 3], rnd=rnd.view(torch.uint32), seed=9,
               out={k: torch.full_like(v, 77) for k, v in want.items()})
    for k in want:
        assert torch.equal(want[k], got[k]) or k == "accept", k
    assert (want["accept"] - got["accept"]).abs().max() <= 1e-6
    # the same coins as given uniforms
    un = torch.empty(B, Q, dtype=torch.float64, device=DEV)
    words = torch.tensor([[i, b, int(rnd[b]), 3 << 24] for b in range(B) for i in range(Q // 4)], dtype=torch.int64, device=DEV)
    out = torch.empty(len(words), 4, dtype=torch.uint32, device=DEV)
    _lib.sd_philox_words(9, words.to(torch.int32).view(torch.uint32), out)
    un[:, :Q] = ((out.view(torch.int32).long() & 0xFFFFFFFF) >> 8).double().add(0.5).mul(2.0 ** -24).view(B, Q)
    w = torch.tensor([[0, b, int(rnd[b]), 4 << 24] for b in range(B)], dtype=torch.int64, device=DEV)
    out = torch.empty(B, 4, dtype=torch.uint32, device=DEV)
    _lib.sd_philox_words(9, w.to(torch.int32).view(torch.uint32), out)
    o = out.view(torch.int32).long() & 0xFFFFFFFF
    un[:, Q - 1] = (((o[:, 0] >> 6) * 2 ** 26 + (o[:, 1] >> 6)).double() + 0.5) * 2.0 ** -52
    same = call(target, uniforms=un)
    assert all(torch.equal(want[k], same[k]) for k in want)
    _check(draft, target, tokens, trees, un, want, "distinct")
    again = dict(want, accept=None)
    _lib.sd_verify_tree(draft, target, tokens, _i32(trees), draws=_lib.SD_TREE_DISTINCT, rnd=rnd, seed=9,
                        out=dict(tau=again["tau"], token=again["token"], path=again["path"]))
    for k, bad in (("tau", want["tau"].long()), ("token", want["token"][:1]), ("path", want["path"].t()), ("accept", want["accept"].cpu())):
        with pytest.raises(_lib.SpecDiffError):
            call(target, uniforms=un, out=dict(want, **{k: bad}))


@pytest.mark.parametrize("draws", ["iid", "distinct"])
def test_the_next_token_follows_the_targets_law(draws):
    """16384 trees of 3 candidates over 6 tokens: the token behind the root is drawn from q (a chi-square of 5
    degrees of freedom stays below 31 but for 1e-5)."""
    B, V = 16384, 6
    g = _gen(110)
    q = torch.tensor([0.05, 0.3, 0.2, 0.1, 0.25, 0.1], device=DEV)
    p = torch.tensor([0.4, 0.1, 0.1, 0.2, 0.05, 0.15], device=DEV)
    target, draft = (torch.log(x).expand(B, 4, V).contiguous() for x in (q, p))
    e = torch.rand(B, 3, V, generator=g, device=DEV).clamp(1e-7, 1 - 1e-7)
    noisy = torch.log(p) - torch.log(-torch.log(e))
    x = noisy.argmax(-1) if draws == "iid" else noisy[:, 0].topk(3).indices
    tokens = torch.cat([torch.zeros(B, 1, device=DEV), x], 1).to(torch.int32)
    un = torch.rand(B, 4, generator=g, device=DEV, dtype=torch.float64)
    got = _lib.sd_verify_tree(draft, target, tokens, _i32([-1, 0, 0, 0]).expand(B, 4).contiguous(), draws=DRAWS[draws], uniforms=un)
    first = torch.where(got["tau"] > 1, tokens.gather(1, got["path"][:, 1:2].clamp(min=0).long())[:, 0], got["token"])
    n = torch.bincount(first.long(), minlength=V).double()
    want = (q.double() / q.double().sum()) * B
    assert float(((n - want) ** 2 / want).sum()) < 31
    assert 0.3 < float((got["tau"] > 1).double().mean()) < 1.0


# 40 * 2^20 logits and more: the root's law comes first, then its children's, then what the walk may still come to.
@pytest.mark.parametrize("near", [1.0, 4.0])
@pytest.mark.parametrize("draws,t", [("iid", "f32"), ("distinct", "bf16"), ("given", "f16"), ("distinct", "f16")])
def test_much_work_in_stages(draws, t, near):
    B, Q, V, wide = 24, 32, 60001, 4
    draft, target, tokens, trees, un = _inputs(B, Q, V, wide, draws, t, 90 + int(near), near=near)
    rows = [(7 * b) % 33 for b in range(B)]
    got = _lib.sd_verify_tree(draft, target, tokens, _i32(trees), draws=DRAWS[draws], max_children=wide, uniforms=un, rows=_i32(rows))
    _check(draft, target, tokens, trees, un, got, draws, rows=rows, wide=wide, seqs=range(0, B, 3))
    again = _lib.sd_verify_tree(draft, target, tokens, _i32(trees), draws=DRAWS[draws], max_children=wide, uniforms=un, rows=_i32(rows))
    for key, value in got.items():
        assert torch.equal(value, again[key]), key
    # the same trees a few at a time, whose nodes are all summed at once (in slices of another size)
    part = slice(8, 11)
    few = _lib.sd_verify_tree(None if draft is None else draft[part], target[part], tokens[part], _i32(trees[part]), draws=DRAWS[draws],
                              max_children=wide, uniforms=un[part], rows=_i32(rows[part]))
    assert torch.equal(few["tau"], got["tau"][part]) and torch.equal(few["path"], got["path"][part])


def test_a_long_chain_in_stages():
    B, K, V = 12, 63, 60001
    draft, target, tokens, trees, un = _inputs(B, K + 1, V, 1, "iid", "bf16", 95, near=0.02)
    trees = [[j - 1 for j in range(K + 1)]] * B
    tokens[:, 1:] = draft[:, :K].float().argmax(-1).to(torch.int32)
    un[:, :K] *= 0.9
    got = _lib.sd_verify_tree(draft, target, tokens, _i32(trees), uniforms=un)
    _check(draft, target, tokens, trees, un, got, "iid", seqs=[0, 5, 11])
    assert (got["tau"] > 3).any()


@pytest.mark.parametrize("draws", list(DRAWS))
@pytest.mark.parametrize("B,K", [(11, 40), (210, 2)])
def test_chains_in_stages_of_rising_depth(B, K, draws):
    """One child a node is tried: of chains, and of trees whose other children are no part of it."""
    V = 60001
    draft, target, tokens, trees, un = _inputs(B, K + 1, V, 2, draws, "f16", 97, near=0.05)
    trees = [[j - 1 for j in range(K + 1)] if b % 3 else trees[b] for b in range(B)]
    for b in range(B):
        for i in range(1, K + 1):
            if b % 3 and draws != "given":
                tokens[b, i] = draft[b, i - 1].float().argmax()
            elif b % 3:
                tokens[b, i] = target[b, i - 1].float().argmax()
    un[:, :K] *= 0.9 if draws != "given" else 0.05
    got = _lib.sd_verify_tree(draft, target, tokens, _i32(trees), draws=DRAWS[draws], max_children=1, uniforms=un)
    _check(draft, target, tokens, trees, un, got, draws, wide=1, seqs=[0, 1, 2, 5, B - 1])
    assert (got["tau"] > 2).any()


@pytest.mark.parametrize("draws", list(DRAWS))
def test_more_children_than_nodes_are_all(draws):
    draft, target, tokens, trees, un = _inputs(4, 3, 900, 6, draws, "f32", 99)
    want = _lib.sd_verify_tree(draft, target, tokens, _i32(trees), draws=DRAWS[draws], uniforms=un)
    for most in (2, 3, 6, 1000):
        got = _lib.sd_verify_tree(draft, target, tokens, _i32(trees), draws=DRAWS[draws], uniforms=un, max_children=most)
        assert all(torch.equal(got[k], want[k]) for k in want)
    _check(draft, target, tokens, trees, un, want, draws)


@pytest.mark.parametrize("draws", list(DRAWS))
def test_stages_in_a_graph(draws):
    B, Q, V, wide = 24, 32, 60001, 4
    draft, target, tokens, trees, un = _inputs(B, Q, V, wide, draws, "bf16", 120, near=2.0)
    ws = torch.empty(_lib.sd_verify_tree_workspace(B, Q, V), dtype=torch.uint8, device=DEV)
    parents, kw = _i32(trees), dict(draws=DRAWS[draws], max_children=wide)
    _lib.sd_verify_tree(draft, target, tokens, parents, uniforms=un, ws=ws, **kw)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = _lib.sd_verify_tree(draft, target, tokens, parents, uniforms=un, ws=ws, **kw)
    for i in range(4):
        ws.fill_(0xA5 if i % 2 else 0xFF)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = _lib.sd_verify_tree(draft, target, tokens, parents, uniforms=un, **kw)
        for key in want:
            assert torch.equal(want[key], kept[key]), (i, key)
        if i < 2:
            _check(draft, target, tokens, parents.tolist(), un, kept, draws, wide=wide, seqs=[i, 11])
        un.copy_(un.flip(0))
        parents.copy_(parents.flip(0))


@pytest.mark.parametrize("draws", list(DRAWS))
def test_equal_calls_have_equal_bits_where_nodes_are_decided_meanwhile(draws):
    """More workgroups than the card holds at once, trees with many inner nodes for each: some start while a node of their
    tree is being decided."""
    B, Q, V, wide = 32, 48, 100003, 4
    draft, target, tokens, trees, un = _inputs(B, Q, V, wide, draws, "bf16", 130, near=1.5)
    assert all(len(set(t[1:])) > 9 for t in trees)
    call = lambda: _lib.sd_verify_tree(draft, target, tokens, _i32(trees), draws=DRAWS[draws], max_children=wide, uniforms=un)  # noqa: E731
    got = call()
    _check(draft, target, tokens, trees, un, got, draws, wide=wide, seqs=range(0, B, 8))
    for _ in range(20):
        again = call()
        assert all(torch.equal(got[k], again[k]) for k in got)
