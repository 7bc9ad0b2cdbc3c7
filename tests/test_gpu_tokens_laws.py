"""sd_verify_tokens where draft and target laws are equal, next to equal or none, and
uniforms next to 1, against the float64 oracle.

What the kernels compute in float64, with u = 2^-53: a weight e^{(x - m) / T} is off by
4e-16 (the end of its series), 40 u (a rounded factor; |x - m| / T up to 40 matters) and 4 u
relative, a row's sum of weights by that and 160 u (its additions, at most), so log S
by less than 3e-14, a log-ratio by 6e-14 and log alpha_j by 6e-14 j.  Log-ratios and
distances of alpha_j from 1 below 2^-44 = 5.7e-14 are taken for 0.
"""
import numpy as np
import pytest
import torch

import test_gpu_tokens as tok
from oracle import tokens as otok
from paper_2606_13426_amd import _lib

pytestmark = pytest.mark.gpu
DEV = "cuda"
MODES = [_lib.SD_BLOCK, _lib.SD_TOKEN]


def _equal(B, K, V, t, seed):
    draft, target, tokens, kb, un = tok._blocks(B, K, V, t, seed)
    target = target.contiguous()
    kb.fill_(K)
    return target[:, :K].contiguous(), target, tokens, kb, un


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("t", list(tok.TYPES))
@pytest.mark.parametrize("V", [2000, 50001])
def test_a_draft_that_equal_laws_reject_is_followed_by_a_draw_from_the_target(V, t, mode):
    """The residual of equal laws has no mass: q is drawn from, not what rounding leaves of q - p."""
    draft, target, tokens, kb, un = _equal(24, 2, V, t, 31)
    tokens[::2, 0] = V  # outside the vocabulary
    for b in range(1, 24, 2):  # or masked in both rows
        draft[b, 0, tokens[b, 0].long()] = target[b, 0, tokens[b, 0].long()] = -float("inf")
    r = _lib.sd_verify_tokens(draft, target, tokens, kb, uniforms=un, mode=mode)
    assert (r["tau"] == 1).all()
    assert tok._check_verify(draft, target, tokens, kb, un, mode, 1.0, r) == (24, 24)


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("t", list(tok.TYPES))
@pytest.mark.parametrize("V", [5, 600, 9000])
def test_rows_of_nothing_but_nan_have_no_law(V, t, mode):
    nan, inf = float("nan"), float("inf")
    draft, target, tokens, kb, un = tok._blocks(8, 3, V, t, 41)
    draft, target = draft.contiguous(), target.contiguous()
    kb.fill_(3)
    tokens[:, 0] = target[:, 0].float().argmax(-1).to(torch.int32)
    draft[0, 0] = nan
    draft[1, 0] = -inf
    draft[1, 0, V // 2] = nan
    draft[2, 2] = nan
    target[3, 0] = nan
    target[4, 0] = -inf
    target[4, 0, V - 1] = nan
    target[5, 3] = nan
    draft[6], target[6] = nan, nan
    r = _lib.sd_verify_tokens(draft, target, tokens, kb, uniforms=un, mode=mode)
    decided, _ = tok._check_verify(draft, target, tokens, kb, un, mode, 1.0, r)
    assert decided >= 7
    for b in (0, 1, 3, 4, 6):
        assert r["tau"][b] == 1 and r["token"][b] == -1, b


@pytest.mark.parametrize("V", [50001, 128256])
@pytest.mark.parametrize("ulps", [1, 2])
@pytest.mark.parametrize("masked", [False, True])
def test_uniforms_next_to_one_draw_a_token(V, ulps, masked):
    """Additions in another order give a thread without mass a sum above the last token's: it is never chosen.

    The drawn token has weight, and behind it no more of the mass than the sums' rounding
    (V u = 1.5e-11 in the worst order)."""
    B = 96
    draft, target, tokens, kb, un = tok._blocks(B, 1, V, "f32", 50 + ulps)
    target = target.contiguous()
    if masked:  # most slices have no mass
        target[:, :, 3000:V - 9000] = -float("inf")
        target[:, :, V - 7:] = -float("inf")
    kb.fill_(1)
    un[:, 1] = 1.0 - ulps * 2.0 ** -53
    r = {k: v.cpu().numpy() for k, v in _lib.sd_verify_tokens(draft, target, tokens, kb, uniforms=un).items()}
    d, q = draft.double().cpu().numpy(), target.double().cpu().numpy()
    for b in range(B):
        lq = otok.row_law(q[b, r["tau"][b] - 1])
        w = np.exp(lq) if r["tau"][b] == 2 else np.maximum(0.0, np.exp(lq) - np.exp(otok.row_law(d[b, 0])))
        x = r["token"][b]
        assert 0 <= x < V and w[x] > 0, (b, x)
        assert w[x + 1:].sum() <= 1.5e-11 * w.sum(), (b, x)


def test_a_uniform_on_a_border_draws_a_token():
    """Few tokens of one weight: half, a quarter of the whole are sums to the last bit, or next to them."""
    B, V = 64, 70000
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    target = torch.full((B, 2, V), -float("inf"), device=DEV)
    allowed = []
    for b in range(B):
        at = torch.randperm(V, generator=g, device=DEV)[:2 + b % 37].sort().values
        target[b, 0, at] = 0.25
        allowed.append(at.tolist())
    target[:, 1] = target[:, 0]
    draft = torch.full((B, 1, V), -float("inf"), device=DEV)  # the residual is the target's law
    tokens, kb = torch.full((B, 1), -1, dtype=torch.int32, device=DEV), torch.ones(B, dtype=torch.int32, device=DEV)
    un = torch.empty(B, 2, dtype=torch.float64, device=DEV)
    for u in (0.5, 0.25, 1.0 / 3.0, 0.2, 0.7):
        un.fill_(u)
        r = _lib.sd_verify_tokens(draft, target, tokens, kb, uniforms=un)
        for b in range(B):
            n = len(allowed[b])
            x = int(r["token"][b])
            assert x in allowed[b], (b, u, x)
            assert abs(allowed[b].index(x) - u * n) <= 1.0 + 1e-9, (b, u, x)


@pytest.mark.parametrize("t,near", [("f32", 1e-2), ("f32", 1e-3), ("f32", 1e-4), ("f32", 1e-6), ("f16", 1e-3), ("bf16", 1e-2)])
@pytest.mark.parametrize("B,V", [(24, 30011), (200, 2049)])
def test_coins_of_laws_that_are_next_to_equal(t, near, B, V):
    """h = v / (v + 1 - alpha) divides two numbers of the laws' difference.

    dh = ((1 - alpha) dv + v dalpha) / (v + 1 - alpha)^2 is at most (dv + dalpha) / (v + 1 - alpha);
    dalpha is 12e-14 j (above), dv no more than dalpha and two sums' 3e-14 each: with j <= 3 and the
    oracle's own share 1e-12 in all.  Every coin's uniform is put that far below or above its h."""
    K = 3
    draft, target, tokens, kb, un = tok._blocks(B, K, V, t, 61, near=near)
    kb.fill_(K)
    d, q = draft.double().cpu().numpy(), target.double().cpu().numpy()
    x, u = tokens.cpu().numpy(), un.cpu().numpy()
    moved = 0
    for b in range(B):
        w = otok.verify_chain(d[b], q[b], x[b], K, u[b, :K], 0.5)
        la = [0.0]
        for j in range(K):
            la.append(min(0.0, la[j] + w["ell"][j]))
        for j in range(1, K + 1):
            a = np.exp(la[j])
            if j < K and a < 1.0:
                v = np.maximum(0.0, np.exp(otok.row_law(q[b, j]) + la[j]) - np.exp(otok.row_law(d[b, j]))).sum()
                margin = 1e-12 / (v + 1.0 - a)
            else:
                margin = 1e-12
            side = 1 if (b + j) % 2 else -1
            u[b, j - 1] = min(max(w["h"][j - 1] + side * margin, 2.0 ** -60), 1.0 - 2.0 ** -53)
            moved += 0.0 < w["h"][j - 1] < 1.0
    assert moved > B
    r = _lib.sd_verify_tokens(draft, target, tokens, kb, uniforms=torch.tensor(u, device=DEV))
    coins, tau, lar = (r[k].cpu().numpy() for k in ("coins", "tau", "log_alpha_res"))
    for b in range(B):
        w = otok.verify_chain(d[b], q[b], x[b], K, u[b, :K], 0.5)
        assert coins[b] == w["coins"] and tau[b] == w["tau"], (b, coins[b], w["coins"], w["h"], u[b])
        assert abs(lar[b] - w["log_alpha_res"]) <= 2.0 ** -24 * abs(w["log_alpha_res"]) + 2e-13


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("t", list(tok.TYPES))
@pytest.mark.parametrize("V", [2049, 50001])
def test_equal_laws_at_other_alignments_are_equal(V, t, mode):
    """Rows of an odd number of logits start at other places of a 16-byte vector, so that the sums of
    equal rows differ by their order: alpha_j is 1 all the same, and h_j with it."""
    B, K = 24, 4
    draft, target, tokens, kb, un = _equal(B, K, V, t, 71)
    kb[::3] = K - 1
    last = kb.long() - 1
    tokens[torch.arange(B, device=DEV), last] = V  # the block's last draft is rejected, and no other
    un[:, :K] = 0.9
    r = _lib.sd_verify_tokens(draft, target, tokens, kb, uniforms=un, mode=mode)
    assert torch.equal(r["tau"], kb) and (r["log_alpha_res"] == 0).all()
    held = r["log_ratio"][torch.arange(K, device=DEV)[None] < last[:, None]]
    assert (held == 0).all()
    assert tok._check_verify(draft, target, tokens, kb, un, mode, 1.0, r) == (B, B)


@pytest.mark.parametrize("t,V", [("f32", 50001), ("f32", 131072), ("bf16", 50001), ("f16", 8193)])
def test_log_ratios_are_rounded_once(t, V):
    """What float64 gives (6e-14, above) rounded to float32: a coin's threshold has no fewer bits."""
    draft, target, tokens, kb, un = tok._blocks(5, 4, V, t, 81)
    kb.fill_(4)
    got = _lib.sd_verify_tokens(draft, target, tokens, kb, uniforms=un)["log_ratio"].cpu().numpy()
    d, q, x = draft.double().cpu().numpy(), target.double().cpu().numpy(), tokens.cpu().numpy()
    for b in range(5):
        for j in range(4):
            want = otok.row_law(q[b, j])[x[b, j]] - otok.row_law(d[b, j])[x[b, j]]
            assert abs(got[b, j] - want) <= 2.0 ** -24 * abs(want) + 1e-13, (b, j, got[b, j], want)


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("t", list(tok.TYPES))
@pytest.mark.parametrize("power", [-60, -20, -5, 5, 20])
def test_temperatures(power, t, mode):
    """From laws of one token to laws of equal ones, next to equal."""
    draft, target, tokens, kb, un = tok._blocks(30, 4, 3001, t, 5)
    r = _lib.sd_verify_tokens(draft, target, tokens, kb, uniforms=un, mode=mode, temperature=2.0 ** power)
    decided, drawn = tok._check_verify(draft, target, tokens, kb, un, mode, 2.0 ** power, r)
    assert decided >= 29 and drawn >= decided - 1


def test_the_largest_vocabulary():
    V = 1 << 24
    draft, target, tokens, kb, un = tok._blocks(2, 1, V, "bf16", 5)
    kb.fill_(1)
    r = _lib.sd_verify_tokens(draft, target, tokens, kb, uniforms=un)
    d, q = draft.double().cpu().numpy(), target.double().cpu().numpy()
    x, u = tokens.cpu().numpy(), un.cpu().numpy()
    for b in range(2):
        w = otok.verify_chain(d[b], q[b], x[b], 1, u[b, :1], u[b, 1])
        assert abs(u[b, 0] - w["h"][0]) > 1e-9 and r["tau"][b] == w["tau"]
        c = np.cumsum(w["w"])
        # (the oracle's sums are off by V u = 1.9e-9 of the whole at most)
        at, goal = int(r["token"][b]), u[b, 1] * c[-1]
        assert w["w"][at] > 0 and c[at] >= goal - 4e-9 * c[-1] and c[at] - w["w"][at] <= goal + 4e-9 * c[-1]
