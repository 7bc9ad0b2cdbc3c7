"""sd_verify_tokens where draft and target laws are equal, next to equal or none, and
uniforms next to 1, against the float64 oracle.
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
