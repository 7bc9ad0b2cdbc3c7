"""sd_verify_tokens where draft and target laws are equal, next to equal or none, and
uniforms next to 1, against the float64 oracle.
"""
import pytest
import torch

import test_gpu_tokens as tok
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
