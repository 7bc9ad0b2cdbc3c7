"""Operands that the binding of the language-model calls refuses before anything is launched."""
import pytest
import torch

from paper_2606_13426_amd import _lib

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _verify(**kw):
    z = lambda *s, t=torch.float32: torch.zeros(*s, dtype=t, device=DEV)  # noqa: E731
    a = dict(draft=z(2, 2, 50), target=z(2, 3, 50), tokens=z(2, 2, t=torch.int32), kb=z(2, t=torch.int32),
             rnd=z(2, t=torch.int32))
    a.update(kw)
    return _lib.sd_verify_tokens(**a)


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16, torch.int64])
def test_rounds_are_whole_numbers_of_32_bits(t):
    with pytest.raises(_lib.SpecDiffError, match="rnd must be"):
        _verify(rnd=torch.ones(2, device=DEV).to(t))
    _verify(rnd=torch.ones(2, device=DEV).to(torch.uint32))


@pytest.mark.parametrize("call", ["verify", "logprobs", "absorbed", "expanded"])
def test_a_workspace_with_gaps_is_refused(call):
    ws = torch.zeros(1 << 26, dtype=torch.uint8, device=DEV)[::2]
    h = lambda *s: torch.zeros(*s, dtype=torch.float16, device=DEV)  # noqa: E731
    i = lambda *s: torch.tensor(s, dtype=torch.int32, device=DEV)  # noqa: E731
    with pytest.raises(_lib.SpecDiffError, match="ws must be contiguous"):
        if call == "verify":
            _verify(ws=ws)
        elif call == "logprobs":
            _lib.sd_token_logprobs(torch.zeros(3, 40, device=DEV), ws=ws)
        elif call == "absorbed":
            _lib.sd_latent_attention(h(1, 1, 2, 192), h(3, 16, 192), i(1), 128, scale=0.1, ws=ws)
        else:
            _lib.sd_latent_attention_expanded(h(3, 2, 64), h(2000, 2, 64), None, h(2000, 2, 64), i(0, 3), i(0, 2000), ws=ws)
