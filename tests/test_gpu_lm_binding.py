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
