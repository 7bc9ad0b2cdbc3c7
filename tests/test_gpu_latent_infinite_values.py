"""An infinite value that a row sees with a weight of 0 (a score far below the row's largest).

The weight is 0 in float32, and 0 times an infinity is NaN: the same for every row that
sees the key, wherever its tile lies (on the causal diagonal, where rows that do not see it
share the tile, or before it).
"""
import pytest
import torch

from paper_2606_13426_amd import _lib

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


def _tokens(L, j, t, low, bad):
    """Latent vectors whose j-th has scores `low` (the others 0) and an infinity in column 3."""
    g = torch.Generator(device=DEV)
    g.manual_seed(4)
    c = torch.zeros(L, 64 + 64, device=DEV)
    c[:, :64] = torch.randn(L, 64, generator=g, device=DEV)
    c[j, 64] = low
    c = c.to(TYPES[t])
    c[j, 3] = bad
    return c


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("low,nan", [(-400.0, True), (-2.0, False)])
@pytest.mark.parametrize("j", [0, 5, 64, 100, 190, 199])
@pytest.mark.parametrize("bad", [float("inf"), -float("inf")])
def test_an_infinity_of_no_weight(t, low, nan, j, bad):
    L = 200
    c = _tokens(L, j, t, low, bad)
    q = torch.zeros(L, 1, 128, device=DEV, dtype=TYPES[t])
    q[..., 64] = 1.0
    cu = torch.tensor([0, L], dtype=torch.int32, device=DEV)
    k, v = torch.zeros(L, 1, 64, device=DEV, dtype=TYPES[t]), c[:, None, :64]
    out, _ = _lib.sd_latent_attention_expanded(q, k, c[:, 64:], v, cu, cu, scale=1.0)
    x = out[:, 0].float()
    assert torch.isfinite(x[:j]).all()
    if j == 0:  # its only key for row 0: weight 1 whatever the score
        assert x[0, 3] == bad
    seen = x[max(j, 1):, 3]
    assert (torch.isnan(seen) if nan else seen == bad).all()
    keep = torch.arange(64, device=DEV) != 3
    assert torch.isfinite(x[:, keep]).all()
