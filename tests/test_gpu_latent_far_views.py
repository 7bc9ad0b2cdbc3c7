"""Views of the two attention forms that lie far apart or in another order: strides of 2^24 elements
and more, heads outside tokens."""
import pytest
import torch

import test_gpu_latent as absorbed
import test_gpu_latent_expanded as expanded
from paper_2606_13426_amd import _lib

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("H,dc,dr", [(3, 128, 64), (5, 72, 8), (64, 512, 64)])
@pytest.mark.parametrize("table", [True, False])
@pytest.mark.parametrize("stride", [(1 << 24) - 8, 1 << 24])
def test_tokens_far_apart(H, dc, dr, table, stride):
    # (the addresses of what no token holds are not touched: 3.5 GB, of which a few lines are)
    B, Q, t, lens = 2, 2, "bf16", [66, 33]
    q, cache, ln, pages = absorbed._case(B, Q, H, dc, dr, lens, t, 3, page=7, table=table)
    n, size, d = cache.shape
    wide = torch.empty(n * size * stride, dtype=cache.dtype, device=DEV).view(n, size, stride)[..., 8:8 + d]
    wide.copy_(cache)
    want = _lib.sd_latent_attention(q, cache, ln, dc, pages=pages, scale=0.1)
    got = _lib.sd_latent_attention(q, wide, ln, dc, pages=pages, scale=0.1)
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])
    absorbed._check(q, cache, ln, dc, pages, None, 0.1, want, t, heads=[0, H - 1])


@pytest.mark.parametrize("H", [20, 70])
@pytest.mark.parametrize("stride", [(1 << 24) - 8, 1 << 24])
def test_heads_far_apart(H, stride):
    dc, dr, t = 128, 64, "f16"
    q, cache, ln, pages = absorbed._case(1, 1, H, dc, dr, [200], t, 4)
    qw = torch.empty(1, 1, H, stride, dtype=q.dtype, device=DEV)[..., :dc + dr]
    ow = torch.empty(1, 1, H, stride, dtype=q.dtype, device=DEV)[..., :dc]
    qw.copy_(q)
    want = _lib.sd_latent_attention(q, cache, ln, dc, pages=pages, scale=0.1)
    got = _lib.sd_latent_attention(qw, cache, ln, dc, pages=pages, scale=0.1, out=ow)
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])


@pytest.mark.parametrize("split", [False, True])
@pytest.mark.parametrize("t", list(expanded.TYPES))
def test_expanded_heads_outside_tokens(t, split):
    nq, nk, H, dn, dr, dv = ([150, 40], [230, 64], 3, 128, 64, 128) if not split else ([70], [2100], 2, 96, 32, 80)
    q, k, kr, v, cq, ck = expanded._case(nq, nk, H, dn, dr, dv, t, 9)
    want = _lib.sd_latent_attention_expanded(q, k, kr, v, cq, ck)
    o = torch.full((H, q.shape[0], dv), 3.0, dtype=q.dtype, device=DEV)
    qh, kh, vh = (x.transpose(0, 1).contiguous().transpose(0, 1) for x in (q, k, v))
    got = _lib.sd_latent_attention_expanded(qh, kh, kr, vh, cq, ck, out=o.transpose(0, 1))
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])
    expanded._check(q, k, kr, v, cq, ck, (dn + dr) ** -0.5, want, t, heads=[0, H - 1], rows=[0, 63, 64, 149])


def test_expanded_tokens_far_apart():
    # the widest strides that are taken: a tile of 64 keys spans 2 GB
    H, d, nq, nk, t, stride = 1, 64, 5, 70, "bf16", (1 << 24) - 8
    q, k, kr, v, cq, ck = expanded._case([nq], [nk], H, d, 64, d, t, 11)
    buf = torch.empty(nk, stride, dtype=k.dtype, device=DEV)
    kw, vw, rw = buf[:, None, :d], buf[:, None, 64:64 + d], buf[:, 128:192]
    kw.copy_(k)
    vw.copy_(v)
    rw.copy_(kr)
    want = _lib.sd_latent_attention_expanded(q, k, kr, v, cq, ck)
    got = _lib.sd_latent_attention_expanded(q, kw, rw, vw, cq, ck)
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])
