"""fp16 rows whose weights span many powers of two, both forms of latent attention,
against the float64 oracle.

fp16 has a normal weight down to 2^-14 and steps of 2^-24 below.  The kernels keep a row's
reference 11 powers of two below its largest weight, so weights down to 2^-25 of the
largest are rounded by half a step (2^-11 relative: the bounds of test_gpu_latent.py), and
smaller ones by 2^-25 2^-11 = 2^-36 of the largest at most, which over n keys is less than
n 2^-36 max |v| of the output.
"""
import numpy as np
import pytest
import torch

import test_gpu_latent as absorbed
import test_gpu_latent_expanded as expanded
from oracle import latent as olat
from paper_2606_13426_amd import _lib

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _sink(L, at, gap, dc, g):
    """Vectors of which one, with a value near 0, has a score `gap` above the others' (by the first rotary column)."""
    c = torch.zeros(L, dc + 64, device=DEV)
    c[:, :dc] = torch.randn(L, dc, generator=g, device=DEV).abs() + 0.5
    c[at, :dc] = 0.0
    c[at, dc] = gap
    return c.half()


def _check_out(out, q, key, val, scale, limits):
    """The bounds of test_gpu_latent.py and what small weights may lose."""
    q, key, val = (x.double().cpu().numpy() for x in (q, key, val))
    want, _, mag = olat.attend(q, key, val, scale, limits)
    for i, n in enumerate(limits):
        ds = (q.shape[1] + 5) * absorbed.U * abs(scale) * (np.abs(key[:n]) @ np.abs(q[i])).max()
        tol = 2 * (ds + 2.0 ** -11 + (n + 4) * absorbed.U) * mag[i] + 2.0 ** -11 * np.abs(want[i]) + 2.0 ** -24
        tol = tol + n * 2.0 ** -36 * np.abs(val[:n]).max()
        err = np.abs(out[i].double().cpu().numpy() - want[i])
        assert (err <= tol).all(), (i, n, float((err / tol).max()))


@pytest.mark.parametrize("gap", [14.0, 17.0, 17.625, 22.0])
@pytest.mark.parametrize("at", [0, 3000, 6100])
@pytest.mark.parametrize("H", [16, 64])
def test_absorbed_rows_with_a_sink(H, at, gap):
    # sequences enough that one workgroup walks all of one (parts of a row have references of their own)
    B, dc, L = 260, 128, 6144
    g = torch.Generator(device=DEV)
    g.manual_seed(5)
    c = _sink(L, at, gap, dc, g)
    cache = c.view(L // 64, 64, dc + 64)
    pages = torch.arange(L // 64, device=DEV, dtype=torch.int32)[None].repeat(B, 1)
    q = torch.zeros(B, 1, H, dc + 64, device=DEV, dtype=torch.float16)
    q[..., dc] = 1.0
    lens = torch.full((B,), L, dtype=torch.int32, device=DEV)
    out, _ = _lib.sd_latent_attention(q, cache, lens, dc, pages=pages, scale=1.0)
    for b in (0, 1, B // 2, B - 1):
        _check_out(out[b, 0, [0, H - 1]], q[b, 0, [0, H - 1]], c, c[:, :dc], 1.0, [L, L])


@pytest.mark.parametrize("gap", [14.0, 17.0, 17.625, 22.0])
@pytest.mark.parametrize("at", [0, 3000, 5400])
def test_expanded_rows_with_a_sink(at, gap):
    # heads enough that no keys are split
    H, nq, nk, d = 64, 640, 6144, 128
    assert _lib.sd_latent_attention_expanded_workspace(1, H, d, 64, d, nq, nk) == 0
    g = torch.Generator(device=DEV)
    g.manual_seed(6)
    c = _sink(nk, at, gap, d, g)
    k = torch.zeros(nk, H, d, device=DEV, dtype=torch.float16)
    v = c[:, None, :d].expand(nk, H, d).contiguous()
    q = torch.zeros(nq, H, d + 64, device=DEV, dtype=torch.float16)
    q[..., d] = 1.0
    cq, ck = (torch.tensor([0, n], dtype=torch.int32, device=DEV) for n in (nq, nk))
    out, _ = _lib.sd_latent_attention_expanded(q, k, c[:, d:], v, cq, ck, scale=1.0)
    rows = [0, 63, 300, nq - 1]
    for h in (0, H - 1):
        _check_out(out[rows, h], q[rows, h], c, c[:, :d], 1.0, [nk - nq + 1 + i for i in rows])


@pytest.mark.parametrize("t", list(absorbed.TYPES))
@pytest.mark.parametrize("power", [10, 18, 22, 24])
def test_weights_of_large_scores_stay_finite(t, power):
    """Scores of up to 2^24 that rise by less than a reference moves for: every value is 3, so is
    every output, whatever the weights are (each half a step off, their sum not)."""
    L, dc, H = 1024, 128, 4
    rise = max(2.0, 2.0 ** (power - 23))  # a tile's step, at least a unit in the last place of a score
    c = torch.zeros(L, dc + 64, device=DEV)
    c[:, :dc] = 3.0
    c[:, dc], c[:, dc + 1] = 2.0 ** (power / 2), (torch.arange(L, device=DEV) // 64).float()
    q = torch.zeros(1, 1, H, dc + 64, device=DEV)
    q[..., dc], q[..., dc + 1] = 2.0 ** (power / 2), rise
    c, q = c.to(absorbed.TYPES[t]), q.to(absorbed.TYPES[t])
    lens = torch.full((200,), L, dtype=torch.int32, device=DEV)
    pages = torch.arange(L // 64, device=DEV, dtype=torch.int32)[None].repeat(200, 1)
    out, lse = _lib.sd_latent_attention(q.expand(200, 1, H, dc + 64).contiguous(), c.view(-1, 64, dc + 64), lens, dc,
                                        pages=pages, scale=1.0)
    e = absorbed._half_step(t)
    assert ((out.float() - 3.0).abs() <= 3 * 3.1 * e).all() and torch.isfinite(lse).all()
    k = torch.zeros(L, H, dc, device=DEV, dtype=c.dtype)
    v = torch.full((L, H, dc), 3.0, device=DEV, dtype=c.dtype)
    cu = [torch.tensor([0, n], dtype=torch.int32, device=DEV) for n in (1, L)]
    out, lse = _lib.sd_latent_attention_expanded(q[0], k, c[:, dc:], v, cu[0], cu[1], scale=1.0)
    assert ((out.float() - 3.0).abs() <= 3 * 3.1 * e).all() and torch.isfinite(lse).all()


def test_fp16_rows_of_random_scores():
    # spread scores (up to about 30 nats below the largest), the bounds of the forms' own tests
    q, cache, ln, pages = absorbed._case(2, 3, 20, 256, 64, [1500, 700], "f16", 17, page=16, spread=4.0)
    got = _lib.sd_latent_attention(q, cache, ln, 256, pages=pages, scale=320 ** -0.5)
    absorbed._check(q, cache, ln, 256, pages, None, 320 ** -0.5, got, "f16", heads=[0, 7, 19])
    q, k, kr, v, cq, ck = expanded._case([300, 70], [900, 70], 3, 128, 64, 128, "f16", 18)
    got = _lib.sd_latent_attention_expanded(q * 4, k, kr, v, cq, ck, scale=192 ** -0.5)
    expanded._check(q * 4, k, kr, v, cq, ck, 192 ** -0.5, got, "f16", rows=[0, 64, 150, 299])
