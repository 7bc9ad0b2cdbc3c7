"""sd_latent_attention against the float64 oracle on the same 16-bit inputs.

With u = 2^-24 and e half a step of the type: a score is a float32 sum of exact
products, off by at most (d + 2) u sum |q c| |scale| (any order), times log2(e)
and back another 3 u |s|; a weight moves by that relative amount, is rounded by e
relative, and the sums over n tokens by n u; so out is off by at most
(ds + e + n u + 4 u) sum_j p_j |v_j| twice (weights and their sum), and e of
itself.  The parts of a split sequence add no more than n u.
"""
import numpy as np
import pytest
import torch

from oracle import latent as olat
from paper_2606_13426_amd import _lib

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


def _half_step(t):
    return torch.finfo(TYPES[t]).eps / 2


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def _case(B, Q, H, dc, dr, lens, t, seed, page=16, table=True, spread=1.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    lens = list(lens)
    per = [max(1, -(-max(n, 0) // page)) for n in lens]
    n_pages = (sum(per) + 2) if table else B
    size = page if table else max(max(lens), 1)
    q = (_randn(g, B, Q, H, dc + dr) * spread).to(TYPES[t])
    cache = _randn(g, n_pages, size, dc + dr).to(TYPES[t])
    pages = None
    if table:
        order = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
        pages = torch.full((B, max(per)), -7, dtype=torch.int32, device=DEV)  # never read past a sequence's pages
        at = 0
        for b, n in enumerate(per):
            pages[b, :n] = order[at:at + n]
            at += n
    return q, cache, torch.tensor(lens, dtype=torch.int32, device=DEV), pages


def _check(q, cache, lens, dc, pages, rows, scale, got, t, seqs=None, heads=None):
    out, lse = (x.double().cpu().numpy() for x in got)
    qn, cn, ln = q.double().cpu().numpy(), cache.double().cpu().numpy(), lens.cpu().numpy()
    B, Q, H, d = qn.shape
    e = _half_step(t)
    for b in range(B) if seqs is None else seqs:
        n = min(max(int(ln[b]), 0), cn.shape[1] if pages is None else pages.shape[1] * cn.shape[1])
        nb = Q if rows is None else min(max(int(rows[b]), 0), Q)
        table = [b] if pages is None else pages[b].cpu().numpy()
        c, have = olat.gather(cn, table, n)
        for h in range(H) if heads is None else heads:
            lim = [n - nb + i + 1 for i in range(nb)]
            seen = [int(have[:max(0, min(v, n))].sum()) for v in lim]
            w, wl, mag = olat.attend(qn[b, :nb, h], c[have], c[have][:, :dc], scale, seen)
            for i in range(nb):
                if seen[i] == 0:
                    assert (out[b, i, h] == 0).all() and lse[b, i, h] == -np.inf, (b, i, h)
                    continue
                s = abs(scale) * (np.abs(c[have][:seen[i]]) @ np.abs(qn[b, i, h]))
                ds = (d + 5) * U * s.max()
                if np.isnan(wl[i]):
                    assert np.isnan(lse[b, i, h]) and np.isnan(out[b, i, h]).all()
                    continue
                assert abs(lse[b, i, h] - wl[i]) <= ds + (seen[i] + 4) * U + U * abs(wl[i]), (b, i, h, lse[b, i, h], wl[i])
                tol = 2 * (ds + e + (seen[i] + 4) * U) * mag[i] + e * np.abs(w[i])
                tol = tol + (2.0 ** -24 if t == "f16" else 0.0)  # fp16's smallest step: weights and outputs below its normal range
                err = np.abs(out[b, i, h] - w[i])
                assert (err <= tol).all(), (b, i, h, float((err / tol).max()))


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("B,Q,H,dc,dr,page,lens", [
    (1, 1, 1, 8, 0, 4, [1]), (1, 1, 16, 512, 64, 64, [777]), (3, 1, 5, 128, 64, 16, [0, 1, 64]),
    (2, 1, 16, 512, 64, 1, [63, 65]), (2, 3, 7, 256, 32, 48, [130, 2]), (1, 9, 4, 512, 64, 100, [3]),
    (4, 2, 16, 384, 64, 64, [200, 64, 128, 1]), (2, 5, 13, 136, 40, 7, [129, 300]), (1, 17, 8, 504, 8, 33, [1000]),
    (2, 1, 128, 512, 64, 64, [515, 90]), (3, 3, 16, 64, 16, 5, [70, -4, 9]), (2, 2, 96, 512, 64, 64, [320, 190]),
    (300, 1, 4, 128, 0, 16, [(37 * i) % 150 for i in range(300)]), (5, 9, 32, 256, 64, 64, [700, 9, 1, 650, 64])])
def test_latent_attention(B, Q, H, dc, dr, page, lens, t):
    q, cache, ln, pages = _case(B, Q, H, dc, dr, lens, t, B * 10 + Q, page)
    scale = (dc + dr) ** -0.5
    got = _lib.sd_latent_attention(q, cache, ln, dc, pages=pages)
    _check(q, cache, ln, dc, pages, None, scale, got, t, seqs=None if B < 10 else range(0, B, 23),
           heads=None if H < 20 else [0, 1, H // 2, H - 1])


@pytest.mark.parametrize("scale", [0.9, -0.05, 0.0])
def test_scales(scale):
    q, cache, ln, pages = _case(2, 2, 3, 128, 64, [150, 70], "bf16", 5)
    got = _lib.sd_latent_attention(q, cache, ln, 128, pages=pages, scale=scale)
    _check(q, cache, ln, 128, pages, None, scale, got, "bf16")


@pytest.mark.parametrize("B,Q,H,lens", [(1, 1, 16, [20000]), (2, 4, 32, [16000, 333]), (1, 2, 128, [9000])])
def test_long_sequences_are_split_and_joined(B, Q, H, lens):
    q, cache, ln, pages = _case(B, Q, H, 512, 64, lens, "bf16", 3, page=64)
    got = _lib.sd_latent_attention(q, cache, ln, 512, pages=pages)
    _check(q, cache, ln, 512, pages, None, 576 ** -0.5, got, "bf16", heads=[0, H - 1])


def test_plain_cache_and_views():
    # no table; q, cache and out as views of larger buffers, heads outside rows
    B, Q, H, dc, dr, L, t = 3, 2, 4, 256, 64, 200, "f16"
    g = torch.Generator(device=DEV)
    g.manual_seed(8)
    q = _randn(g, B, H, Q, dc + dr + 8).to(TYPES[t])[..., 8:].transpose(1, 2)
    cache = _randn(g, B + 1, L, 2, dc + dr).to(TYPES[t])[:B, :, 1]
    ln = torch.tensor([200, 131, 900], dtype=torch.int32, device=DEV)  # the last is clamped to the page
    out = torch.full((B, H, Q, dc + 16), 9.0, dtype=TYPES[t], device=DEV)
    got = _lib.sd_latent_attention(q, cache, ln, dc, out=out[..., 16:].transpose(1, 2))
    _check(q, cache, ln, dc, None, None, (dc + dr) ** -0.5, got, t)
    assert (out[..., :16] == 9.0).all()


def test_rows_past_a_sequences_own_are_left_as_they_were():
    B, Q, H, dc = 5, 4, 6, 128
    q, cache, ln, pages = _case(B, Q, H, dc, 64, [300, 2, 0, 65, 40], "bf16", 4)
    rows = torch.tensor([2, 4, 3, 0, 99], dtype=torch.int32, device=DEV)
    q[0, 2:] = float("nan")
    q[3] = float("nan")
    out = torch.full((B, Q, H, dc), 7.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((B, Q, H), 7.0, device=DEV)
    got = _lib.sd_latent_attention(q, cache, ln, dc, pages=pages, rows=rows, out=out, lse=lse)
    _check(q, cache, ln, dc, pages, rows, (dc + 64) ** -0.5, got, "bf16")
    assert (out[0, 2:] == 7).all() and (lse[0, 2:] == 7).all() and (out[3] == 7).all() and (lse[3] == 7).all()


def test_pages_that_do_not_exist_hold_no_tokens():
    q, cache, ln, pages = _case(3, 2, 5, 128, 64, [150, 150, 40], "bf16", 6)
    n = cache.shape[0]
    pages[0, 2], pages[0, 4], pages[1, 0], pages[1, 9] = -1, n, 2 ** 31 - 1, -2 ** 31
    pages[2] = -1
    got = _lib.sd_latent_attention(q, cache, ln, 128, pages=pages)
    _check(q, cache, ln, 128, pages, None, 192 ** -0.5, got, "bf16")
    assert (got[0][2] == 0).all() and (got[1][2] == -float("inf")).all()


@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
@pytest.mark.parametrize("t", list(TYPES))
def test_what_a_row_does_not_see_has_no_part_in_it(t, bad):
    B, Q, H, dc, page = 2, 5, 24, 256, 16
    q, cache, ln, pages = _case(B, Q, H, dc, 64, [203, 66], t, 7, page)
    want = _lib.sd_latent_attention(q, cache, ln, dc, pages=pages)
    dirty = cache.clone()
    used = torch.zeros(cache.shape[:2], dtype=torch.bool, device=DEV)
    for b, n in enumerate(ln.tolist()):
        for j in range(n):
            used[pages[b, j // page], j % page] = True
    dirty[~used] = bad  # places behind the sequences' last tokens, and pages of nobody
    got = _lib.sd_latent_attention(q, dirty, ln, dc, pages=pages)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    # the last draft's vector: only the last row sees it
    for b, n in enumerate(ln.tolist()):
        dirty[pages[b, (n - 1) // page], (n - 1) % page] = bad
    got = _lib.sd_latent_attention(q, dirty, ln, dc, pages=pages)
    assert torch.isfinite(got[0][:, :-1].float()).all() and torch.isnan(got[0][:, -1].float()).any()
    e = _half_step(t)
    assert ((got[0] - want[0]).abs()[:, :-1].double() <= 4 * e * want[0].abs().double().amax()[None]).all()
    assert torch.equal(got[1][:, :-1], want[1][:, :-1])


def test_a_nan_that_is_seen_shows():
    q, cache, ln, pages = _case(1, 1, 2, 128, 64, [100], "bf16", 9)
    cache[pages[0, 1], 3, 140] = float("nan")  # the rotary part: only the score
    out, lse = _lib.sd_latent_attention(q, cache, ln, 128, pages=pages)
    assert torch.isnan(out.float()).all() and torch.isnan(lse).all()


def test_offsets_past_32_bits():
    # a cache of 5 GB, its tokens at both ends
    dc, dr, page = 512, 64, 64
    n_pages = 72000
    cache = torch.zeros(n_pages, page, dc + dr, dtype=torch.bfloat16, device=DEV)
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    ids = torch.tensor([n_pages - 1, 0, n_pages - 2, 36500, 58255], device=DEV)
    small = _randn(g, len(ids), page, dc + dr).to(torch.bfloat16)
    cache[ids] = small
    q = _randn(g, 1, 1, 16, dc + dr).to(torch.bfloat16)
    ln = torch.tensor([300], dtype=torch.int32, device=DEV)
    big = _lib.sd_latent_attention(q, cache, ln, dc, pages=ids[None].to(torch.int32))
    order = torch.arange(len(ids), device=DEV, dtype=torch.int32)[None]
    few = _lib.sd_latent_attention(q, small, ln, dc, pages=order)
    assert torch.equal(big[0], few[0]) and torch.equal(big[1], few[1])


def test_calls_repeat_to_the_bit_and_replay_in_a_graph():
    B, Q, H, dc = 3, 2, 20, 512
    q, cache, ln, pages = _case(B, Q, H, dc, 64, [3000, 70, 1500], "bf16", 12)
    ws = torch.empty(_lib.sd_latent_attention_workspace(B, Q, H, dc, 64), dtype=torch.uint8, device=DEV)
    want = [x.clone() for x in _lib.sd_latent_attention(q, cache, ln, dc, pages=pages, ws=ws)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = _lib.sd_latent_attention(q, cache, ln, dc, pages=pages)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, other))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = _lib.sd_latent_attention(q, cache, ln, dc, pages=pages, ws=ws)
    for i in range(3):
        ws.fill_(0xFF)
        for x in held:
            x.fill_(-3)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, held)), i
    ln.copy_(torch.tensor([10, 2900, 0], dtype=torch.int32))  # other lengths, the same graph
    want = [x.clone() for x in _lib.sd_latent_attention(q, cache, ln, dc, pages=pages[:, :], ws=ws)]
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, held))


@pytest.mark.parametrize("tokens", [300, 2 ** 18, 2 ** 22])
@pytest.mark.parametrize("B,Q,H,dc,dr,lens", [
    (3, 1, 64, 512, 64, [515, 90, 0]), (2, 3, 33, 512, 64, [290, 3]), (1, 9, 32, 256, 64, [300]), (2, 2, 16, 128, 32, [64, 200]),
    (2, 1, 200, 384, 64, [128, 129]), (5, 1, 17, 512, 64, [63, 0, 65, 1, 300])])
def test_tables_of_every_width(B, Q, H, dc, dr, lens, tokens):
    """The rows a workgroup takes go by what the table's pages could hold; what stands past the sequences' own
    pages is never read."""
    q, cache, ln, pages = _case(B, Q, H, dc, dr, lens, "bf16", 20 + B, page=16)
    wide = torch.full((B, max(tokens // 16, pages.shape[1])), -7, dtype=torch.int32, device=DEV)
    wide[:, :pages.shape[1]] = pages
    ws = torch.full((_lib.sd_latent_attention_workspace(B, Q, H, dc, dr) + 4096,), 0x5A, dtype=torch.uint8, device=DEV)
    got = _lib.sd_latent_attention(q, cache, ln, dc, pages=wide, ws=ws[:-4096])
    _check(q, cache, ln, dc, pages, None, (dc + dr) ** -0.5, got, "bf16", heads=[0, 1, H // 2, H - 1])
    assert (ws[-4096:] == 0x5A).all()
    # an infinity in the last token: only the last row sees it
    for b, n in enumerate(lens):
        if n:
            cache[pages[b, (n - 1) // 16], (n - 1) % 16, 3] = float("inf")
    out, lse = _lib.sd_latent_attention(q, cache, ln, dc, pages=wide)
    if Q > 1:
        assert torch.isfinite(out[:, :-1].float()).all()


@pytest.mark.parametrize("tokens", [300, 2 ** 18, 2 ** 22])
@pytest.mark.parametrize("B,Q,H,order", [(3, 2, 40, "heads first"), (2, 3, 31, "gaps"), (2, 1, 70, "gaps"), (1, 5, 13, "rows apart")])
def test_views_of_q_and_of_the_output(B, Q, H, order, tokens):
    """Orders and strides of q and out that a workgroup's rows do not lie level in, and such that they do."""
    dc, dr, t = 256, 64, "bf16"
    d = dc + dr
    q, cache, ln, pages = _case(B, Q, H, dc, dr, [170, 65, 9][:B], t, 30 + B, page=16)
    wide = torch.full((B, max(tokens // 16, pages.shape[1])), -7, dtype=torch.int32, device=DEV)
    wide[:, :pages.shape[1]] = pages
    if order == "heads first":
        qv, shape = q.transpose(1, 2).contiguous().transpose(1, 2), (B, H, Q, dc)
        ov = lambda x: x.transpose(1, 2)  # noqa: E731
    elif order == "gaps":
        qv = torch.full((B, Q, H, d + 24), 5.0, dtype=q.dtype, device=DEV)[..., 8:8 + d]
        qv.copy_(q)
        shape, ov = (B, Q, H, dc + 8), lambda x: x[..., :dc]
    else:
        qv = torch.full((B, 2 * Q + 1, H, d), 5.0, dtype=q.dtype, device=DEV)[:, 1::2]
        qv.copy_(q)
        shape, ov = (B, 2 * Q, H, dc), lambda x: x[:, ::2]
    out = torch.full(shape, 3.0, dtype=q.dtype, device=DEV)
    got = _lib.sd_latent_attention(qv, cache, ln, dc, pages=wide, out=ov(out))
    _check(q, cache, ln, dc, pages, None, d ** -0.5, got, t, heads=[0, 1, H // 2, H - 1])
    ov(out).fill_(3.0)
    assert (out == 3.0).all()
