"""sd_latent_attention_tree against the float64 oracle; the bounds are those of test_gpu_latent.py,
a row's tokens being the prefix, itself and its ancestors."""
import numpy as np
import pytest
import torch

import test_gpu_latent as chain
from oracle import latent as olat
from oracle import tree
from paper_2606_13426_amd import _lib

pytestmark = pytest.mark.gpu
DEV, U, TYPES = "cuda", chain.U, chain.TYPES


def _grown(seed, B, Q, wide=3):
    r = np.random.default_rng(seed)
    return [[-1] + [int(r.integers(max(0, (i - 1) // wide - 1), i)) for i in range(1, Q)] for _ in range(B)]


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _check(q, cache, lens, parents, dc, pages, rows, scale, got, t, seqs=None, heads=None):
    out, lse = (x.double().cpu().numpy() for x in got)
    qn, cn = q.double().cpu().numpy(), cache.double().cpu().numpy()
    B, Q, H, d = qn.shape
    e = chain._half_step(t)
    for b in range(B) if seqs is None else seqs:
        n = min(max(int(lens[b]), 0), cn.shape[1] if pages is None else pages.shape[1] * cn.shape[1])
        nb = Q if rows is None else min(max(int(rows[b]), 0), Q)
        c, have = olat.gather(cn, [b] if pages is None else pages[b].cpu().numpy(), n)
        kin = tree.sees([int(p) for p in parents[b]], nb)
        for i in range(nb):
            see = np.zeros(n, bool)
            see[:max(n - nb, 0)] = True
            for j in np.nonzero(kin[i])[0]:
                if n - nb + j >= 0:
                    see[n - nb + j] = True
            see &= have
            k = c[see]
            for h in range(H) if heads is None else heads:
                w, wl, mag = (x[0] for x in olat.attend(qn[b, i, h][None], k, k[:, :dc], scale, [len(k)]))
                if len(k) == 0:
                    assert (out[b, i, h] == 0).all() and lse[b, i, h] == -np.inf, (b, i, h)
                    continue
                if np.isnan(wl):
                    assert np.isnan(lse[b, i, h]) and np.isnan(out[b, i, h]).all()
                    continue
                ds = (d + 5) * U * abs(scale) * (np.abs(k) @ np.abs(qn[b, i, h])).max()
                assert abs(lse[b, i, h] - wl) <= ds + (len(k) + 4) * U + U * abs(wl), (b, i, h, lse[b, i, h], wl)
                tol = 2 * (ds + e + (len(k) + 4) * U) * mag + e * np.abs(w) + (2.0 ** -24 if t == "f16" else 0.0)
                same = (out[b, i, h] == w) | (np.isnan(out[b, i, h]) & np.isnan(w))  # (infinite values)
                with np.errstate(invalid="ignore"):
                    assert (same | (np.abs(out[b, i, h] - w) <= tol)).all(), (b, i, h)


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("B,Q,H,dc,dr,page,lens", [
    (1, 1, 1, 8, 0, 4, [1]), (1, 2, 16, 512, 64, 64, [2]), (3, 5, 5, 128, 64, 16, [0, 5, 64]), (2, 16, 16, 512, 64, 1, [63, 130]),
    (2, 64, 4, 256, 32, 48, [64, 150]), (1, 9, 4, 512, 64, 100, [3]), (4, 33, 3, 384, 64, 64, [200, 97, 128, 33]),
    (2, 7, 13, 136, 40, 7, [129, 300]), (2, 20, 32, 512, 64, 64, [515, 90]), (3, 64, 1, 64, 16, 5, [70, -4, 91]),
    (150, 3, 4, 128, 0, 16, [(37 * i) % 150 for i in range(150)]), (1, 31, 64, 504, 8, 33, [1000]),
    (5, 9, 48, 256, 64, 64, [700, 9, 64, 650, 73])])
def test_tree_attention(B, Q, H, dc, dr, page, lens, t):
    q, cache, ln, pages = chain._case(B, Q, H, dc, dr, lens, t, B * 10 + Q, page)
    parents = _grown(B + Q, B, Q)
    got = _lib.sd_latent_attention_tree(q, cache, ln, _i32(parents), dc, pages=pages, scale=(dc + dr) ** -0.5)
    _check(q, cache, lens, parents, dc, pages, None, (dc + dr) ** -0.5, got, t, seqs=None if B < 10 else range(0, B, 23),
           heads=None if H < 10 else [0, H // 2, H - 1])


@pytest.mark.parametrize("B,Q,H,lens", [(1, 16, 4, [20000]), (2, 32, 32, [9000, 4133])])
def test_long_sequences_are_split_and_joined(B, Q, H, lens):
    q, cache, ln, pages = chain._case(B, Q, H, 512, 64, lens, "bf16", 3, page=64)
    parents = _grown(5, B, Q)
    got = _lib.sd_latent_attention_tree(q, cache, ln, _i32(parents), 512, pages=pages, scale=0.07)
    _check(q, cache, lens, parents, 512, pages, None, 0.07, got, "bf16", heads=[0, H - 1])


def test_a_chain_of_nodes_is_the_chain_form():
    for B, Q, H, lens in ((2, 9, 32, [700, 64]), (3, 64, 2, [64, 128, 65]), (1, 5, 4, [130])):
        q, cache, ln, pages = chain._case(B, Q, H, 512, 64, lens, "bf16", 7, page=48)
        parents = _i32([list(range(-1, Q - 1))] * B)
        want = _lib.sd_latent_attention(q, cache, ln, 512, pages=pages, scale=0.07)
        got = _lib.sd_latent_attention_tree(q, cache, ln, parents, 512, pages=pages, scale=0.07)
        assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])


def test_parents_of_no_node_and_rows_past_a_sequences_own():
    B, Q, H, dc = 5, 6, 6, 128
    parents = [[7, 0, 5, -1, 3, 2 ** 31 - 1], [-2 ** 31, 1, 0, 2, 4, 4], [0, 0, 0, 0, 0, 0], [-1, 0, 1, 2, 3, 4], [9, 9, 9, 9, 9, 9]]
    lens, rows = [300, 4, 0, 65, 40], [6, 4, 3, 0, 99]
    q, cache, ln, pages = chain._case(B, Q, H, dc, 64, lens, "bf16", 4)
    q[1, 4:] = float("nan")
    q[3] = float("nan")
    out, lse = torch.full((B, Q, H, dc), 7.0, dtype=torch.bfloat16, device=DEV), torch.full((B, Q, H), 7.0, device=DEV)
    got = _lib.sd_latent_attention_tree(q, cache, ln, _i32(parents), dc, pages=pages, rows=_i32(rows), scale=0.07, out=out, lse=lse)
    _check(q, cache, lens, parents, dc, pages, rows, 0.07, got, "bf16")
    assert (out[1, 4:] == 7).all() and (lse[1, 4:] == 7).all() and (out[3] == 7).all() and (lse[3] == 7).all()


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("H", [2, 40])
def test_values_that_are_no_numbers_in_nodes_others_do_not_see(H, t):
    """Nodes hold NaN, infinities and the type's largest value: only they and their descendants know of them."""
    B, Q, dc = 2, 12, 256
    lens = [150, 12]
    q, cache, ln, pages = chain._case(B, Q, H, dc, 64, lens, t, 6)
    parents = [[-1, 0, 0, 1, 1, 2, 2, 3, 5, 5, 8, 4]] * 2
    for b in range(B):
        for node, value in ((3, float("nan")), (6, float("inf")), (9, -float("inf")), (11, torch.finfo(TYPES[t]).min)):
            j = lens[b] - Q + node
            cache[pages[b, j // 16], j % 16, 5::64] = value
    got = _lib.sd_latent_attention_tree(q, cache, ln, _i32(parents), dc, pages=pages, scale=0.05)
    clean = [i for i in range(Q) if i not in (3, 7, 6, 9, 11)]
    assert torch.isfinite(got[0][:, clean].float()).all() and torch.isfinite(got[1][:, clean]).all()
    assert torch.isnan(got[0][:, [3, 7]].float()).all()
    keep = cache.clone()
    keep[~torch.isfinite(keep)] = 0  # what the clean rows see does not depend on it
    keep[keep == torch.finfo(TYPES[t]).min] = 0
    again = _lib.sd_latent_attention_tree(q, keep, ln, _i32(parents), dc, pages=pages, scale=0.05)
    assert torch.equal(again[0][:, clean], got[0][:, clean]) and torch.equal(again[1][:, clean], got[1][:, clean])
    _check(q[:, clean[:3]], cache, [n - Q + 3 for n in lens], [p[:3] for p in parents], dc, pages, None, 0.05,
           tuple(x[:, clean[:3]] for x in got), t)


def test_pages_that_do_not_exist_plain_caches_and_views():
    q, cache, ln, pages = chain._case(3, 8, 5, 128, 64, [150, 150, 40], "bf16", 6)
    parents = _grown(3, 3, 8)
    pages[0, 9], pages[0, 2], pages[1, 0], pages[2, 2] = -1, cache.shape[0], 2 ** 31 - 1, -2 ** 31
    got = _lib.sd_latent_attention_tree(q, cache, ln, _i32(parents), 128, pages=pages, scale=-0.1)
    _check(q, cache, [150, 150, 40], parents, 128, pages, None, -0.1, got, "bf16")
    B, Q, H, dc, L = 3, 6, 4, 256, 200
    g = torch.Generator(device=DEV)
    g.manual_seed(8)
    q = torch.randn(B, H, Q, dc + 72, generator=g, device=DEV).half()[..., 8:].transpose(1, 2)
    cache = torch.randn(B + 1, L, 2, dc + 64, generator=g, device=DEV).half()[:B, :, 1]
    out = torch.full((B, H, Q, dc + 16), 9.0, dtype=torch.float16, device=DEV)
    parents, lens = _grown(9, B, Q), [200, 131, 900]
    got = _lib.sd_latent_attention_tree(q, cache, _i32(lens), _i32(parents), dc, scale=0.05, out=out[..., 16:].transpose(1, 2))
    _check(q, cache, lens, parents, dc, None, None, 0.05, got, "f16")
    assert (out[..., :16] == 9.0).all()


# The kernel of 128 rows a workgroup is chosen by the tokens that the table has room for, which
# these sequences do not fill.
def _roomy(pages, page, B, rows):
    blocks = B * (-(-rows // 128))
    width = -(-64 * (5120 // blocks + 1) // page)
    return torch.cat([pages, torch.full((B, max(0, width - pages.shape[1])), -7, dtype=torch.int32, device=DEV)], 1)


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("B,Q,H,page,lens,rows", [
    (1, 16, 8, 64, [16], None), (1, 16, 8, 64, [31], None), (1, 16, 8, 33, [150], None), (2, 17, 9, 7, [200, 61], None),
    (3, 64, 2, 1, [64, 97, 130], None), (5, 20, 16, 48, [515, 20, 0, 7, -3], [20, 3, 9, 20, 5]), (2, 33, 4, 100, [1000, 40], [33, 1]),
    (70, 8, 16, 16, [(37 * b) % 150 + 3 for b in range(70)], [b % 10 - 1 for b in range(70)]), (1, 64, 128, 64, [3000], None),
    (4, 32, 12, 64, [700, 641, 32, 2100], [32, 7, 32, 20])])
def test_many_rows(B, Q, H, page, lens, rows, t):
    q, cache, ln, pages = chain._case(B, Q, H, 512, 64, lens, t, B * 10 + Q, page)
    pages = _roomy(pages, page, B, Q * H)
    parents = _grown(B + Q, B, Q)
    out, lse = torch.full((B, Q, H, 512), 7.0, dtype=TYPES[t], device=DEV), torch.full((B, Q, H), 7.0, device=DEV)
    _lib.sd_profile_enable(True)
    got = _lib.sd_latent_attention_tree(q, cache, ln, _i32(parents), 512, pages=pages, scale=0.06, out=out, lse=lse,
                                        rows=None if rows is None else _i32(rows))
    torch.cuda.synchronize()
    _lib.sd_profile_enable(False)
    assert "latent_wide" in _lib.sd_profile_read()
    _check(q, cache, lens, parents, 512, pages, rows, 0.06, got, t, seqs=None if B < 10 else range(0, B, 9),
           heads=None if H < 5 else [0, H // 2, H - 1])
    for b in range(B):
        n = Q if rows is None else min(max(rows[b], 0), Q)
        assert (out[b, n:] == 7).all() and (lse[b, n:] == 7).all()


@pytest.mark.parametrize("t", list(TYPES))
def test_many_rows_values_that_are_no_numbers(t):
    """As above with nodes that hold NaN, infinities and the lowest value, in cut and in whole blocks."""
    for lens in ([150, 16], [1000, 90]):
        B, Q, H = 2, 16, 24
        q, cache, ln, pages = chain._case(B, Q, H, 512, 64, lens, t, 6)
        pages = _roomy(pages, 16, B, Q * H)
        parents = [[-1, 0, 0, 1, 1, 2, 2, 3, 5, 5, 8, 4, 10, 12, 9, 6]] * B
        bad = {3: float("nan"), 6: float("inf"), 9: -float("inf"), 11: torch.finfo(TYPES[t]).min}
        for b in range(B):
            for node, value in bad.items():
                j = lens[b] - Q + node
                cache[pages[b, j // 16], j % 16, 5::64] = value
        got = _lib.sd_latent_attention_tree(q, cache, ln, _i32(parents), 512, pages=pages, scale=0.05)
        kin = tree.sees(parents[0], Q)
        clean = [i for i in range(Q) if not any(kin[i, n] for n in bad)]
        assert torch.isfinite(got[0][:, clean].float()).all() and torch.isfinite(got[1][:, clean]).all()
        assert torch.isnan(got[0][:, [3, 7]].float()).all()
        keep = cache.clone()
        keep[~torch.isfinite(keep) | (keep == torch.finfo(TYPES[t]).min)] = 0
        again = _lib.sd_latent_attention_tree(q, keep, ln, _i32(parents), 512, pages=pages, scale=0.05)
        assert torch.equal(again[0][:, clean], got[0][:, clean]) and torch.equal(again[1][:, clean], got[1][:, clean])
        _check(q[:, :3], keep, [n - Q + 3 for n in lens], [p[:3] for p in parents], 512, pages, None, 0.05,
               tuple(x[:, :3] for x in got), t, heads=[0, 23])
        # an infinite value of positive weight stays one: only the latent part of node 9 is, not what its scores are of
        cache[~torch.isfinite(cache) | (cache == torch.finfo(TYPES[t]).min)] = 0
        q[..., 7] = 0
        for b in range(B):
            j = lens[b] - Q + 5
            cache[pages[b, j // 16], j % 16, 7] = float("inf")
        sees5 = [i for i in range(Q) if kin[i, 5]]
        got = _lib.sd_latent_attention_tree(q, cache, ln, _i32(parents), 512, pages=pages, scale=0.05)
        rest = [i for i in range(Q) if not kin[i, 5]]
        assert torch.isfinite(got[0][:, rest].float()).all() and torch.isnan(got[0][:, sees5].float()).all()


def test_many_rows_missing_pages_views_and_scales():
    B, Q, H, dc, t = 2, 24, 6, 512, "f16"
    g = torch.Generator(device=DEV)
    g.manual_seed(8)
    for scale in (-0.04, 0.0):
        q = torch.randn(B, H, Q, dc + 72, generator=g, device=DEV).half()[..., 8:].transpose(1, 2)
        cache = torch.randn(40, 16, 2, dc + 64, generator=g, device=DEV).half()[:, :, 1]
        out = torch.full((B, H, Q, dc + 16), 9.0, dtype=torch.float16, device=DEV)
        pages = torch.randperm(40, generator=g, device=DEV)[:36].view(B, 18).int()
        pages[0, 3], pages[0, 16], pages[1, 0] = -1, 40, 2 ** 31 - 1
        pages = _roomy(pages, 16, B, Q * H)
        parents, lens = _grown(9, B, Q), [280, 131]
        got = _lib.sd_latent_attention_tree(q, cache, _i32(lens), _i32(parents), dc, pages=pages, scale=scale,
                                            out=out[..., 16:].transpose(1, 2))
        _check(q, cache, lens, parents, dc, pages, None, scale, got, t)
        assert (out[..., :16] == 9.0).all()


def test_many_rows_of_many_trees():
    """256 blocks of rows, mostly whole, and strides of 2^24 elements."""
    B, Q, H = 8, 32, 128
    lens = [150, 40, 32, 700, 90, 64, 33, 500]
    q, cache, ln, pages = chain._case(B, Q, H, 512, 64, lens, "bf16", 12, page=64)
    parents = _grown(3, B, Q)
    got = _lib.sd_latent_attention_tree(q, cache, ln, _i32(parents), 512, pages=pages, scale=0.06)
    _check(q, cache, lens, parents, 512, pages, None, 0.06, got, "bf16", seqs=[0, 2, 3, 6], heads=[0, 77, 127])
    far = torch.empty(40, 1 << 24, dtype=torch.bfloat16, device=DEV)[:, :576]
    far.copy_(torch.randn(40, 576, device=DEV))
    q = q[:1, :16, :8].contiguous()
    table = _roomy(_i32([[(7 * j) % 40 for j in range(40)]]), 1, 1, 128)
    got = _lib.sd_latent_attention_tree(q, far[:, None], _i32([40]), _i32(_grown(4, 1, 16)), 512, pages=table, scale=0.06)
    _check(q, far[:, None], [40], _grown(4, 1, 16), 512, table, None, 0.06, got, "bf16")
    got = _lib.sd_latent_attention_tree(q, far[None], _i32([40]), _i32(_grown(4, 1, 16)), 512, scale=0.06)
    _check(q, far[None], [40], _grown(4, 1, 16), 512, None, None, 0.06, got, "bf16")


@pytest.mark.parametrize("B,Q,H,longest", [(48, 64, 16, 300), (130, 33, 12, 200), (20, 60, 32, 520), (300, 16, 8, 90)])
def test_many_rows_in_blocks_that_are_not_cut(B, Q, H, longest):
    lens = [longest - (b * 41) % (longest - 3) if b % 7 else [0, Q, -2, longest][b // 7 % 4] for b in range(B)]
    rows = [Q - (b * 5) % Q if b % 5 else [Q, 0, Q + 3, -1][b // 5 % 4] for b in range(B)]
    q, cache, ln, pages = chain._case(B, Q, H, 512, 64, lens, "bf16", 31, page=16)
    pages = _roomy(pages, 16, B, Q * H)
    parents = _grown(41, B, Q)
    out, lse = torch.full((B, Q, H, 512), 7.0, dtype=torch.bfloat16, device=DEV), torch.full((B, Q, H), 7.0, device=DEV)
    got = _lib.sd_latent_attention_tree(q, cache, ln, _i32(parents), 512, pages=pages, scale=0.06, rows=_i32(rows), out=out, lse=lse)
    seqs = sorted({0, 1, 5, 7, 14, 21, B // 2, B - 2, B - 1} & set(range(B)))
    _check(q, cache, lens, parents, 512, pages, rows, 0.06, got, "bf16", seqs=seqs, heads=[0, H - 1])
    for b in range(B):
        n = min(max(rows[b], 0), Q)
        assert (out[b, n:] == 7).all() and (lse[b, n:] == 7).all() and torch.isfinite(out[b, :n].float()).all()


def test_many_rows_in_a_graph_and_on_two_streams():
    """Replays see new queries, lengths and trees; a workspace holds nothing of the call before."""
    B, Q, H, dc, t = 3, 24, 32, 512, "bf16"
    lens = [900, 333, 1500]
    q, cache, ln, pages = chain._case(B, Q, H, dc, 64, lens, t, 44, page=48)
    pages = _roomy(pages, 48, B, Q * H)
    parents = _i32(_grown(6, B, Q))
    ws = torch.empty(_lib.sd_latent_attention_tree_workspace(B, Q, H, dc, 64), dtype=torch.uint8, device=DEV)
    other = torch.empty_like(ws)
    outs = [torch.zeros(B, Q, H, dc, dtype=TYPES[t], device=DEV) for _ in range(3)]
    lses = [torch.zeros(B, Q, H, device=DEV) for _ in range(3)]

    def call(k, w):
        return _lib.sd_latent_attention_tree(q, cache, ln, parents, dc, pages=pages, scale=0.05, out=outs[k], lse=lses[k], ws=w)

    call(0, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(0, ws)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for i in range(4):
        ws.fill_(0xA5)
        torch.cuda.synchronize()
        graph.replay()
        for k, (s, w) in enumerate(zip(streams, (ws, other))):
            if k == 0:
                torch.cuda.synchronize()
                w.fill_(0xFF)
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                call(1 + k, w)
        torch.cuda.synchronize()
        for k in (1, 2):
            assert torch.equal(outs[0], outs[k]) and torch.equal(lses[0], lses[k]), (i, k)
        _check(q, cache, ln.tolist(), parents.tolist(), dc, pages, None, 0.05, (outs[0], lses[0]), t, heads=[i, H - 1])
        q.copy_(q.flip(1))
        ln.copy_(_i32([[40, 1400, 24], [700, 701, 24 + i], [1500, 333, 64]][i % 3]).clamp(max=pages.shape[1] * 48))
        ln.clamp_(max=_i32(lens))
        parents.copy_(_i32(_grown(7 + i, B, Q)))


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("lens", [(40, 64), (300, 61), (64, 7000)])
@pytest.mark.parametrize("Q,H,rows", [(55, 7, (55, 37)), (64, 2, (64, 1)), (43, 3, (43, 1)), (3, 43, (3, 3)), (2, 65, (2, 1)), (1, 131, (1, 1)),
                                      (64, 3, (43, 64))])
def test_many_rows_that_leave_one_to_three_in_a_block(Q, H, rows, lens, t):
    """A block's last rows are fewer than the wavefronts that store them; whole blocks (one tile) and cut ones."""
    B = 2
    q, cache, ln, pages = chain._case(B, Q, H, 512, 64, list(lens), t, 7 * Q + H, 16)
    pages = _roomy(pages, 16, B, Q * H)
    parents = _grown(B + Q, B, Q)
    out, lse = torch.full((B, Q, H, 528), 7.0, dtype=TYPES[t], device=DEV), torch.full((B, Q, H), 7.0, device=DEV)
    _lib.sd_profile_enable(True)
    got = _lib.sd_latent_attention_tree(q, cache, ln, _i32(parents), 512, pages=pages, scale=0.06, out=out[..., 8:520], lse=lse,
                                        rows=_i32(list(rows)))
    torch.cuda.synchronize()
    _lib.sd_profile_enable(False)
    assert "latent_wide" in _lib.sd_profile_read()
    _check(q, cache, list(lens), parents, 512, pages, list(rows), 0.06, got, t, heads=None if H < 8 else [0, H // 2, H - 1])
    assert (out[..., :8] == 7).all() and (out[..., 520:] == 7).all()
    for b in range(B):
        assert (out[b, rows[b]:] == 7).all() and (lse[b, rows[b]:] == 7).all()
