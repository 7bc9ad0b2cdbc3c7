"""sd_latent_append and sd_latent_keep against the float64 oracle.

Latent vectors and kept vectors are copied: equal bits.  A rotated element is x cos a - y sin a
(or x sin a + y cos a) with the angle's product in float64 on both sides.  With u = 2^-24, sine and
cosine of the reduced angle are off by 3 u at most (their argument's rounding, two roundings of
the series' largest terms, its end below 2^-29), the two products and their sum by 2 u (|x| + |y|),
together 5 u (|x| + |y|), and the result's rounding by half a step of the type.
"""
import numpy as np
import pytest
import torch

from oracle import tree
from paper_2606_13426_amd import _lib

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _freq(dr):
    return 10000.0 ** (-torch.arange(dr // 2, device=DEV, dtype=torch.float64) * 2.0 / max(dr, 1))


def _table(g, B, per, n_pages):
    return torch.randperm(n_pages, generator=g, device=DEV)[: B * per].view(B, per).to(torch.int32)


def _near(got, x, pos, freq, halves, t, what):
    x, got = x.double().cpu().numpy(), got.double().cpu().numpy()
    f = freq.cpu().numpy()
    want = tree.rotate(x, pos, f, halves)
    half = x.shape[-1] // 2
    size = np.abs(x[..., :half]) + np.abs(x[..., half:]) if halves else np.abs(x[..., ::2]) + np.abs(x[..., 1::2])
    size = np.concatenate([size, size], -1) if halves else np.repeat(size, 2, -1)
    tol = 5 * U * size + torch.finfo(TYPES[t]).eps / 2 * (np.abs(want) + 5 * U * size) + (2.0 ** -25 if t == "f16" else 0.0)
    assert (np.abs(got - want) <= tol).all(), (what, float((np.abs(got - want) / np.maximum(tol, 1e-300)).max()))


def _check(latent, k_rope, before, cache, lens, freq, pages, n_of, row, pos_of, q, q_out, k_out, halves, t):
    """Every row of every sequence; row(b, i) its index, pos_of(b, i) its position."""
    page, n_pages, dc = cache.shape[1], cache.shape[0], latent.shape[-1]
    want = before.clone()
    for b in range(len(lens)):
        for i in range(n_of[b]):
            place, r = max(int(lens[b]), 0) - n_of[b] + i, row(b, i)
            pg = -1
            if pages is None:
                pg = b if 0 <= place < page else -1
            elif 0 <= place < pages.shape[1] * page:
                pg = int(pages[b, place // page])
            if q is not None:
                _near(q_out[r], q[r], pos_of(b, i), freq, halves, t, ("q", b, i))
            if k_out is not None:
                _near(k_out[r], k_rope[r], pos_of(b, i), freq, halves, t, ("k", b, i))
            if 0 <= pg < n_pages:
                at = (pg, place % page if pages is not None else place)
                assert torch.equal(cache[at][:dc], latent[r]), (b, i)
                if cache.shape[2] > dc:
                    _near(cache[at][dc:], k_rope[r], pos_of(b, i), freq, halves, t, ("cache", b, i))
                want[at] = cache[at]
    assert torch.equal(want, cache)  # nothing else was written


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("B,Q,H,dc,dr,page,lens,rows", [
    (1, 1, 1, 8, 8, 1, [1], None), (1, 1, 16, 512, 64, 64, [777], None), (3, 5, 7, 136, 40, 7, [5, 60, 33], [5, 0, 3]),
    (4, 3, 33, 384, 32, 48, [100, 3, 48, 50], [3, 9, 1, -2]), (2, 64, 128, 512, 64, 100, [64, 300], None),
    (2, 4, 0, 504, 56, 16, [40, 31], None), (2, 6, 0, 256, 0, 5, [19, 6], [6, 2]), (70, 2, 3, 64, 16, 4, [9] * 70, None)])
def test_rows_of_chains(B, Q, H, dc, dr, page, lens, rows, halves, t):
    g = _gen(B * 100 + Q)
    dt = TYPES[t]
    per = -(-max(lens) // page)
    before = torch.randn(B * per + 2, page, dc + dr, generator=g, device=DEV).to(dt)
    pages = _table(g, B, per, B * per + 2)
    down = torch.randn(B, Q, dc + dr, generator=g, device=DEV).to(dt)
    q = torch.randn(B, Q, H, dr, generator=g, device=DEV).to(dt) if H else None
    cache, freq = before.clone(), _freq(dr)
    q_out = torch.full((B, Q, H, dc + dr), 7.0, device=DEV, dtype=dt) if H else None
    k_rope = down[..., dc:] if dr else None
    k_out = torch.full((B, Q, dr), 7.0, device=DEV, dtype=dt) if dr and B % 2 else None
    n_of = [Q if rows is None else min(max(r, 0), Q) for r in (rows or [0] * B)]
    got = _lib.sd_latent_append(down[..., :dc], k_rope, cache, _i32(lens), freq if dr else None, pages=pages,
                                rows=None if rows is None else _i32(rows), q=q, q_out=None if q is None else q_out[..., dc:],
                                k_out=k_out, rope=_lib.SD_ROPE_HALVES if halves else _lib.SD_ROPE_PAIRS)
    _check(down[..., :dc], k_rope, before, cache, lens, freq, pages, n_of, lambda b, i: (b, i),
           lambda b, i: lens[b] - n_of[b] + i, q, got, k_out, halves, t)
    for b in range(B):
        if H:
            assert (q_out[b, n_of[b]:] == 7).all() and (q_out[..., :dc] == 7).all()
        if k_out is not None:
            assert (k_out[b, n_of[b]:] == 7).all()


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("lens,counts", [([1], [1]), ([500, 3, 90], [500, 3, 17]), ([40, 0, 7, 0, 0, 130], [33, 0, 7, 0, 0, 1]),
                                         ([5 + b % 9 for b in range(300)], [b % 5 for b in range(300)])])
def test_ragged_prompts(lens, counts, t):
    H, dc, dr, page, B, T = 5, 128, 64, 16, len(lens), sum(counts)
    g = _gen(T)
    dt = TYPES[t]
    per = -(-max(lens) // page)
    before = torch.randn(B * per + 2, page, dc + dr, generator=g, device=DEV).to(dt)
    pages = _table(g, B, per, B * per + 2)
    lead, behind = 3, 2  # rows of no sequence
    latent = torch.randn(T + lead + behind, dc, generator=g, device=DEV).to(dt)
    k_rope = torch.randn(T + lead + behind, dr, generator=g, device=DEV).to(dt)
    q = torch.randn(T + lead + behind, H, dr, generator=g, device=DEV).to(dt)
    starts = [lead + sum(counts[:b]) for b in range(B + 1)]
    cache, freq, q_in, k_in = before.clone(), _freq(dr), q.clone(), k_rope.clone()
    got = _lib.sd_latent_append(latent, k_rope, cache, _i32(lens), freq, pages=pages, cu=_i32(starts), q=q, q_out=q, k_out=k_rope)
    assert got is q  # in place, the keys too
    _check(latent, k_in, before, cache, lens, freq, pages, counts, lambda b, i: (starts[b] + i,),
           lambda b, i: lens[b] - counts[b] + i, q_in, q, k_rope, False, t)
    for x, y in ((q, q_in), (k_rope, k_in)):
        assert torch.equal(x[:lead], y[:lead]) and torch.equal(x[T + lead:], y[T + lead:])


@pytest.mark.parametrize("t", list(TYPES))
def test_trees_are_turned_by_their_depths(t):
    B, Q, H, dc, dr, page = 4, 9, 6, 128, 32, 16
    parents = [[-1, 0, 0, 1, 1, 3, 3, 6, 2], [-1, 0, 1, 2, 3, 4, 5, 6, 7], [3, 9, 1, -5, 3, 4, 0, 2 ** 31 - 1, 7],
               [-1, 0, 0, 0, 0, 0, 0, 0, 0]]
    lens, n_of = [70, 9, 33, 12], [9, 9, 8, 4]
    g = _gen(4)
    before = torch.randn(B * 5, page, dc + dr, generator=g, device=DEV).to(TYPES[t])
    pages = _table(g, B, 5, B * 5)
    latent, k_rope, q = (torch.randn(B, Q, *s, generator=g, device=DEV).to(TYPES[t]) for s in ((dc,), (dr,), (H, dr)))
    cache, freq = before.clone(), _freq(dr)
    q_out = _lib.sd_latent_append(latent, k_rope, cache, _i32(lens), freq, pages=pages, rows=_i32(n_of), parents=_i32(parents), q=q)
    _check(latent, k_rope, before, cache, lens, freq, pages, n_of, lambda b, i: (b, i),
           lambda b, i: lens[b] - n_of[b] + tree.depth(parents[b], i), q, q_out, None, False, t)


def test_places_that_do_not_exist_are_not_stored():
    B, Q, dc, dr, page, t = 5, 4, 64, 16, 8, "bf16"
    g = _gen(5)
    before = torch.randn(12, page, dc + dr, generator=g, device=DEV).to(TYPES[t])
    pages = _table(g, B, 2, 12)
    pages[0, 1], pages[1, 0], pages[2, 1] = -1, 12, 2 ** 31 - 1
    lens = [10, 9, 18, 2, -3]  # over a page's border, past the table, fewer than the rows, none
    latent, k_rope, q = (torch.randn(B, Q, *s, generator=g, device=DEV).to(TYPES[t]) for s in ((dc,), (dr,), (2, dr)))
    cache, freq = before.clone(), _freq(dr)
    q_out = _lib.sd_latent_append(latent, k_rope, cache, _i32(lens), freq, pages=pages, q=q)
    _check(latent, k_rope, before, cache, lens, freq, pages, [Q] * B, lambda b, i: (b, i),
           lambda b, i: max(lens[b], 0) - Q + i, q, q_out, None, False, t)
    # without a table: page b, of page_size tokens
    cache = before.clone()
    _lib.sd_latent_append(latent, k_rope, cache, _i32(lens), freq)
    _check(latent, k_rope, before, cache, lens, freq, None, [Q] * B, lambda b, i: (b, i),
           lambda b, i: max(lens[b], 0) - Q + i, None, None, None, False, t)


def test_far_positions_views_and_odd_values():
    """Positions of 2^29, heads outside rows, places 2^30 elements and more behind the cache's start."""
    B, Q, H, dc, dr, t = 2, 3, 4, 64, 64, "f16"
    g = _gen(6)
    latent, k_rope = (torch.randn(Q, B, d, generator=g, device=DEV).to(TYPES[t]).transpose(0, 1) for d in (dc, dr))
    q = torch.randn(B, H, Q, dr + 8, generator=g, device=DEV).to(TYPES[t])[..., 8:].transpose(1, 2)
    out = torch.full((B, H, Q, dr + 16), 7.0, device=DEV, dtype=TYPES[t])
    # two pages of 2^23 tokens; the table's other pages do not exist
    few = torch.zeros(2, 1 << 23, dc + dr, device=DEV, dtype=TYPES[t])
    pages = torch.full((B, 64), -1, dtype=torch.int32, device=DEV)
    pages[0, 63], pages[1, 40] = 1, 0
    lens = [64 * (1 << 23), 40 * (1 << 23) + 2]
    freq = _freq(dr)
    latent = latent.clone()
    latent[0, 1, 5], latent[1, 2, 0] = float("nan"), float("inf")
    _lib.sd_latent_append(latent, k_rope, few, _i32([n - 1 for n in lens]), freq, pages=pages, q=q,
                          q_out=out[..., 16:].transpose(1, 2))
    for b in range(B):
        for i in range(Q):
            place = lens[b] - 1 - Q + i
            pg = int(pages[b, place >> 23])
            if pg >= 0:
                got = few[pg, place & ((1 << 23) - 1)]
                assert torch.equal(got[:dc].view(torch.int16), latent[b, i].view(torch.int16)), (b, i)
                _near(got[dc:], k_rope[b, i], place, freq, False, t, (b, i))
            _near(out[b, :, i, 16:], q[b, i], place, freq, False, t, ("q", b, i))
    assert (out[..., :16] == 7).all()


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("layers,B,Q,d,page,over", [(1, 1, 1, 8, 1, False), (3, 4, 12, 576, 5, False), (2, 3, 64, 200, 48, True),
                                                    (5, 2, 100, 64, 16, False)])
def test_kept_branches(layers, B, Q, d, page, over, t):
    g = _gen(layers * 10 + B)
    r = np.random.default_rng(Q)
    lens = [Q + 3 + 7 * b for b in range(B)]
    n_of = [max(1, Q - 2 * b) for b in range(B)]
    per = -(-max(lens) // page)
    n_pages = B * per + 1
    # layers over pages, or pages over layers
    shape = (n_pages, layers, page, d) if over else (layers, n_pages, page, d)
    whole = torch.randn(*shape, generator=g, device=DEV).to(TYPES[t])
    cache = whole.transpose(0, 1) if over else whole
    pages = _table(g, B, per, n_pages)
    paths, taus = np.full((B, Q), -1), []
    for b in range(B):
        tau = int(r.integers(0, n_of[b] + 1)) if B > 1 else n_of[b]
        paths[b, :tau] = np.sort(r.choice(n_of[b], tau, replace=False))
        taus.append(tau + (5 if b == 2 else 0))  # (past the rows: clamped, and the path ends in -1)
    want = cache.double().cpu().numpy().copy()
    new = [[tree.keep(want[y], pages[b].cpu().numpy(), lens[b] - n_of[b], paths[b], taus[b], n_of[b]) for b in range(B)]
           for y in range(layers)][0]
    got = _lib.sd_latent_keep(cache if layers > 1 or over else cache[0], _i32(lens), _i32(taus), _i32(paths.tolist()), pages=pages,
                              rows=_i32(n_of))
    assert got.tolist() == new
    assert np.array_equal(cache.double().cpu().numpy(), want)


def test_kept_branches_that_are_none():
    """Paths that fall, repeat, leave the rows; places in no page; no rows; lengths below the rows."""
    B, Q, d, page = 7, 6, 64, 4
    paths = [[0, 3, 3, 4, 5, -1], [2, 1, 0, 0, 0, 0], [0, 2, 9, 3, 4, 5], [-1, 2, 3, 4, 5, 5], [1, 2, 3, 4, 5, -1],
             [0, 4, 5, -1, -1, -1], [1, 3, 5, -1, -1, -1]]
    taus, n_of, lens = [5, 3, 6, 2, 5, 3, 3], [6, 6, 6, 6, 6, 0, 6], [10, 11, 9, 8, 8, 9, 3]
    g = _gen(9)
    cache = torch.randn(2, 24, page, d, generator=g, device=DEV).bfloat16()
    pages = _table(g, B, 3, 24)
    pages[4, 0], pages[4, 1] = -1, 24
    want = cache.double().cpu().numpy().copy()
    new = [[tree.keep(want[y], pages[b].cpu().numpy(), lens[b] - n_of[b], paths[b], taus[b], n_of[b]) for b in range(B)]
           for y in range(2)][0]
    got = _lib.sd_latent_keep(cache, _i32(lens), _i32(taus), _i32(paths), pages=pages, rows=_i32(n_of))
    assert got.tolist() == new and np.array_equal(cache.double().cpu().numpy(), want)
    # a plain cache, page b its sequence's; the lengths are not asked for by a caller of the C call
    plain = torch.randn(B, 12, d, generator=g, device=DEV).bfloat16()
    want = plain.double().cpu().numpy().copy()
    new = [tree.keep(want, [b], lens[b] - Q, paths[b], taus[b], Q) for b in range(B)]
    assert _lib.sd_latent_keep(plain, _i32(lens), _i32(taus), _i32(paths)).tolist() == new
    assert np.array_equal(plain.double().cpu().numpy(), want)
