"""sd_latent_attention_expanded against the float64 oracle on the same 16-bit inputs.

The bounds of test_gpu_latent.py: a score off by (d + 5) u sum |q k| |scale|, a weight
by that and half a step e of the type, sums over n keys by n u, all of sum_j p_j |v_j|
and twice (weights and their sum); e of the output itself.
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


def _offsets(counts, first=0):
    return torch.tensor(np.concatenate([[first], first + np.cumsum(counts)]), dtype=torch.int32, device=DEV)


def _case(nq, nk, H, dn, dr, dv, t, seed, extra=0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    Tq, Tk = sum(nq) + 2 * extra, sum(nk) + 2 * extra
    r = lambda *s: torch.randn(*s, generator=g, device=DEV).to(TYPES[t])  # noqa: E731
    return (r(max(Tq, 1), H, dn + dr), r(max(Tk, 1), H, dn), r(max(Tk, 1), dr) if dr else None, r(max(Tk, 1), H, dv),
            _offsets(nq, extra), _offsets(nk, extra))


def _check(q, k, kr, v, cq, ck, scale, got, t, seqs=None, heads=None, rows=None):
    out, lse = (x.double().cpu().numpy() for x in got)
    qn, kn, vn = (x.double().cpu().numpy() for x in (q, k, v))
    rn = np.zeros((len(kn), 0)) if kr is None else kr.double().cpu().numpy()
    a, b = cq.cpu().numpy(), ck.cpu().numpy()
    e = torch.finfo(TYPES[t]).eps / 2
    d = qn.shape[2]
    for s in range(len(a) - 1) if seqs is None else seqs:
        n, m = a[s + 1] - a[s], b[s + 1] - b[s]
        at = range(n) if rows is None else sorted({r for r in rows if 0 <= r < n} | {n - 1})
        for h in range(qn.shape[1]) if heads is None else heads:
            key = np.concatenate([kn[b[s]:b[s + 1], h], rn[b[s]:b[s + 1]]], 1)
            val = vn[b[s]:b[s + 1], h]
            idx = np.array(list(at), dtype=int)
            lim = np.clip(m - n + idx + 1, 0, m)
            w, wl, mag = olat.attend(qn[a[s] + idx, h], key, val, scale, lim)
            for j, i in enumerate(idx):
                o, l = out[a[s] + i, h], lse[a[s] + i, h]
                if lim[j] == 0:
                    assert (o == 0).all() and l == -np.inf, (s, h, i)
                    continue
                sc = abs(scale) * (np.abs(key[:lim[j]]) @ np.abs(qn[a[s] + i, h])).max()
                ds = (d + 5) * U * sc
                assert abs(l - wl[j]) <= ds + (lim[j] + 4) * U + U * abs(wl[j]), (s, h, i, l, wl[j])
                tol = 2 * (ds + e + (lim[j] + 4) * U) * mag[j] + e * np.abs(w[j])
                tol = tol + (2.0 ** -24 if t == "f16" else 0.0)
                err = np.abs(o - w[j])
                assert (err <= tol).all(), (s, h, i, float((err / tol).max()))


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("nq,nk,H,dn,dr,dv", [
    ([1], [1], 1, 8, 0, 8), ([1, 1, 3], [1, 64, 65], 2, 128, 64, 128), ([129, 0, 5], [129, 7, 5], 3, 128, 64, 128),
    ([64, 128, 33], [64, 128, 200], 2, 64, 32, 64), ([300], [300], 1, 96, 32, 80), ([5, 2], [3, 0], 2, 128, 64, 128),
    ([257], [700], 2, 128, 64, 128), ([31] * 9, [40] * 9, 5, 40, 8, 24), ([200], [130], 1, 128, 16, 64),
    ([1] * 70, [17] * 70, 2, 64, 64, 64), ([127, 1, 128, 129], [127, 1, 128, 129], 8, 128, 64, 128)])
def test_expanded(nq, nk, H, dn, dr, dv, t):
    q, k, kr, v, cq, ck = _case(nq, nk, H, dn, dr, dv, t, sum(nq) + H)
    got = _lib.sd_latent_attention_expanded(q, k, kr, v, cq, ck)
    _check(q, k, kr, v, cq, ck, (dn + dr) ** -0.5, got, t, seqs=None if len(nq) < 20 else [0, 33, 69])


@pytest.mark.parametrize("scale", [1.2, -0.1, 0.0])
def test_scales(scale):
    # 1.2: scores of hundreds, so the reference moves again and again
    q, k, kr, v, cq, ck = _case([150], [260], 2, 128, 64, 128, "bf16", 4)
    got = _lib.sd_latent_attention_expanded(q, k, kr, v, cq, ck, scale=scale)
    _check(q, k, kr, v, cq, ck, scale, got, "bf16")


def test_scores_that_rise_with_the_keys():
    # every tile moves the reference: keys along one direction, longer and longer
    q, k, kr, v, cq, ck = _case([100], [640], 1, 64, 0, 64, "bf16", 4)
    k.copy_((torch.ones_like(k, dtype=torch.float32) * torch.arange(640, device=DEV)[:, None, None] / 64).to(k.dtype))
    q.copy_((q.float().abs() * 0.5).to(q.dtype))
    got = _lib.sd_latent_attention_expanded(q, k, kr, v, cq, ck, scale=0.5)
    _check(q, k, kr, v, cq, ck, 0.5, got, "bf16")


@pytest.mark.parametrize("n,nq,nk,H", [(1, 64, 4500, 2), (1, 1000, 3001, 1), (2, 3, 9000, 4), (1, 1, 20000, 16)])
def test_split_keys_are_joined(n, nq, nk, H):
    assert _lib.sd_latent_attention_expanded_workspace(n, H, 128, 64, 128, n * nq, n * nk) > 0
    q, k, kr, v, cq, ck = _case([nq] * n, [nk] * n, H, 128, 64, 128, "bf16", 6)
    got = _lib.sd_latent_attention_expanded(q, k, kr, v, cq, ck)
    _check(q, k, kr, v, cq, ck, 192 ** -0.5, got, "bf16", heads=[0, H - 1], rows=[0, 1, 63, 500])


def test_long_prompts():
    q, k, kr, v, cq, ck = _case([2100, 1500], [2100, 1500], 4, 128, 64, 128, "f16", 6)
    got = _lib.sd_latent_attention_expanded(q, k, kr, v, cq, ck)
    _check(q, k, kr, v, cq, ck, 192 ** -0.5, got, "f16", heads=[0, 3], rows=[0, 63, 64, 127, 128, 1000, 1499])


def test_views_and_rows_of_no_sequence():
    # keys and values as halves of one buffer, queries and outputs as every other head; offsets that start
    # behind the first rows and end before the last
    H, dn, dr, dv, x = 3, 128, 64, 128, 5
    q, k, kr, v, cq, ck = _case([70, 40], [90, 40], H, dn, dr, dv, "bf16", 8, extra=x)
    kv = torch.cat([k, v], 2)
    qq = torch.stack([q, q * 0 + 9], 2).reshape(q.shape[0], 2 * H, -1)
    out = torch.full((q.shape[0], 2 * H, dv), 5.0, dtype=q.dtype, device=DEV)
    lse = torch.full((q.shape[0], H), 5.0, device=DEV)
    q[:x], q[-x:] = float("nan"), float("nan")
    kr[:x], kr[-x:] = float("nan"), float("nan")
    kv[:x], kv[-x:] = float("nan"), float("nan")
    got = _lib.sd_latent_attention_expanded(qq[:, ::2], kv[..., :dn], kr, kv[..., dn:], cq, ck, out=out[:, ::2], lse=lse)
    _check(q, k, kr, v, cq, ck, 192 ** -0.5, got, "bf16")
    assert (out[:, 1::2] == 5).all() and (out[:x] == 5).all() and (out[-x:] == 5).all() and (lse[-x:] == 5).all()


@pytest.mark.parametrize("split", [False, True])
@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
def test_what_a_row_does_not_see_has_no_part_in_it(bad, split):
    nq, nk, H = (200, 230, 40) if not split else (150, 1100, 2)
    q, k, kr, v, cq, ck = _case([nq], [nk], H, 128, 64, 128, "bf16", 9)
    assert (_lib.sd_latent_attention_expanded_workspace(1, H, 128, 64, 128, nq, nk) > 0) == split
    want = _lib.sd_latent_attention_expanded(q, k, kr, v, cq, ck)
    for j in (nk - 1, nk - 70, nk - nq + 64):
        d = [x.clone() for x in (k, kr, v)]
        d[2][j, :, 3] = bad
        first = j - (nk - nq)  # the first row that sees key j
        out, lse = _lib.sd_latent_attention_expanded(q, d[0], d[1], d[2], cq, ck)
        assert torch.isfinite(out[:first].float()).all()
        assert ((out - want[0]).abs()[:first].float() <= 2.0 ** -6 * want[0].abs().float().amax()).all()
        keep = torch.arange(128, device=DEV) != 3
        assert torch.isfinite(out[first:][..., keep].float()).all()
        hit = out[first:, :, 3].float()
        assert (torch.isnan(hit) if bad != bad else hit == bad).all()
        assert torch.allclose(lse, want[1], rtol=1e-5)
        d[0][j], d[1][j], d[2][j] = bad, bad, bad  # the whole token: rows that see it are NaN
        out, lse = _lib.sd_latent_attention_expanded(q, d[0], d[1], d[2], cq, ck)
        assert torch.isfinite(out[:first].float()).all() and torch.equal(lse[:first], want[1][:first])
        assert torch.isnan(out[first:].float()).any(-1).all()


def test_offsets_out_of_order_or_range_stay_inside():
    # not a meaningful call: it must only stay inside its tensors (outputs behind Tq untouched by construction)
    q, k, kr, v, _, _ = _case([100], [100], 2, 64, 64, 64, "bf16", 3)
    for a, b in (([0, 90, 40, 100], [0, 50, 70, 100]), ([-5, 300, 50, 2 ** 31 - 1], [0, -7, 2 ** 30, 100])):
        cq = torch.tensor(a, dtype=torch.int64, device=DEV).to(torch.int32)
        ck = torch.tensor(b, dtype=torch.int64, device=DEV).to(torch.int32)
        _lib.sd_latent_attention_expanded(q, k, kr, v, cq, ck)
    torch.cuda.synchronize()


def test_calls_repeat_to_the_bit_and_replay_in_a_graph():
    q, k, kr, v, cq, ck = _case([300, 20], [900, 1500], 3, 128, 64, 128, "bf16", 2)
    need = _lib.sd_latent_attention_expanded_workspace(2, 3, 128, 64, 128, 320, 2400)
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    want = [x.clone() for x in _lib.sd_latent_attention_expanded(q, k, kr, v, cq, ck, ws=ws)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = _lib.sd_latent_attention_expanded(q, k, kr, v, cq, ck)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(want, other))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = _lib.sd_latent_attention_expanded(q, k, kr, v, cq, ck, ws=ws)
    for i in range(3):
        ws.fill_(0xFF)
        for x in held:
            x.fill_(-3)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(want, held)), i


@pytest.mark.parametrize("t", list(TYPES))
def test_both_forms_agree(t):
    """One sequence's drafted rows through the cache (keys and values from the latent vectors by the
    up-projections folded into q and out) and through expanded keys and values."""
    H, dc, dr, dn, dv, L, Q = 4, 128, 64, 64, 64, 300, 5
    g = torch.Generator(device=DEV)
    g.manual_seed(5)
    r = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    c, kr = r(L, dc).to(TYPES[t]), r(L, dr).to(TYPES[t])
    wk, wv = r(H, dc, dn) / dc ** 0.5, r(H, dc, dv) / dc ** 0.5
    qn, qr = r(Q, H, dn), r(Q, H, dr).to(TYPES[t])
    k = torch.matmul(c.float()[None], wk).transpose(0, 1).contiguous().to(TYPES[t])
    v = torch.matmul(c.float()[None], wv).transpose(0, 1).contiguous().to(TYPES[t])
    cu = [torch.tensor([0, n], dtype=torch.int32, device=DEV) for n in (Q, L)]
    scale = (dn + dr) ** -0.5
    q = torch.cat([qn.to(TYPES[t]), qr], 2)
    a, la = _lib.sd_latent_attention_expanded(q, k, kr, v, cu[0], cu[1], scale=scale)
    qa = torch.matmul(qn.transpose(0, 1), wk.transpose(1, 2).contiguous()).transpose(0, 1)
    cache = torch.cat([c, kr], 1)[None].contiguous()
    lens = torch.tensor([L], dtype=torch.int32, device=DEV)
    o, lb = _lib.sd_latent_attention(torch.cat([qa.to(TYPES[t]), qr], 2)[None], cache, lens, dc, scale=scale)
    b = torch.matmul(o[0].float().transpose(0, 1), wv).transpose(0, 1)
    # k, v, the folded q and the latent output are each rounded once: a score of |q||k| terms is off by
    # about e sqrt(d) of its terms' size (4 e in units of 1 here, times 3 for the largest of 1500), the
    # output by that and 4 e of values of size 1
    e = torch.finfo(TYPES[t]).eps / 2
    assert ((la - lb[0]).abs() <= 24 * e).all()
    assert ((a.float() - b).abs() <= 24 * e).all()
