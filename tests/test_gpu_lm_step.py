"""The language-model calls one after another, as a serving step makes them.

Prompts go through the expanded form and drafted rows through the absorbed form of one
attention: the heads' keys and values are columns of the cached vectors (so nothing is
rounded between the forms), k_h = c[a_h], v_h = c[b_h], and a head's absorbed query is its
query put at a_h.  The outputs make logits, the logits are verified, and the accepted
lengths go into the next step.  Every stage is held against its oracle on the inputs that
the stage before really made.
"""
import numpy as np
import pytest
import torch

import test_gpu_latent as absorbed
import test_gpu_latent_expanded as expanded
import test_gpu_tokens as tok
from paper_2606_13426_amd import _lib

pytestmark = pytest.mark.gpu
DEV = "cuda"
H, DC, DR, DN, DV, PAGE = 4, 128, 32, 64, 64, 16
SCALE = (DN + DR) ** -0.5


class _Model:
    def __init__(self, B, K, V, t, seed, longest):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        r = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
        self.B, self.K, self.V, self.t = B, K, V, t
        dt = absorbed.TYPES[t]
        per = -(-longest // PAGE)
        self.cache = r(B * per + 1, PAGE, DC + DR).to(dt)
        self.pages = torch.randperm(B * per + 1, generator=g, device=DEV)[:B * per].view(B, per).to(torch.int32)
        self.a = torch.stack([torch.randperm(DC, generator=g, device=DEV)[:DN] for _ in range(H)])
        self.b = torch.stack([torch.randperm(DC, generator=g, device=DEV)[:DV] for _ in range(H)])
        self.head = r(H * DV, V) * (H * DV) ** -0.5 * 6
        self.near = r(H * DV, V) * (H * DV) ** -0.5 * 2  # what the draft's head lacks
        self.dt = dt

    def absorb(self, q):
        """[..][H][DN + DR] to [..][H][DC + DR]."""
        out = torch.zeros(*q.shape[:-1], DC + DR, dtype=self.dt, device=DEV)
        idx = self.a.expand(*q.shape[:-1], DN)
        out.scatter_(-1, idx, q[..., :DN])
        out[..., DC:] = q[..., DN:]
        return out

    def values(self, lat):
        """The heads' own columns of [..][H][DC]."""
        return lat.gather(-1, self.b.expand(*lat.shape[:-1], DV))

    def logits(self, o):
        x = o.float().flatten(-2)
        full = torch.matmul(x, self.head)
        return full.to(self.dt), torch.matmul(x, self.head + self.near).to(self.dt)


@pytest.mark.parametrize("t", ["bf16", "f16"])
def test_prompts_through_both_forms(t):
    lens = [37, 1, 90, 0]
    m = _Model(4, 3, 11, t, 5, 96)
    nq = [n for n in lens]
    g = torch.Generator(device=DEV)
    g.manual_seed(6)
    Q = max(lens)
    q = torch.randn(4, Q, H, DN + DR, generator=g, device=DEV).to(m.dt)
    ln = torch.tensor(lens, dtype=torch.int32, device=DEV)
    qa = m.absorb(q)
    got = _lib.sd_latent_attention(qa, m.cache, ln, DC, pages=m.pages, rows=ln, scale=SCALE)
    absorbed._check(qa, m.cache, ln, DC, m.pages, ln, SCALE, got, t)
    c = torch.cat([m.cache[m.pages[b].long()].flatten(0, 1)[:n] for b, n in enumerate(lens)])
    k, v = c[:, m.a], c[:, m.b]
    qp = torch.cat([q[b, :n] for b, n in enumerate(lens)])
    cu = expanded._offsets(nq)
    out, lse = _lib.sd_latent_attention_expanded(qp, k, c[:, DC:], v, cu, cu)
    expanded._check(qp, k, c[:, DC:], v, cu, cu, SCALE, (out, lse), t)
    # One and the same number in exact arithmetic: each is off by 2 (e + small) sum p |v| + e |out| at
    # most, where sum p |v| <= max |v|; 1.1 stands for the float32 parts, which are below e / 20.
    e = absorbed._half_step(t)
    own = m.values(got[0])
    for b, n in enumerate(lens):
        x, y = own[b, :n].double(), out[cu[b]:cu[b + 1]].double()
        assert (x - y).abs().max().item() <= 2 * 1.1 * 3 * e * c.double().abs().max().item() if n else True
        assert (got[1][b, :n] - lse[cu[b]:cu[b + 1]]).abs().max().item() <= 1e-4 if n else True


def _step(m, q, lens, tokens, kb, un, ws):
    lat, _ = _lib.sd_latent_attention(m.absorb(q), m.cache, lens, DC, pages=m.pages, scale=SCALE, ws=ws[0])
    target, guess = m.logits(m.values(lat))
    draft = guess[:, :m.K].contiguous()
    r = _lib.sd_verify_tokens(draft, target, tokens, kb, uniforms=un, ws=ws[1])
    lt = _lib.sd_token_logprobs(target[:, :m.K].reshape(-1, m.V), tokens.view(-1), n_top=3, ws=ws[2])
    ld = _lib.sd_token_logprobs(draft.view(-1, m.V), tokens.view(-1), ws=ws[2])
    # the rows that were accepted, and the token drawn behind them, stay in the sequence
    after = lens - (m.K + 1) + r["tau"]
    return dict(draft=draft, target=target, after=after, lt=lt["logprob"], ld=ld["logprob"], ids=lt["top_ids"], **r)


@pytest.mark.parametrize("t", ["bf16", "f16"])
def test_a_serving_step_and_its_graph(t):
    B, K, V = 5, 3, 1003
    m = _Model(B, K, V, t, 7, 256)
    g = torch.Generator(device=DEV)
    g.manual_seed(8)
    q = torch.randn(B, K + 1, H, DN + DR, generator=g, device=DEV).to(m.dt)
    lens = torch.tensor([250, 4, 64, 131, 17], dtype=torch.int32, device=DEV)
    kb = torch.tensor([3, 3, 2, 3, 0], dtype=torch.int32, device=DEV)
    tokens = torch.randint(0, V, (B, K), generator=g, device=DEV, dtype=torch.int32)
    un = torch.rand(B, K + 1, generator=g, device=DEV, dtype=torch.float64)
    need = (_lib.sd_latent_attention_workspace(B, K + 1, H, DC, DR), _lib.sd_verify_tokens_workspace(B, K, V),
            _lib.sd_token_logprobs_workspace(B * K, V, 3))
    ws = [torch.empty(n, dtype=torch.uint8, device=DEV) for n in need]
    # drafts that the draft's law likes, so that some are accepted
    tokens.copy_(_step(m, q, lens, tokens, kb, un, ws)["draft"].float().argmax(-1))
    held, graph = None, torch.cuda.CUDAGraph()
    for _ in range(2):
        _step(m, q, lens, tokens, kb, un, ws)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        held = _step(m, q, lens, tokens, kb, un, ws)
    accepted = 0
    for i in range(4):
        want = {k: v.clone() for k, v in _step(m, q, lens, tokens, kb, un, ws).items()}
        for w in ws:
            w.fill_(0xA5)
        graph.replay()
        torch.cuda.synchronize()
        for k in want:
            assert torch.equal(want[k].view(torch.uint8), held[k].view(torch.uint8)), (i, k)
        # (tokens that the largest logit chose are no draws of the draft's law; verification takes any)
        said = {k: want[k] for k in ("tau", "token", "log_alpha_res", "log_ratio", "coins")}
        tok._check_verify(want["draft"], want["target"], tokens, kb, un, _lib.SD_BLOCK, 1.0, said)
        accepted += int((want["tau"] > 1).sum())
        # log q_j(x_j) - log p_j(x_j) from the rows' own log-probabilities: each of the three is off by (10 + 2 E|d|)
        # u and half a step of itself (the bounds of test_gpu_tokens.py)
        lt, ld, ell = (x.double().cpu().numpy() for x in (want["lt"].view(B, K), want["ld"].view(B, K), want["log_ratio"]))
        z, y = want["target"].double().cpu().numpy(), want["draft"].double().cpu().numpy()
        for b in range(B):
            for j in range(int(kb[b])):
                es, ed = tok._spread(z[b, j])[0], tok._spread(y[b, j])[0]
                tol = (40 + 4 * es + 4 * ed + abs(lt[b, j]) + abs(ld[b, j]) + abs(ell[b, j])) * tok.U
                assert abs(ell[b, j] - (lt[b, j] - ld[b, j])) <= tol, (i, b, j)
        top = want["ids"].view(B, K, 3)[:, :, 0].cpu().numpy()
        for b in range(B):
            for j in range(K):
                assert z[b, j, top[b, j]] == z[b, j].max()
        # the next step: other lengths, rows and uniforms through the same graph
        lens.copy_(torch.minimum(want["after"].clamp(min=0) + K + 1, torch.tensor(256, device=DEV)))
        q.copy_(torch.randn(B, K + 1, H, DN + DR, generator=g, device=DEV))
        un.copy_(torch.rand(B, K + 1, generator=g, device=DEV, dtype=torch.float64))
        tokens.copy_(_step(m, q, lens, tokens, kb, un, ws)["draft"].float().argmax(-1))
    assert accepted > 0


def test_calls_on_two_streams_at_once():
    m = _Model(3, 2, 5000, "bf16", 9, 512)
    g = torch.Generator(device=DEV)
    g.manual_seed(10)
    args = []
    for i in range(2):
        q = torch.randn(3, 3, H, DN + DR, generator=g, device=DEV).to(m.dt)
        lens = torch.tensor([500 - 100 * i, 3, 130], dtype=torch.int32, device=DEV)
        kb = torch.full((3,), 2, dtype=torch.int32, device=DEV)
        tokens = torch.randint(0, m.V, (3, 2), generator=g, device=DEV, dtype=torch.int32)
        un = torch.rand(3, 3, generator=g, device=DEV, dtype=torch.float64)
        args.append((m, q, lens, tokens, kb, un, [None, None, None]))
    want = [_step(*a) for a in args]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in args]
    got = [[], []]
    for _ in range(3):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(_step(*args[i]))
    torch.cuda.synchronize()
    for i in range(2):
        for r in got[i]:
            for k in r:
                assert torch.equal(r[k].view(torch.uint8), want[i][k].view(torch.uint8)), (i, k)


def test_two_graphs_share_a_workspace():
    lens = [torch.tensor(v, dtype=torch.int32, device=DEV) for v in ([900, 40], [3, 700])]
    m = _Model(2, 2, 2000, "bf16", 11, 1024)
    q = torch.randn(2, 3, H, DN + DR, device=DEV).to(m.dt)
    kb = torch.full((2,), 2, dtype=torch.int32, device=DEV)
    tokens = torch.randint(0, m.V, (2, 2), device=DEV, dtype=torch.int32)
    un = torch.rand(2, 3, device=DEV, dtype=torch.float64)
    need = max(_lib.sd_latent_attention_workspace(2, 3, H, DC, DR), _lib.sd_verify_tokens_workspace(2, 2, m.V),
               _lib.sd_token_logprobs_workspace(4, m.V, 3))
    ws = [torch.empty(need, dtype=torch.uint8, device=DEV)] * 3  # one for all calls of both
    want = [_step(m, q, n, tokens, kb, un, ws) for n in lens]
    graphs, held = [torch.cuda.CUDAGraph() for _ in lens], []
    torch.cuda.synchronize()
    for n, graph in zip(lens, graphs):
        with torch.cuda.graph(graph):
            held.append(_step(m, q, n, tokens, kb, un, ws))
    for i in (0, 1, 0, 0, 1):
        graphs[i].replay()
        torch.cuda.synchronize()
        for k in want[i]:
            assert torch.equal(held[i][k].view(torch.uint8), want[i][k].view(torch.uint8)), (i, k)


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("rows,V", [(3, 9000), (1100, 20001)])
def test_alternatives_of_rows_with_few_tokens_allowed(rows, V, t):
    """Masks that leave one token, fewer than are asked for, more, and none (by -inf and by the lowest value)."""
    x = tok._rows(rows, V, t, 12)
    low = torch.finfo(x.dtype).min
    allowed = {0: 1, 1: 5, 2: 40}
    keep = torch.zeros(rows, V, dtype=torch.bool, device=DEV)
    g = torch.Generator(device=DEV)
    g.manual_seed(13)
    for i, n in allowed.items():
        keep[i, torch.randperm(V, generator=g, device=DEV)[:n]] = True
    masked = torch.where(keep, x, torch.full_like(x, -float("inf")))
    lowest = torch.where(keep, x, torch.full_like(x, low))
    for z in (masked, lowest):
        z[3:] = x[3:]
        if rows > 3:
            z[3] = z[0, 0] * 0 + low
            z[rows - 1] = -float("inf")
        r = _lib.sd_token_logprobs(z, torch.arange(rows, dtype=torch.int32, device=DEV) % V, n_top=20)
        tok._check_logprobs(z, torch.arange(rows, dtype=torch.int32, device=DEV) % V, 20, 1.0, r,
                            range(rows) if rows <= 3 else [0, 1, 2, 3, rows // 2, rows - 1])


def test_given_outputs_are_checked():
    B, K, V = 2, 2, 50
    draft, target = torch.randn(B, K, V, device=DEV), torch.randn(B, K + 1, V, device=DEV)
    tokens, kb = torch.zeros(B, K, dtype=torch.int32, device=DEV), torch.full((B,), K, dtype=torch.int32, device=DEV)
    un = torch.rand(B, K + 1, dtype=torch.float64, device=DEV)
    out = _lib.sd_verify_tokens(draft, target, tokens, kb, uniforms=un)
    again = {k: torch.zeros_like(v) for k, v in out.items()}
    _lib.sd_verify_tokens(draft, target, tokens, kb, uniforms=un, out=again)
    assert all(torch.equal(out[k], again[k]) for k in out)
    for k, bad in (("tau", again["tau"].long()), ("token", again["token"][:1]), ("log_ratio", again["log_ratio"].t()),
                   ("coins", again["coins"].cpu()), ("log_alpha_res", again["log_alpha_res"].double())):
        with pytest.raises(_lib.SpecDiffError):
            _lib.sd_verify_tokens(draft, target, tokens, kb, uniforms=un, out=dict(again, **{k: bad}))
