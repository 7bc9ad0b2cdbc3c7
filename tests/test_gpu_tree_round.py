"""A round of tree drafts as a serving step makes it: append, tree attention, verification, keep, and the next
round on what is left in the cache; eagerly, captured, on two streams, and with a shared workspace."""
import numpy as np
import pytest
import torch

import test_gpu_append as app
import test_gpu_tree_attention as att
import test_gpu_verify_tree as ver
from oracle import tree
from paper_2606_13426_amd import _lib

pytestmark = pytest.mark.gpu
DEV = "cuda"
H, DC, DR, PAGE, LAYERS = 4, 128, 32, 16, 2
SCALE = (64 + DR) ** -0.5


class _Serving:
    """What a serving program keeps: caches, a page table, lengths, and products that stand for a model."""

    def __init__(self, B, Q, V, t, seed, longest=256):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(seed)
        dt = app.TYPES[t]
        r = lambda *s: torch.randn(*s, generator=self.g, device=DEV)  # noqa: E731
        self.B, self.Q, self.V, self.t, self.dt, self.r = B, Q, V, t, dt, r
        per = -(-longest // PAGE)
        self.cache = r(LAYERS, B * per + 1, PAGE, DC + DR).to(dt)
        self.pages = torch.randperm(B * per + 1, generator=self.g, device=DEV)[: B * per].view(B, per).to(torch.int32)
        self.head, self.near = r(LAYERS * H * DC, V) * (LAYERS * H * DC) ** -0.5 * 8, r(LAYERS * H * DC, V) * (LAYERS * H * DC) ** -0.5
        self.freq = 10000.0 ** (-torch.arange(DR // 2, device=DEV, dtype=torch.float64) * 2 / DR)
        self.ws = [torch.empty(n, dtype=torch.uint8, device=DEV) for n in (
            _lib.sd_latent_attention_tree_workspace(B, Q, H, DC, DR), _lib.sd_verify_tree_workspace(B, Q, V))]
        self.new = r(LAYERS, B, Q, DC + DR).to(dt)
        self.q = r(LAYERS, B, Q, H, DC + DR).to(dt)
        self.lens = torch.tensor([100 - 17 * b for b in range(B)], dtype=torch.int32, device=DEV)
        self.trees = att._grown(seed, B, Q)
        self.parents = torch.tensor(self.trees, dtype=torch.int32, device=DEV)
        self.rows = torch.tensor([max(1, Q - b) for b in range(B)], dtype=torch.int32, device=DEV)
        self.tokens = torch.randint(0, V, (B, Q), generator=self.g, device=DEV, dtype=torch.int32)
        self.un = torch.rand(B, Q, generator=self.g, device=DEV, dtype=torch.float64)

    def step(self):
        lens = self.lens + self.rows
        outs, turned = [], []
        for y in range(LAYERS):
            q = self.q[y].clone()
            _lib.sd_latent_append(self.new[y, ..., :DC], self.new[y, ..., DC:], self.cache[y], lens, self.freq, pages=self.pages,
                                  rows=self.rows, parents=self.parents, q=q[..., DC:], q_out=q[..., DC:])
            turned.append(q)
            out = torch.zeros(self.B, self.Q, H, DC, dtype=self.dt, device=DEV)
            lse = torch.zeros(self.B, self.Q, H, device=DEV)
            outs.append(_lib.sd_latent_attention_tree(q, self.cache[y], lens, self.parents, DC, pages=self.pages, rows=self.rows,
                                                      scale=SCALE, out=out, lse=lse, ws=self.ws[0]))
        x = torch.cat([o.flatten(2) for o, _ in outs], -1).float()
        target, draft = torch.matmul(x, self.head).to(self.dt), torch.matmul(x, self.head + self.near).to(self.dt)
        r = _lib.sd_verify_tree(draft, target, self.tokens, self.parents, rows=self.rows, max_children=6, uniforms=self.un, ws=self.ws[1])
        before = self.cache.clone()
        after = _lib.sd_latent_keep(self.cache, lens, r["tau"], r["path"], pages=self.pages, rows=self.rows)
        return dict(lens=lens, q=torch.stack(turned), out=torch.stack([o for o, _ in outs]), lse=torch.stack([l for _, l in outs]), target=target, draft=draft, before=before, after=after,
                    cache=self.cache.clone(), **r)

    def likely(self, seed):
        """Drafts that the draft's laws like, from the laws of a first pass."""
        held = self.cache.clone()
        draft = self.step()["draft"].float()
        self.cache.copy_(held)
        top = draft.topk(6, -1).indices
        for b in range(self.B):
            had = [0] * self.Q
            for i in range(1, self.Q):
                p = self.trees[b][i]
                self.tokens[b, i] = top[b, p, had[p] % 6]
                had[p] += 1


def _check_step(m, start, r):
    lens, rows = r["lens"].tolist(), m.rows.tolist()
    for y in range(LAYERS):
        app._check(m.new[y, ..., :DC], m.new[y, ..., DC:], start[y], r["before"][y], lens, m.freq, m.pages, rows, lambda b, i: (b, i),
                   lambda b, i: lens[b] - rows[b] + tree.depth(m.trees[b], i), m.q[y, ..., DC:], r["q"][y, ..., DC:], None, False, m.t)
        att._check(r["q"][y], r["before"][y], lens, m.trees, DC, m.pages, rows, SCALE, (r["out"][y], r["lse"][y]), m.t)
    ver._check(r["draft"], r["target"], m.tokens, m.trees, m.un, r, "iid", rows=rows, wide=6)
    want = r["before"].double().cpu().numpy()
    for y in range(LAYERS):
        new = [tree.keep(want[y], m.pages[b].cpu().numpy(), lens[b] - rows[b], r["path"][b].tolist(), int(r["tau"][b]), rows[b])
               for b in range(m.B)]
    assert np.array_equal(r["cache"].double().cpu().numpy(), want) and r["after"].tolist() == new


@pytest.mark.parametrize("t", ["bf16", "f16"])
def test_rounds_and_their_graph(t):
    m = _Serving(4, 12, 1003, t, 21)
    m.likely(1)
    held = m.cache.clone()
    for _ in range(2):
        m.step()
        m.cache.copy_(held)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = m.step()
    m.cache.copy_(held)
    accepted = 0
    for i in range(4):
        start = m.cache.clone()
        want = m.step()
        _check_step(m, start, want)
        after = m.cache.clone()
        m.cache.copy_(start)
        for w in m.ws:
            w.fill_(0xA5)
        graph.replay()
        torch.cuda.synchronize()
        for k in want:
            assert torch.equal(want[k].view(torch.uint8), kept[k].view(torch.uint8)), (i, k)
        assert torch.equal(m.cache.view(torch.uint8), after.view(torch.uint8))
        accepted += int((want["tau"] > 1).sum())
        # the next round: the kept lengths, new rows, trees' tokens and coins through the same graph
        m.lens.copy_(want["after"].clamp(max=200))
        m.new.copy_(m.r(*m.new.shape))
        m.q.copy_(m.r(*m.q.shape))
        m.un.copy_(torch.rand(m.B, m.Q, generator=m.g, device=DEV, dtype=torch.float64))
        m.likely(i)
    assert accepted > 0


def test_a_kept_branch_is_a_chain_in_the_cache():
    """After keep the cache is what it were if the accepted tokens had come one after another."""
    m = _Serving(3, 10, 700, "bf16", 23)
    m.likely(2)
    start = m.cache.clone()
    r = m.step()
    other, lens = start.clone(), r["after"]
    for b in range(m.B):
        n = int(r["tau"][b])
        at = r["path"][b, :n].long()
        for y in range(LAYERS):
            rows = m.new[y, b, at][None]
            _lib.sd_latent_append(rows[..., :DC], rows[..., DC:], other[y], lens[b:b + 1], m.freq, pages=m.pages[b:b + 1])
    for b in range(m.B):
        flat = [x[:, m.pages[b].long()].flatten(1, 2)[:, : int(lens[b])] for x in (other, m.cache)]
        assert torch.equal(flat[0], flat[1]), b
    assert int((r["tau"] > 1).sum()) > 0
    # and the next token's attention over it is the chain form's
    q = m.r(3, 1, H, DC + DR).to(m.dt)
    parents = torch.full((3, 1), -1, dtype=torch.int32, device=DEV)
    a = _lib.sd_latent_attention_tree(q, m.cache[0], lens, parents, DC, pages=m.pages, scale=SCALE)
    c = _lib.sd_latent_attention(q, other[0], lens, DC, pages=m.pages, scale=SCALE)
    assert torch.equal(a[0], c[0]) and torch.equal(a[1], c[1])


def test_rounds_on_two_streams_at_once():
    ms = [_Serving(3, 9, 5000, "bf16", 25 + i) for i in range(2)]
    starts = [m.cache.clone() for m in ms]
    want = [m.step() for m in ms]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in ms]
    for _ in range(3):
        got = []
        for m, s, start in zip(ms, streams, starts):
            with torch.cuda.stream(s):
                m.cache.copy_(start)
                got.append(m.step())
        torch.cuda.synchronize()
        for w, r in zip(want, got):
            for k in w:
                assert torch.equal(w[k].view(torch.uint8), r[k].view(torch.uint8)), k


def test_two_graphs_share_a_workspace():
    ms = [_Serving(2, 7, 2000, "bf16", 31), _Serving(3, 12, 900, "bf16", 32)]
    most = torch.empty(max(w.numel() for m in ms for w in m.ws), dtype=torch.uint8, device=DEV)
    starts, want, graphs, kept = [m.cache.clone() for m in ms], [], [torch.cuda.CUDAGraph() for _ in ms], []
    for m in ms:
        m.ws = [most, most]  # one for all calls of both
        want.append(m.step())
    torch.cuda.synchronize()
    for m, graph in zip(ms, graphs):
        with torch.cuda.graph(graph):
            kept.append(m.step())
    for i in (0, 1, 0, 0, 1):
        ms[i].cache.copy_(starts[i])
        graphs[i].replay()
        torch.cuda.synchronize()
        for k in want[i]:
            assert torch.equal(kept[i][k].view(torch.uint8), want[i][k].view(torch.uint8)), (i, k)
