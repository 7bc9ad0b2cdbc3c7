"""The operators of a round of tree drafts, as cases to be timed and checked.

A case is one call of one operator:

  append   sd_latent_append: new tokens' latent vectors into the paged cache, the
           rotary parts of their keys and queries turned by the tokens' positions
           on the way (single tokens, trees of drafts, ragged prompts);
  tree     sd_latent_attention_tree: every drafted row of a tree attends to its
           sequence's cached prefix, to itself and to its ancestors;
  verify   sd_verify_tree: which branch of a tree of drafted tokens the target
           accepts, and the draw of the token that follows it;
  keep     sd_latent_keep: the accepted branch's cached vectors move up behind the
           prefix, in every layer's cache.

`run` computes the plain form with elementary torch operations, or with `own` set
the library's kernels.
"""
import math
import random

import torch

own = False
DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
LARGEST_TREE = 64


def listed():
    return [
        # one user, one token, one layer of a small model: latency
        dict(name="append_1x1", kind="append", B=1, Q=1, H=16, dc=512, dr=64, page=64, longest=777, prompts=False,
             tree=False, halves=False, dtype="bf16"),
        # a serving batch's trees of 24 drafts, all heads on one card, odd pages
        dict(name="append_64x24_tree", kind="append", B=64, Q=24, H=128, dc=512, dr=64, page=48, longest=600,
             prompts=False, tree=True, halves=False, dtype="bf16"),
        # ragged prompts of some thousand tokens, rotated in halves
        dict(name="append_prompts_5x4500", kind="append", B=5, Q=4500, H=32, dc=512, dr=64, page=64, longest=4500,
             prompts=True, tree=False, halves=True, dtype="f16"),
        # one user's tree of 16 nodes over a short context: latency
        dict(name="tree_1x16_700", kind="tree", B=1, Q=16, H=16, dc=512, dr=64, page=64, longest=700, wide=3,
             ragged=False, dtype="bf16"),
        # a batch's trees of 20 nodes, a quarter of the heads, odd pages
        dict(name="tree_24x20_5003", kind="tree", B=24, Q=20, H=32, dc=512, dr=64, page=48, longest=5003, wide=4,
             ragged=True, dtype="f16"),
        # trees of 32 nodes, all heads: the products count
        dict(name="tree_8x32_6000", kind="tree", B=8, Q=32, H=128, dc=512, dr=64, page=64, longest=6000, wide=4,
             ragged=True, dtype="bf16"),
        # the widest tree over one very long context, few heads
        dict(name="tree_1x64_100000", kind="tree", B=1, Q=64, H=16, dc=512, dr=64, page=128, longest=100000, wide=6,
             ragged=False, dtype="bf16"),
        # one user's tree of 12 nodes, drafts drawn independently: latency
        dict(name="verify_1x12x32000", kind="verify", B=1, Q=12, V=32000, wide=3, draws="iid", ragged=False, dtype="f32"),
        # the likeliest tokens of a drafter as candidates, a vocabulary of odd size (rows at 2-byte addresses)
        dict(name="verify_24x24x50001_given", kind="verify", B=24, Q=24, V=50001, wide=4, draws="given", ragged=True,
             dtype="f16"),
        # a serving batch's trees over a large vocabulary, siblings drawn without replacement
        dict(name="verify_32x32x131072_distinct", kind="verify", B=32, Q=32, V=131072, wide=4, draws="distinct",
             ragged=True, dtype="bf16"),
        # one layer, one user: latency
        dict(name="keep_1x1x16", kind="keep", layers=1, B=1, Q=16, d=576, page=64, longest=777, dtype="bf16"),
        # all layers of a deep model, a serving batch
        dict(name="keep_61x64x24", kind="keep", layers=61, B=64, Q=24, d=576, page=48, longest=190, dtype="bf16"),
    ]


def _spread(rng, lo, hi):
    """A whole number of [lo, hi], uniform in its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["append", "tree", "tree", "verify", "verify", "keep"])
    dtype, page = rng.choice(["bf16", "f16"]), rng.choice([1, 16, 48, 64, 100, 128])
    dc, dr = rng.choice([128, 256, 384, 512, 512, 512]), rng.choice([32, 64, 64])
    if kind == "append":
        prompts, H = rng.random() < 0.4, rng.choice([1, 7, 16, 32, 64, 128])
        Q = _spread(rng, 1, 4500) if prompts else _spread(rng, 1, LARGEST_TREE)
        # at most the tokens and heads of the largest listed case
        most = min(16000, 500_000 // H) // Q
        return dict(kind=kind, B=_spread(rng, 1, max(1, min(128, most))), Q=Q, H=H, dc=dc, dr=dr, page=page,
                    longest=max(Q, _spread(rng, 1, 2000)), prompts=prompts, tree=not prompts and rng.random() < 0.6,
                    halves=rng.random() < 0.5, dtype=dtype)
    if kind == "tree":
        Q, H = _spread(rng, 1, LARGEST_TREE), rng.choice([4, 7, 16, 32, 64, 128])
        longest = _spread(rng, Q, 100000)
        # at most the work of the largest listed cases: 300000 cached tokens, 100 million (row, token) pairs
        most = min(300000 // longest, 100_000_000 // (longest * Q * H))
        longest = min(longest, max(Q, 100_000_000 // (Q * H)))
        return dict(kind=kind, B=_spread(rng, 1, max(1, min(128, most))), Q=Q, H=H, dc=dc, dr=dr, page=page,
                    longest=longest, wide=rng.choice([1, 2, 3, 4, 8]), ragged=rng.random() < 0.7, dtype=dtype)
    if kind == "verify":
        V, Q = _spread(rng, 1000, 200000), _spread(rng, 2, LARGEST_TREE)
        return dict(kind=kind, B=_spread(rng, 1, max(1, min(64, 130_000_000 // (V * Q)))), Q=Q, V=V,
                    wide=rng.choice([1, 2, 3, 4, 6]), draws=rng.choice(["iid", "distinct", "given"]),
                    ragged=rng.random() < 0.6, dtype=rng.choice(["f32", "bf16", "f16"]))
    Q, layers, d = _spread(rng, 2, LARGEST_TREE), _spread(rng, 1, 61), dc + dr
    # at most 400 MB of caches
    most = 200_000_000 // (layers * d * 256)
    return dict(kind=kind, layers=layers, B=_spread(rng, 1, max(1, min(64, most))), Q=Q, d=d, page=page,
                longest=Q + _spread(rng, 1, 128), dtype=dtype)


# ------------------------------------------------------------------ inputs --
def _lengths(case):
    """The sequences' lengths with their new rows: the longest, and where they are ragged others down to an
    eighth of it."""
    B, L, Q = case["B"], case["longest"], case["Q"]
    if not case.get("ragged", True):
        return [L] * B
    return [max(Q, L - (L * 7 * ((b * 37) % 64)) // (8 * 64)) for b in range(B)]


def _rows(case):
    """The new rows of every sequence: trees cut short near the end of an answer, prompts of any length."""
    B, Q = case["B"], case["Q"]
    if case.get("prompts"):
        return [max(1, Q - (Q * 3 * ((b * 29) % 32)) // (4 * 32)) for b in range(B)]
    if not case.get("ragged", True):
        return [Q] * B
    return [max(1, Q - (Q * ((b * 13) % 16)) // 32) for b in range(B)]


def _kept(case):
    """How many rows of every sequence are kept: the root and up to 7 accepted drafts that lie further behind."""
    return [1 + min((b * 5 + 3) % 8, (n - 1) // 2) for b, n in enumerate(_rows(case))]


def _grown(seed, B, Q, wide):
    """Trees of Q nodes, node 0 the root: each next node below an earlier one with fewer than `wide` children,
    more often below an early (likely) one."""
    rng = random.Random(seed)
    trees = []
    for _ in range(B):
        parents, room, has = [-1], [0], [0] * Q
        for i in range(1, Q):
            at = int(len(room) * rng.random() ** 2)
            p = room[at]
            parents.append(p)
            has[p] += 1
            if has[p] == wide:
                del room[at]
            room.append(i)
        trees.append(parents)
    return trees


def _depths(parents):
    d = []
    for p in parents:
        d.append(0 if p < 0 else d[p] + 1)
    return d


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _paged(g, lens, page):
    """A page table for these lengths in a random order, and the number of pages."""
    per = [-(-n // page) for n in lens]
    n_pages, width = sum(per) + 3, max(per)
    order = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    pages = torch.zeros(len(lens), width, dtype=torch.int32, device=DEV)
    have = torch.arange(width, device=DEV)[None, :] < torch.tensor(per, device=DEV)[:, None]
    pages[have] = order[: sum(per)]
    return pages, n_pages


def _logits(g, rows, V):
    """Rows of logits as a trained model gives them: a bulk of unlikely tokens and a few likely ones."""
    x = torch.randn(rows, V, generator=g, device=DEV, dtype=torch.float32).mul_(2.0)
    at = torch.randint(0, V, (rows, 1), generator=g, device=DEV) + torch.arange(24, device=DEV) * (V // 24)
    up = torch.rand(rows, 24, generator=g, device=DEV) * 9.0 + 3.0
    return x.scatter_add_(1, at % V, up)


def _ranks(parents):
    """The place of every node among its siblings (parents [B][Q], -1: none)."""
    same = parents[:, :, None] == parents[:, None, :]
    return torch.tril(same, -1).sum(2)


def _prepare_append(case, seed, g, t):
    B, Q, H, dc, dr = (case[k] for k in ("B", "Q", "H", "dc", "dr"))
    n = _rows(case)
    lens = [max(a, b) for a, b in zip(_lengths(case), n)]
    pages, n_pages = _paged(g, lens, case["page"])
    r = lambda *shape: torch.randn(*shape, generator=g, device=DEV, dtype=torch.float32).to(t)  # noqa: E731
    lead = (sum(n),) if case["prompts"] else (B, Q)
    down = r(*lead, dc + dr)  # one product's output: the latent vector and the rotary part side by side
    s = dict(case=case, latent=down[..., :dc], k_rope=down[..., dc:], q=r(*lead, H, dr), pages=pages,
             cache=r(n_pages, case["page"], dc + dr), lens=_i32(lens), rows=None, cu=None, parents=None, k_out=None,
             freq=10000.0 ** (-torch.arange(dr // 2, device=DEV, dtype=torch.float64) * 2.0 / dr))
    # where the queries of the attention that follows have their rotary part
    s["q_out"] = torch.zeros(*lead, H, (128 if case["prompts"] else dc) + dr, device=DEV, dtype=t)[..., -dr:]
    if case["prompts"]:
        s["cu"] = _i32([sum(n[:b]) for b in range(B + 1)])
        s["k_out"] = torch.zeros(sum(n), dr, device=DEV, dtype=t)
    else:
        s["rows"] = _i32(n)
        if case["tree"]:
            s["parents"] = _i32(_grown(seed, B, Q, 4))
    return s


def _prepare_tree(case, seed, g, t):
    B, Q, H, dc, dr = (case[k] for k in ("B", "Q", "H", "dc", "dr"))
    lens = _lengths(case)
    pages, n_pages = _paged(g, lens, case["page"])
    q = torch.randn(B, Q, H, dc + dr, generator=g, device=DEV).to(t)
    cache = torch.randn(n_pages, case["page"], dc + dr, generator=g, device=DEV, dtype=torch.float32).to(t)
    return dict(case=case, q=q, cache=cache, pages=pages, longest=max(lens), lens=_i32(lens), rows=_i32(_rows(case)),
                parents=_i32(_grown(seed, B, Q, case["wide"])), scale=1.0 / math.sqrt(128 + dr),
                out=torch.zeros(B, Q, H, dc, device=DEV, dtype=t), lse=torch.zeros(B, Q, H, device=DEV))


def _prepare_verify(case, seed, g, t):
    B, Q, V, wide = case["B"], case["Q"], case["V"], case["wide"]
    trees = _grown(seed, B, Q, wide)
    parents = _i32(trees)
    target = _logits(g, B * Q, V).view(B, Q, V)
    # the drafter's logits of the same places, and the candidates that it hands out below each
    draft = (target + 0.6 * torch.randn(B, Q, V, generator=g, device=DEV)).to(t)
    noise = -torch.log(-torch.log(torch.rand(B, Q, V, generator=g, device=DEV).clamp_(1e-7, 1 - 1e-7)))
    up = parents.long().clamp(min=0)
    if case["draws"] == "iid":
        tokens = torch.cat([(draft[b].float()[up[b]] + noise[b]).argmax(-1)[None] for b in range(B)])
    else:
        of = torch.cat([(draft[b].float() + (noise[b] if case["draws"] == "distinct" else 0.0)).topk(wide, -1).indices[None]
                        for b in range(B)])  # [B][Q][wide], in the order of the draws
        tokens = of.gather(1, up[:, :, None].expand(-1, -1, wide)).gather(2, _ranks(parents).clamp(max=wide - 1)[:, :, None])[:, :, 0]
    uniforms = torch.rand(B, Q, generator=g, device=DEV, dtype=torch.float64).clamp_(1e-12, 1 - 1e-12)
    return dict(case=case, target=target.to(t), draft=None if case["draws"] == "given" else draft, parents=parents,
                tokens=tokens.to(torch.int32), rows=_i32(_rows(case)), uniforms=uniforms,
                depth=max(max(_depths(p)) for p in trees))


def _prepare_keep(case, seed, g, t):
    B, Q, layers = case["B"], case["Q"], case["layers"]
    rng, n, tau = random.Random(seed), _rows(case), _kept(case)
    lens = _lengths(case)
    pages, n_pages = _paged(g, lens, case["page"])
    # (the accepted nodes lie behind the places that they move to, so a repeated pass moves the same vectors)
    paths = [[0] + sorted(rng.sample(range(a, m), a - 1)) + [-1] * (Q - a) for a, m in zip(tau, n)]
    cache = torch.empty(layers, n_pages, case["page"], case["d"], device=DEV, dtype=t).normal_(generator=g)
    return dict(case=case, cache=cache, pages=pages, lens=_i32(lens), rows=_i32(n), tau=_i32(tau), path=_i32(paths))


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return dict(append=_prepare_append, tree=_prepare_tree, verify=_prepare_verify,
                keep=_prepare_keep)[case["kind"]](case, seed, g, TYPES[case["dtype"]])


# --------------------------------------------------------------- one pass --
def _ancestors(parents):
    """[B][Q][Q]: whether the second node is the first or one of its ancestors (trees of up to 64 nodes)."""
    Q = parents.shape[1]
    reach = torch.eye(Q, device=DEV) + (parents[:, :, None] == torch.arange(Q, device=DEV)).float()
    for _ in range(6):
        reach = torch.bmm(reach, reach).clamp_(max=1.0)
    return reach > 0


def _places(s, at):
    """The cache rows (over all pages) of the tokens `at` [B][...]."""
    page = s["case"]["page"]
    return s["pages"].long().gather(1, (at // page).flatten(1)).view(at.shape) * page + at % page


def _rotated(x, pos, freq, halves):
    """The pairs of x [tokens][...][d] turned by pos [tokens] times the frequencies."""
    a = (pos.double()[:, None] * freq).view(-1, *[1] * (x.dim() - 2), freq.numel())
    c, v = torch.cos(a).float(), torch.sin(a).float()
    y = x.float()
    if halves:
        y1, y2 = y[..., : freq.numel()], y[..., freq.numel() :]
        return torch.cat([y1 * c - y2 * v, y1 * v + y2 * c], -1).to(x.dtype)
    y1, y2 = y[..., 0::2], y[..., 1::2]
    return torch.stack([y1 * c - y2 * v, y1 * v + y2 * c], -1).flatten(-2).to(x.dtype)


def _plain_append(s):
    c, d = s["case"], s["cache"].shape[2]
    T = s["latent"].shape[:-1].numel()
    if c["prompts"]:
        b = torch.searchsorted(s["cu"], torch.arange(T, device=DEV, dtype=torch.int32), right=True) - 1
        i, n = torch.arange(T, device=DEV) - s["cu"].long()[b], (s["cu"][1:] - s["cu"][:-1]).long()
        real = torch.ones(T, dtype=torch.bool, device=DEV)
    else:
        b = torch.arange(T, device=DEV) // c["Q"]
        i, n = torch.arange(T, device=DEV) % c["Q"], s["rows"].long()
        real = i < n[b]
    first = (s["lens"].long() - n)[b]
    pos = first + (i if s["parents"] is None else _ancestors(s["parents"]).sum(2).flatten() - 1)
    # (rows that are not there store the sequence's first one once more)
    at = first + torch.where(real, i, torch.zeros_like(i))
    row = s["pages"].long()[b, at // c["page"]] * c["page"] + at % c["page"]
    flat, latent = s["cache"].view(-1, d), s["latent"].reshape(T, -1)
    k = _rotated(s["k_rope"].reshape(T, -1), pos, s["freq"], c["halves"])
    of = torch.where(real, torch.arange(T, device=DEV), torch.arange(T, device=DEV) - i)
    flat[row] = torch.cat([latent, k], 1)[of]
    q = _rotated(s["q"].reshape(T, c["H"], -1), pos, s["freq"], c["halves"]).view(s["q"].shape)
    s["q_out"].copy_(torch.where(real.view(*s["q"].shape[:-2], 1, 1), q, s["q_out"]))
    if s["k_out"] is not None:
        s["k_out"].copy_(k)
        return dict(cache=s["cache"], q=s["q_out"], k=s["k_out"])
    return dict(cache=s["cache"], q=s["q_out"])


def _plain_tree(s):
    c = s["case"]
    B, Q, H, dc, L = c["B"], c["Q"], c["H"], c["dc"], s["longest"]
    at = torch.arange(L, device=DEV)
    row = _places(s, at.expand(B, L).clamp(max=s["pages"].shape[1] * c["page"] - 1))
    keys = s["cache"].reshape(-1, s["cache"].shape[2])[row].float()  # [B][L][dc + dr]
    q = s["q"].float().reshape(B, Q * H, -1)
    score = torch.bmm(q, keys.transpose(1, 2).contiguous()) * s["scale"]
    prefix = (s["lens"] - s["rows"]).long()
    node = (at - prefix[:, None]).clamp(-1, Q - 1)  # [B][L]: which row a token is of, -1 in the prefix
    below = _ancestors(s["parents"]).gather(2, node.clamp(min=0)[:, None, :].expand(-1, Q, -1))
    seen = ((node < 0)[:, None, :] | below) & (at < s["lens"][:, None])[:, None, :]
    seen = seen.repeat_interleave(H, 1)
    score = score.masked_fill_(~seen, -math.inf)
    m = score.amax(-1, keepdim=True)
    p = torch.exp(score - m)
    l = p.sum(-1, keepdim=True)
    out = (torch.bmm(p, keys[:, :, :dc].contiguous()) / l).view(B, Q, H, dc).to(s["q"].dtype)
    lse = (m + torch.log(l)).view(B, Q, H)
    real = (torch.arange(Q, device=DEV) < s["rows"][:, None])[:, :, None]
    return dict(out=torch.where(real[..., None], out, s["out"]), lse=torch.where(real, lse, s["lse"]))


def _law(x):
    x = x.double()
    e = torch.exp(x - x.amax(-1, keepdim=True))
    return e / e.sum(-1, keepdim=True)


def _plain_verify(s):
    """In 64 bits: coins are compared with ratios of laws and a cumulative sum with a uniform."""
    c = s["case"]
    B, Q, V, wide = c["B"], c["Q"], c["V"], c["wide"]
    b, tokens, n = torch.arange(B, device=DEV), s["tokens"].long(), s["rows"].long()
    # [B][Q + 1][wide]: the children of every node in their order (the last row takes the nodes that are not there)
    kids = torch.full((B, Q + 1, wide), -1, dtype=torch.long, device=DEV)
    node = torch.arange(Q, device=DEV)
    up = torch.where((node < n[:, None]) & (s["parents"] >= 0), s["parents"].long(), torch.full_like(tokens, Q))
    kids.view(B, -1).scatter_(1, up * wide + _ranks(s["parents"]).clamp(max=wide - 1), node.expand(B, Q))
    cur = torch.zeros(B, dtype=torch.long, device=DEV)
    tau, walking = torch.ones_like(cur), torch.ones(B, dtype=torch.bool, device=DEV)
    path = torch.full((B, Q), -1, dtype=torch.long, device=DEV)
    path[:, 0] = 0
    chance = torch.full((B, Q + 1), -1.0, dtype=torch.float64, device=DEV)
    final = torch.zeros(B, V, dtype=torch.float64, device=DEV)
    for _ in range(s["depth"] + 1):
        r = _law(s["target"][b, cur])
        p = _law(s["draft"][b, cur]) if s["draft"] is not None else None
        taken = torch.full_like(cur, -1)
        for k in range(wide):
            kid = kids[b, cur, k]
            tried = walking & (kid >= 0) & (taken < 0)
            x = tokens[b, kid.clamp(min=0)][:, None]
            of = torch.zeros_like(r).scatter_(1, x, 1.0) if p is None else p  # a given candidate is its whole law
            h = (r.gather(1, x) / of.gather(1, x)).squeeze(1)
            chance.scatter_(1, torch.where(tried, kid, torch.full_like(kid, Q))[:, None], h.clamp(max=1.0)[:, None])
            yes = tried & (s["uniforms"][b, (kid - 1).clamp(min=0)] < h)
            left = (r - of).clamp_(min=0)
            left = left / left.sum(1, keepdim=True)
            r = torch.where((tried & ~yes)[:, None], left, r)
            if c["draws"] == "distinct":
                p = p.scatter(1, x, 0.0)
                p = p / p.sum(1, keepdim=True)
            taken = torch.where(yes, kid, taken)
        final = torch.where((walking & (taken < 0))[:, None], r, final)
        walking = walking & (taken >= 0)
        cur = torch.where(walking, taken, cur)
        at = torch.where(walking, tau, torch.full_like(tau, Q))
        path = torch.cat([path, path[:, :1]], 1).scatter(1, at[:, None], cur[:, None])[:, :Q]
        tau = tau + walking
    cum = final.cumsum(1)
    token = (cum <= s["uniforms"][:, -1:] * cum[:, -1:]).sum(1).clamp(max=V - 1)
    return dict(tau=tau.to(torch.int32), token=token.to(torch.int32), path=path.to(torch.int32),
                accept=chance[:, :Q].float())


def _plain_keep(s):
    layers, j = s["case"]["layers"], torch.arange(s["case"]["Q"], device=DEV)
    first = (s["lens"] - s["rows"]).long()[:, None]
    # (rows that are not kept store the root, which stays where it is, once more)
    kept = j < s["tau"][:, None]
    src = _places(s, first + torch.where(kept, s["path"].long(), torch.zeros_like(s["path"].long())))
    to = _places(s, first + torch.where(kept, j, torch.zeros_like(j)))
    flat = s["cache"].view(layers, -1, s["cache"].shape[3])
    flat[:, to.flatten()] = flat[:, src.flatten()]
    return dict(cache=s["cache"], lens=s["lens"] - s["rows"] + s["tau"])


def _workspace(s, query, *sizes):
    """The call's workspace, allocated at the state's first call and kept with it, as a serving loop keeps it."""
    if "ws" not in s:
        s["ws"] = torch.empty(query(*sizes), dtype=torch.uint8, device=DEV)
    return s["ws"]


def _own(s):
    from paper_2606_13426_amd import _lib
    c = s["case"]
    if c["kind"] == "append":
        q = _lib.sd_latent_append(s["latent"], s["k_rope"], s["cache"], s["lens"], s["freq"], pages=s["pages"],
                                  rows=s["rows"], cu=s["cu"], parents=s["parents"], q=s["q"], q_out=s["q_out"],
                                  k_out=s["k_out"], rope=_lib.SD_ROPE_HALVES if c["halves"] else _lib.SD_ROPE_PAIRS)
        return dict(cache=s["cache"], q=q) | (dict(k=s["k_out"]) if s["k_out"] is not None else {})
    if c["kind"] == "tree":
        ws = _workspace(s, _lib.sd_latent_attention_tree_workspace, c["B"], c["Q"], c["H"], c["dc"], c["dr"])
        out, lse = _lib.sd_latent_attention_tree(s["q"], s["cache"], s["lens"], s["parents"], c["dc"], pages=s["pages"],
                                                 rows=s["rows"], scale=s["scale"], out=s["out"], lse=s["lse"], ws=ws)
        return dict(out=out, lse=lse)
    if c["kind"] == "verify":
        ws = _workspace(s, _lib.sd_verify_tree_workspace, c["B"], c["Q"], c["V"])
        how = dict(iid=_lib.SD_TREE_IID, distinct=_lib.SD_TREE_DISTINCT, given=_lib.SD_TREE_GIVEN)[c["draws"]]
        r = _lib.sd_verify_tree(s["draft"], s["target"], s["tokens"], s["parents"], rows=s["rows"], draws=how,
                                max_children=c["wide"], uniforms=s["uniforms"], ws=ws)
        return {k: r[k] for k in ("tau", "token", "path", "accept")}
    lens = _lib.sd_latent_keep(s["cache"], s["lens"], s["tau"], s["path"], pages=s["pages"], rows=s["rows"])
    return dict(cache=s["cache"], lens=lens)


def run(state):
    if own:
        return _own(state)
    return dict(append=_plain_append, tree=_plain_tree, verify=_plain_verify,
                keep=_plain_keep)[state["case"]["kind"]](state)


# ------------------------------------------------------------------- work --
def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "append":
        T, H, dc, dr = sum(_rows(case)), case["H"], case["dc"], case["dr"]
        outs = 3 if case["prompts"] else 2  # a token's vector is read and written, its rotary part once more for prompts
        return dict(bytes=e * T * (2 * dc + outs * dr + 2 * H * dr) + 12 * case["B"], flops=3 * T * (H + 1) * dr)
    if case["kind"] == "tree":
        B, Q, H, dc, dr = (case[k] for k in ("B", "Q", "H", "dc", "dr"))
        lens, rows = _lengths(case), _rows(case)
        depths = [sum(_depths(p[:n])) + n for p, n in zip(_grown(1, B, Q, case["wide"]), rows)]
        pairs = sum(n * (l - n) + d for n, l, d in zip(rows, lens, depths)) * H
        return dict(bytes=e * (sum(lens) * (dc + dr) + sum(rows) * H * (2 * dc + dr)) + 4 * sum(rows) * (H + 1) +
                    4 * sum(-(-n // case["page"]) for n in lens), flops=2 * pairs * (2 * dc + dr))
    if case["kind"] == "verify":
        # the root is always decided: its rows are what no walk does without
        B, Q, V = case["B"], case["Q"], case["V"]
        laws = 1 if case["draws"] == "given" else 2
        return dict(bytes=B * (laws * V * e + 24 * Q + 8), flops=B * laws * V * 4)
    moved = case["layers"] * sum(a - 1 for a in _kept(case))
    return dict(bytes=2 * e * moved * case["d"] + case["B"] * (4 * case["Q"] + 16), flops=0)


# ------------------------------------------------------------ exact values --
def _exact_append(s, case):
    n = _rows(case)
    lens, pages, parents = s["lens"].tolist(), s["pages"].tolist(), s["parents"].tolist() if s["parents"] is not None else None
    cache, q_out = s["cache"].double(), s["q_out"].double()
    k_out = torch.zeros_like(s["k_rope"], dtype=torch.float64)
    at, first = 0, []
    for b in range(case["B"]):
        d = _depths(parents[b]) if parents is not None else list(range(n[b]))
        new = slice(at, at + n[b]) if case["prompts"] else (b, slice(0, n[b]))
        pos = torch.tensor([lens[b] - n[b] + d[i] for i in range(n[b])], dtype=torch.float64, device=DEV)
        turn = torch.polar(torch.ones(n[b], s["freq"].numel(), dtype=torch.float64, device=DEV), pos[:, None] * s["freq"])

        def rotate(x):
            x = x.double()
            half = x.shape[-1] // 2
            z = torch.complex(x[..., :half].contiguous(), x[..., half:].contiguous()) if case["halves"] else \
                torch.complex(x[..., ::2].contiguous(), x[..., 1::2].contiguous())
            z = z * (turn if x.dim() == 2 else turn[:, None])
            return torch.cat([z.real, z.imag], -1) if case["halves"] else torch.view_as_real(z).flatten(-2)

        k_out[new] = rotate(s["k_rope"][new])
        q_out[new] = rotate(s["q"][new])
        place = [lens[b] - n[b] + i for i in range(n[b])]
        pg = torch.tensor([pages[b][p // case["page"]] for p in place], device=DEV)
        of = torch.tensor([p % case["page"] for p in place], device=DEV)
        cache[pg, of] = torch.cat([s["latent"][new].double(), k_out[new]], -1)
        at += n[b]
    return dict(cache=cache, q=q_out, k=k_out) if case["prompts"] else dict(cache=cache, q=q_out)


def _exact_tree(s, case):
    B, Q, H, dc = (case[k] for k in ("B", "Q", "H", "dc"))
    out, lse = s["out"].double(), s["lse"].double()
    lens, parents = s["lens"].tolist(), s["parents"].tolist()
    for b, n in enumerate(_rows(case)):
        c = s["cache"][s["pages"][b, : -(-lens[b] // case["page"])].long()].flatten(0, 1)[: lens[b]].double()
        see = torch.zeros(n, lens[b], dtype=torch.bool)
        for i in range(n):
            see[i, : lens[b] - n] = True
            j = i
            while j >= 0:
                see[i, lens[b] - n + j] = True
                j = parents[b][j]
        z = (s["q"][b, :n].reshape(n * H, -1).double() @ c.T) * s["scale"]
        z[~see.to(DEV).repeat_interleave(H, 0)] = -math.inf
        l = torch.logsumexp(z, 1)
        out[b, :n] = (torch.exp(z - l[:, None]) @ c[:, :dc]).view(n, H, dc)
        lse[b, :n] = l.view(n, H)
    return dict(out=out, lse=lse)


def _exact_verify(s, case):
    B, Q = case["B"], case["Q"]
    parents, tokens, u = s["parents"].tolist(), s["tokens"].tolist(), s["uniforms"].tolist()
    accept = torch.full((B, Q), -1.0, dtype=torch.float64)
    for b, n in enumerate(_rows(case)):
        node = 0
        while node is not None:
            r = torch.softmax(s["target"][b, node].double(), 0)
            p = torch.softmax(s["draft"][b, node].double(), 0) if s["draft"] is not None else None
            at, node = node, None
            for i in range(at + 1, n):
                if parents[b][i] != at:
                    continue
                x = tokens[b][i]
                ratio = float(r[x]) if p is None else float(r[x] / p[x])
                accept[b, i] = min(1.0, ratio)
                if u[b][i - 1] < ratio:
                    node = i
                    break
                if p is None:
                    r[x] = 0.0
                else:
                    r = (r - p).clamp(min=0)
                r = r / r.sum()
                if case["draws"] == "distinct":
                    p[x] = 0.0
                    p = p / p.sum()
    return dict(tau=None, token=None, path=None, accept=accept)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "append":
        return _exact_append(s, case)
    if case["kind"] == "tree":
        return _exact_tree(s, case)
    if case["kind"] == "verify":
        return _exact_verify(s, case)
    cache = s["cache"].double()
    lens, pages, path = s["lens"].tolist(), s["pages"].tolist(), s["path"].tolist()
    kept, P = [], case["page"]
    for b, (n, a) in enumerate(zip(_rows(case), _kept(case))):
        first = lens[b] - n
        for j in range(a):
            old, new = first + path[b][j], first + j
            cache[:, pages[b][new // P], new % P] = cache[:, pages[b][old // P], old % P]
        kept.append(first + a)
    return dict(cache=cache, lens=torch.tensor(kept, dtype=torch.int32, device=DEV))
