"""Refusals of the tree-draft calls, none of which reaches a HIP call."""
import ctypes

import pytest
import torch

from paper_2606_13426_amd import _lib

P = ctypes.c_void_p(256)  # never dereferenced: validation fails first
ODD = ctypes.c_void_p(264)
S, SH = _lib.sd_stride, _lib.sd_stride_h


@pytest.fixture(scope="module")
def lib():
    import os
    if not os.path.exists(_lib.LIB_PATH):
        from paper_2606_13426_amd import build
        build.build()
    return _lib.load()


def _refused(status, needle):
    assert status == _lib.SD_EINVAL
    assert needle in _lib.last_error(), _lib.last_error()


def _append(lib, **kw):
    a = dict(B=2, Q=3, H=4, dc=128, dr=64, type=1, rope=0, freq=P, latent=P, ls=S(576, 192), k_rope=P, krs=S(576, 192), cu=None,
             parents=None, lens=P, rows=None, cache=P, ps=16 * 192, ts=192, n_pages=9, size=16, pages=P, pstride=4,
             max_pages=4, k_out=None, kos=S(0, 0), q=P, qs=SH(768, 256, 64), q_out=P, qos=SH(768, 256, 64))
    a.update(kw)
    return lib.sd_latent_append(*a.values(), None)


@pytest.mark.parametrize("kw,needle", [
    (dict(B=0), "B >= 1"), (dict(Q=0), "B >= 1"), (dict(H=-1), "H >= 0"), (dict(dc=0), "d_latent = 0"),
    (dict(dc=520), "d_latent = 520"), (dict(dc=132), "d_latent = 132"), (dict(dr=72), "d_rope = 72"), (dict(dr=4), "d_rope = 4"),
    (dict(type=0), "type"), (dict(rope=2), "rope"), (dict(freq=None), "NULL"), (dict(latent=None), "NULL"),
    (dict(k_rope=None), "NULL"), (dict(lens=None), "NULL"), (dict(cache=None), "NULL"), (dict(H=0), "q and q_out"),
    (dict(q=None), "q and q_out"), (dict(q_out=None), "q and q_out"), (dict(dr=0), "d_rope > 0"),
    (dict(dr=0, H=0, q=None, q_out=None, k_out=P), "d_rope > 0"), (dict(cu=P, rows=P), "with cu"),
    (dict(cu=P, parents=P), "with cu"), (dict(parents=P, Q=65, ls=S(1 << 20, 192)), "Q = 65"), (dict(n_pages=0), "n_pages"),
    (dict(size=0), "page_size"), (dict(max_pages=5), "pages_stride"), (dict(max_pages=0), "max_pages"),
    (dict(size=1 << 28, ps=1 << 40), "2^30 tokens"), (dict(pages=None, n_pages=1), "n_pages = 1"), (dict(ts=184), "cache strides"),
    (dict(ts=196), "cache strides"), (dict(ps=100), "cache strides"), (dict(ls=S(576, 120)), "latent strides"),
    (dict(ls=S(570, 192)), "latent strides"), (dict(ls=S(200, 192)), "latent strides"), (dict(krs=S(576, 196)), "k_rope strides"),
    (dict(k_out=P, kos=S(100, 64)), "k_out strides"), (dict(qs=SH(768, 256, 60)), "q strides"),
    (dict(qos=SH(700, 256, 64)), "q_out strides"), (dict(qos=SH(768, 64, 64)), "q_out strides"),
    (dict(latent=ODD), "16-byte"), (dict(k_rope=ODD), "16-byte"), (dict(cache=ODD), "16-byte"), (dict(q=ODD), "16-byte"),
    (dict(q_out=ODD), "16-byte"), (dict(k_out=ODD, kos=S(192, 64)), "16-byte"),
    (dict(B=1 << 20, Q=1 << 12, ls=S(1 << 20, 192), krs=S(1 << 20, 192), qs=SH(1 << 20, 256, 64), qos=SH(1 << 20, 256, 64)),
     "too many rows")])
def test_latent_append_refuses(lib, kw, needle):
    _refused(_append(lib, **kw), needle)


def _tree(lib, **kw):
    a = dict(B=2, Q=2, H=4, dc=128, dr=64, type=1, scale=0.1, q=P, qs=SH(1536, 768, 192), cache=P, ps=16 * 192, ts=192,
             n_pages=9, size=16, pages=P, pstride=4, max_pages=4, lens=P, rows=None, parents=P, out=P,
             os=SH(1024, 512, 128), lse=None, ws=P, ws_bytes=1 << 40)
    a.update(kw)
    return lib.sd_latent_attention_tree(*a.values(), None)


@pytest.mark.parametrize("kw,needle", [
    (dict(Q=65), "Q = 65"), (dict(parents=None), "NULL"), (dict(B=0), "sd_latent_attention_tree: need B"),
    (dict(lens=None), "NULL"), (dict(type=0), "type"), (dict(dc=132), "d_latent = 132"), (dict(ts=184), "cache strides"),
    (dict(qs=SH(1536, 768, 190)), "q strides"), (dict(os=SH(1024, 512, 120)), "out strides"), (dict(q=ODD), "16-byte"),
    (dict(ws_bytes=64), "workspace 64 <"), (dict(ws=ctypes.c_void_p(128)), "256-byte"),
    (dict(size=1 << 28, ps=1 << 40), "2^30 tokens")])
def test_tree_attention_refuses(lib, kw, needle):
    _refused(_tree(lib, **kw), needle)


def _verify(lib, **kw):
    a = dict(B=2, Q=4, V=10, draws=0, type=0, T=1.0, wide=2, draft=P, ds=S(40, 10), target=P, ts=S(40, 10), tokens=P, parents=P,
             rows=None, uniforms=P, round=None, seed=0, tau=P, token=P, path=P, accept=None, ws=P, ws_bytes=1 << 30)
    a.update(kw)
    return lib.sd_verify_tree(*a.values(), None)


@pytest.mark.parametrize("kw,needle", [
    (dict(B=0), "B = 0"), (dict(Q=0), "Q = 0"), (dict(Q=65), "Q = 65"), (dict(V=0), "V = 0"), (dict(V=(1 << 24) + 1), "V = 16777217"),
    (dict(draws=3), "draws"), (dict(type=3), "type"), (dict(T=0.0), "temperature"), (dict(T=float("nan")), "temperature"),
    (dict(wide=0), "max_children = 0"), (dict(wide=5), "max_children = 5"), (dict(draft=None), "draft must be NULL"),
    (dict(draws=2), "draft must be NULL"), (dict(target=None), "NULL"), (dict(tokens=None), "NULL"), (dict(parents=None), "NULL"),
    (dict(tau=None), "NULL"), (dict(token=None), "NULL"), (dict(path=None), "NULL"), (dict(ws=None), "NULL"),
    (dict(uniforms=None), "uniforms and round"), (dict(ds=S(40, 9)), "draft stride"), (dict(ts=S(39, 10)), "target stride"),
    (dict(target=ctypes.c_void_p(258)), "aligned"), (dict(draft=ctypes.c_void_p(257), type=1), "aligned"),
    (dict(ws_bytes=100), "workspace 100 <"), (dict(ws=ctypes.c_void_p(64)), "256-byte"),
    (dict(B=2 ** 31 - 1, V=1 << 20, ds=S(1 << 22, 1 << 20), ts=S(1 << 22, 1 << 20), ws_bytes=2 ** 63 - 1), "too many rows")])
def test_verify_tree_refuses(lib, kw, needle):
    _refused(_verify(lib, **kw), needle)


def _keep(lib, **kw):
    a = dict(layers=3, B=2, Q=4, d=192, type=1, cache=P, ls=9 * 16 * 192, ps=16 * 192, ts=192, n_pages=9, size=16, pages=P,
             pstride=4, max_pages=4, lens=P, rows=None, tau=P, path=P, new_lens=None)
    a.update(kw)
    return lib.sd_latent_keep(*a.values(), None)


@pytest.mark.parametrize("kw,needle", [
    (dict(layers=0), "layers >= 1"), (dict(B=0), "B >= 1"), (dict(Q=0), "Q >= 1"), (dict(d=4), "d = 4"), (dict(d=584), "d = 584"),
    (dict(d=100), "d = 100"), (dict(type=0), "type"), (dict(cache=None), "NULL"), (dict(lens=None), "NULL"), (dict(tau=None), "NULL"),
    (dict(path=None), "NULL"), (dict(n_pages=0), "n_pages"), (dict(ts=100), "cache strides"), (dict(ps=100), "cache strides"),
    (dict(pages=None, n_pages=1), "n_pages = 1"), (dict(max_pages=5), "pages_stride"), (dict(ls=16 * 192), "layer stride"),
    (dict(ls=9 * 16 * 192 + 4), "layer stride"), (dict(ls=0), "layer stride"), (dict(cache=ODD), "16-byte"),
    (dict(new_lens=P), "overlaps"), (dict(new_lens=ctypes.c_void_p(260)), "overlaps"),
    (dict(B=1 << 20, Q=1 << 12), "too many rows"), (dict(layers=1 << 20, B=1 << 20), "too many rows")])
def test_latent_keep_refuses(lib, kw, needle):
    _refused(_keep(lib, **kw), needle)


def test_workspace_queries_of_refused_sizes_are_zero(lib):
    assert lib.sd_verify_tree_workspace(0, 4, 10) == lib.sd_verify_tree_workspace(1, 65, 10) == lib.sd_verify_tree_workspace(1, 4, 0) == 0
    assert lib.sd_latent_attention_tree_workspace(1, 65, 4, 128, 64) == lib.sd_latent_attention_tree_workspace(1, 4, 4, 100, 64) == 0
    assert lib.sd_verify_tree_workspace(1, 1, 1) > 0
    assert lib.sd_latent_attention_tree_workspace(1, 4, 4, 128, 64) == lib.sd_latent_attention_workspace(1, 4, 4, 128, 64) > 0


def test_the_binding_refuses():
    h, i, f = (lambda *s: torch.zeros(*s).half()), (lambda *s: torch.zeros(*s, dtype=torch.int32)), torch.zeros(32).double()
    cache = h(3, 16, 192)
    for call, match in (
            (lambda: _lib.sd_latent_append(h(2, 3, 128), h(2, 3, 64), cache, i(2), f), "not on the current GPU"),
            (lambda: _lib.sd_latent_append(h(2, 3, 128), None, cache, i(2), f), "k_rope must be"),
            (lambda: _lib.sd_latent_append(h(2, 3, 128), h(2, 3, 64), cache, i(2), f, cu=i(3)), "latent must be"),
            (lambda: _lib.sd_latent_append(h(2, 3, 128), h(2, 3, 64), cache, i(2), f, q=h(2, 3, 4, 32)), "q must be"),
            (lambda: _lib.sd_latent_append(h(2, 3, 128), h(2, 3, 64), cache, i(2), f, q_out=h(2, 3, 4, 64)), "q_out goes with q"),
            (lambda: _lib.sd_latent_append(h(2, 3, 128), h(2, 3, 64), cache, i(2), f, k_out=h(2, 3, 32)), "k_out must be"),
            (lambda: _lib.sd_latent_attention_tree(h(2, 3, 4, 192), cache, i(2), None, 128, scale=1.0), "parents"),
            (lambda: _lib.sd_latent_attention_tree(h(2, 3, 4, 192), cache, i(2), i(2, 3), 128, scale=1.0), "not on the current GPU"),
            (lambda: _lib.sd_verify_tree(h(2, 4, 10), h(2, 4, 11), i(2, 4), i(2, 4)), "one type"),
            (lambda: _lib.sd_verify_tree(None, h(2, 4, 10), i(2, 4), i(2, 4)), "not on the current GPU"),
            (lambda: _lib.sd_latent_keep(h(16, 192), i(2), i(2), i(2, 4)), "cache must be"),
            (lambda: _lib.sd_latent_keep(cache, i(2), i(2), i(8)), "path must be"),
            (lambda: _lib.sd_latent_keep(cache, i(2), i(2), i(2, 4)), "not on the current GPU")):
        with pytest.raises(_lib.SpecDiffError, match=match):
            call()


def test_the_binding_refuses_logits_whose_rows_are_not_contiguous():
    x, i = torch.zeros(2, 10, 3), torch.zeros(2, 3, dtype=torch.int32)
    with pytest.raises(_lib.SpecDiffError, match="contiguous rows"):
        _lib.sd_verify_tree(x.transpose(1, 2), x.transpose(1, 2), i, i, uniforms=torch.zeros(2, 3, dtype=torch.float64))
    with pytest.raises(_lib.SpecDiffError, match="contiguous rows"):
        _lib.sd_verify_tree(x.transpose(1, 2), torch.zeros(2, 3, 10), i, i, uniforms=torch.zeros(2, 3, dtype=torch.float64))


@pytest.mark.parametrize("kw", [dict(tau=P), dict(rows=P), dict(path=P), dict(path=ctypes.c_void_p(256 - 4 * 7)), dict(tau=ctypes.c_void_p(252)),
                                dict(rows=ctypes.c_void_p(260))])
def test_latent_keep_refuses_new_lengths_over_what_other_layers_read(lib, kw):
    """B = 2, Q = 4: eight bytes of new lengths at 256, the other arrays elsewhere but for one."""
    far = {k: ctypes.c_void_p(4096 * (i + 1)) for i, k in enumerate(("lens", "rows", "tau", "path"))}
    _refused(_keep(lib, **{**far, **kw, "new_lens": P}), "overlaps")
