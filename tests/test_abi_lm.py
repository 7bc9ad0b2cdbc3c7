"""Refusals of the language-model calls, none of which reaches a HIP call."""
import ctypes

import pytest
import torch

from paper_2606_13426_amd import _lib

P = ctypes.c_void_p(256)  # never dereferenced: validation fails first
ODD = ctypes.c_void_p(257)


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


def _logprobs(lib, **kw):
    a = dict(rows=2, V=10, type=0, logits=P, ld=10, T=1.0, n_tok=1, tokens=P, logprob=P, entropy=None, lse=None,
             n_top=2, ids=P, tops=P, ws=P, ws_bytes=1 << 30)
    a.update(kw)
    return lib.sd_token_logprobs(*a.values(), None)


@pytest.mark.parametrize("kw,needle", [
    (dict(rows=0), "rows = 0"), (dict(V=0), "V = 0"), (dict(V=(1 << 24) + 1, ld=1 << 30), "V = 16777217"),
    (dict(type=3), "type"), (dict(n_tok=-1), "n_tok"), (dict(n_top=33), "n_top = 33"), (dict(n_top=-1), "n_top"),
    (dict(T=0.0), "temperature"), (dict(T=float("nan")), "temperature"), (dict(T=float("inf")), "temperature"),
    (dict(T=-1.0), "temperature"), (dict(logits=None), "non-NULL"), (dict(ws=None), "non-NULL"),
    (dict(tokens=None), "tokens"), (dict(logprob=None), "tokens"), (dict(ids=None), "top_ids"),
    (dict(ld=9), "row stride"), (dict(logits=ODD), "aligned"), (dict(logits=ODD, type=1), "aligned"),
    (dict(ws_bytes=8), "workspace 8 <"), (dict(ws=ctypes.c_void_p(128)), "256-byte"),
    (dict(rows=2 ** 31 - 1, V=1 << 20, ld=1 << 20, n_top=0, ids=None, ws_bytes=2 ** 62), "too many rows")])
def test_token_logprobs_refuses(lib, kw, needle):
    _refused(_logprobs(lib, **kw), needle)


def _verify(lib, **kw):
    s = _lib.sd_stride
    a = dict(B=2, K=3, V=10, mode=0, type=0, T=1.0, draft=P, ds=s(30, 10), target=P, ts=s(40, 10), tokens=P, kb=P,
             uniforms=P, round=None, seed=0, tau=P, token=P, lar=P, ratio=P, coins=None, ws=P, ws_bytes=1 << 30)
    a.update(kw)
    return lib.sd_verify_tokens(*a.values(), None)


@pytest.mark.parametrize("kw,needle", [
    (dict(B=0), "B = 0"), (dict(K=0), "K = 0"), (dict(K=65), "K = 65"), (dict(V=0), "V = 0"), (dict(mode=2), "mode"),
    (dict(type=-1), "type"), (dict(T=0.0), "temperature"), (dict(draft=None), "NULL"), (dict(tau=None), "NULL"),
    (dict(uniforms=None), "uniforms and round"), (dict(ds=_lib.sd_stride(30, 9)), "draft stride"),
    (dict(ts=_lib.sd_stride(39, 10)), "target stride"), (dict(draft=ODD), "aligned"),
    (dict(target=ODD, type=2), "aligned"), (dict(ws_bytes=100), "workspace 100 <"),
    (dict(ws=ctypes.c_void_p(64)), "256-byte"),
    (dict(B=2 ** 31 - 1, ws_bytes=2 ** 63 - 1, V=1 << 15, ds=_lib.sd_stride(1 << 20, 1 << 15),
          ts=_lib.sd_stride(1 << 20, 1 << 15)), "too many rows")])
def test_verify_tokens_refuses(lib, kw, needle):
    _refused(_verify(lib, **kw), needle)


def test_workspace_queries_of_refused_sizes_are_zero(lib):
    assert lib.sd_token_logprobs_workspace(0, 10, 0) == 0
    assert lib.sd_token_logprobs_workspace(1, 0, 0) == 0
    assert lib.sd_token_logprobs_workspace(1, 10, 33) == 0
    assert lib.sd_verify_tokens_workspace(1, 65, 10) == 0
    assert lib.sd_verify_tokens_workspace(1, 1, (1 << 24) + 1) == 0
    assert lib.sd_token_logprobs_workspace(1, 10, 4) > 0 and lib.sd_verify_tokens_workspace(1, 1, 10) > 0


def test_the_binding_refuses_operands_off_the_gpu_or_of_another_shape():
    x = torch.zeros(2, 10)
    with pytest.raises(_lib.SpecDiffError, match="not on the current GPU"):
        _lib.sd_token_logprobs(x)
    with pytest.raises(_lib.SpecDiffError, match="contiguous rows"):
        _lib.sd_token_logprobs(torch.zeros(10, 2).T)
    with pytest.raises(_lib.SpecDiffError, match="target must be"):
        _lib.sd_verify_tokens(torch.zeros(2, 3, 10), torch.zeros(2, 3, 10), None, None)
    with pytest.raises(_lib.SpecDiffError, match="one type"):
        _lib.sd_verify_tokens(torch.zeros(2, 3, 10), torch.zeros(2, 4, 10).half(), None, None)


def _latent(lib, **kw):
    s = _lib.sd_stride_h
    a = dict(B=2, Q=2, H=4, dc=128, dr=64, type=1, scale=0.1, q=P, qs=s(1536, 768, 192), cache=P, ps=16 * 192, ts=192,
             n_pages=9, size=16, pages=P, pstride=4, max_pages=4, lens=P, rows=None, out=P, os=s(1024, 512, 128), lse=None,
             ws=P, ws_bytes=1 << 40)
    a.update(kw)
    return lib.sd_latent_attention(*a.values(), None)


@pytest.mark.parametrize("kw,needle", [
    (dict(B=0), "B >= 1"), (dict(Q=0), "B >= 1"), (dict(H=0), "B >= 1"), (dict(dc=0), "d_latent = 0"),
    (dict(dc=520), "d_latent = 520"), (dict(dc=132), "d_latent = 132"), (dict(dr=72), "d_rope = 72"),
    (dict(dr=-8), "d_rope"), (dict(dr=4), "d_rope = 4"), (dict(type=0), "type"), (dict(scale=float("nan")), "scale"),
    (dict(scale=float("inf")), "scale"), (dict(q=None), "NULL"), (dict(lens=None), "NULL"), (dict(ws=None), "NULL"),
    (dict(n_pages=0), "n_pages"), (dict(size=0), "page_size"), (dict(max_pages=5), "pages_stride"),
    (dict(size=1 << 28, ps=1 << 40), "2^30 tokens"), (dict(pages=None, n_pages=1), "n_pages = 1"),
    (dict(ts=184), "cache strides"), (dict(ts=196), "cache strides"), (dict(ps=100), "cache strides"),
    (dict(qs=_lib.sd_stride_h(1536, 768, 190)), "q strides"), (dict(qs=_lib.sd_stride_h(1536, 192, 192)), "q strides"),
    (dict(os=_lib.sd_stride_h(1024, 512, 120)), "out strides"), (dict(q=ctypes.c_void_p(264)), "16-byte"),
    (dict(cache=ctypes.c_void_p(258)), "16-byte"), (dict(ws_bytes=64), "workspace 64 <"),
    (dict(ws=ctypes.c_void_p(128)), "256-byte"), (dict(B=1 << 20, Q=1 << 10), "2^30 rows"),
    (dict(B=1 << 20, size=1 << 24, max_pages=4, ps=1 << 40), "too many rows and tokens")])
def test_latent_attention_refuses(lib, kw, needle):
    _refused(_latent(lib, **kw), needle)


def test_latent_binding_refuses():
    assert _lib.sd_latent_attention_workspace(1, 1, 1, 12, 0) == 0
    q, c, n = torch.zeros(1, 1, 2, 192).half(), torch.zeros(3, 16, 192).half(), torch.ones(1, dtype=torch.int32)
    with pytest.raises(_lib.SpecDiffError, match="agree in d"):
        _lib.sd_latent_attention(q, c[..., :184], n, 128)
    with pytest.raises(_lib.SpecDiffError, match="agree in d and type"):
        _lib.sd_latent_attention(q, c.bfloat16(), n, 128)
    with pytest.raises(_lib.SpecDiffError, match="not on the current GPU"):
        _lib.sd_latent_attention(q, c, n, 128)


def _expanded(lib, **kw):
    s = _lib.sd_stride_h
    a = dict(n=2, H=4, dn=128, dr=64, dv=128, type=1, scale=0.1, Tq=50, q=P, qs=s(0, 768, 192), Tk=90, k=P,
             ks=s(0, 1024, 256), kr=P, krs=64, v=P, vs=s(0, 1024, 256), cu_q=P, cu_k=P, out=P, os=s(0, 512, 128), lse=None,
             ws=P, ws_bytes=1 << 40)
    a.update(kw)
    return lib.sd_latent_attention_expanded(*a.values(), None)


@pytest.mark.parametrize("kw,needle", [
    (dict(n=0), ">= 1"), (dict(H=0), ">= 1"), (dict(Tq=0), ">= 1"), (dict(Tk=0), ">= 1"), (dict(dn=136), "d_nope = 136"),
    (dict(dn=0), "d_nope = 0"), (dict(dv=20), "d_v = 20"), (dict(dr=72), "d_rope = 72"), (dict(dr=60), "d_rope = 60"),
    (dict(type=0), "type"), (dict(scale=float("nan")), "scale"), (dict(q=None), "NULL"), (dict(kr=None), "NULL"),
    (dict(cu_k=None), "NULL"), (dict(qs=_lib.sd_stride_h(0, 768, 190)), "q strides"),
    (dict(qs=_lib.sd_stride_h(0, 700, 192)), "q strides"), (dict(ks=_lib.sd_stride_h(0, 1024, 120)), "k strides"),
    (dict(ks=_lib.sd_stride_h(0, 1 << 24, 256)), "k strides"), (dict(vs=_lib.sd_stride_h(0, 128, 128)), "v strides"),
    (dict(os=_lib.sd_stride_h(0, 512, 64)), "out strides"), (dict(krs=56), "k_rope stride"),
    (dict(krs=68), "k_rope stride"), (dict(v=ctypes.c_void_p(264)), "16-byte"), (dict(Tk=1 << 30), "too many rows"),
    (dict(Tq=1 << 29, H=8, qs=_lib.sd_stride_h(0, 1536, 192)), "too many rows"),
    (dict(n=1, Tk=8000, ws=None), "NULL workspace"), (dict(n=1, Tk=8000, ws_bytes=10), "workspace 10 <"),
    (dict(n=1, Tk=8000, ws=ctypes.c_void_p(128)), "256-byte")])
def test_expanded_refuses(lib, kw, needle):
    _refused(_expanded(lib, **kw), needle)


def test_expanded_binding_refuses():
    h, i = (lambda *s: torch.zeros(*s).half()), torch.zeros(3, dtype=torch.int32)
    with pytest.raises(_lib.SpecDiffError, match="agree in heads"):
        _lib.sd_latent_attention_expanded(h(5, 2, 192), h(9, 3, 128), h(9, 64), h(9, 3, 128), i, i)
    with pytest.raises(_lib.SpecDiffError, match="k_rope must be"):
        _lib.sd_latent_attention_expanded(h(5, 2, 192), h(9, 2, 128), None, h(9, 2, 128), i, i)
    with pytest.raises(_lib.SpecDiffError, match="not on the current GPU"):
        _lib.sd_latent_attention_expanded(h(5, 2, 192), h(9, 2, 128), h(9, 64), h(9, 2, 128), i, i)
    assert _lib.sd_latent_attention_expanded_workspace(1, 2, 130, 64, 128, 5, 9) == 0
