"""Views and sizes of the language-model calls that no launch may get; none reaches a HIP call."""
import os
import warnings

import pytest
import torch

import test_abi_lm as abi
from paper_2606_13426_amd import _lib

lib = abi.lib
S = _lib.sd_stride_h


@pytest.mark.parametrize("os", [S(512, 512, 128), S(1016, 512, 128), S(128, 512, 128), S(768, 128, 256)])
def test_sequences_of_the_output_may_not_overlap(lib, os):
    abi._refused(abi._latent(lib, os=os), "out strides")


@pytest.mark.parametrize("os", [S(1024, 512, 128), S(512, 1024, 128), S(256, 512, 1024), S(128, 1024, 256),
                                S(512, 128, 1024), S(1536, 1024, 128)])
def test_outputs_nested_in_any_order_do_not(lib, os):
    abi._refused(abi._latent(lib, os=os, ws_bytes=64), "workspace 64 <")  # the check behind


def test_more_heads_than_a_grid_holds(lib):
    a = dict(n=1, Tq=1, Tk=1, qs=S(0, 0, 192), ks=S(0, 0, 256), vs=S(0, 0, 256), os=S(0, 0, 128))
    abi._refused(abi._expanded(lib, H=65536, **a), "too many rows")
    abi._refused(abi._expanded(lib, H=65535, scale=float("nan"), **a), "scale")  # the check behind
    assert lib.sd_latent_attention_expanded_workspace(1, 65536, 128, 64, 128, 1, 8000) == 0


@pytest.mark.parametrize("call", ["logprobs", "verify", "expanded"])
def test_more_workgroups_than_a_launch_holds(lib, call):
    """A launch's first dimension holds fewer than 2^32 threads: 2^24 - 1 workgroups of 256."""
    if call == "logprobs":
        s = abi._logprobs(lib, rows=1 << 24, V=1, ld=1, n_tok=0, n_top=0, ws_bytes=2 ** 62)
    elif call == "verify":
        s = abi._verify(lib, B=(1 << 24) // 3 + 1, K=1, V=1, ds=_lib.sd_stride(1, 1), ts=_lib.sd_stride(2, 1), ws_bytes=2 ** 62)
    else:
        s = abi._expanded(lib, n=(1 << 24) - 1, H=1, Tq=256, Tk=1 << 20, qs=S(0, 192, 192), os=S(0, 128, 128))
    abi._refused(s, "too many rows")


def test_widths_that_the_binding_cannot_split():
    h, i = (lambda *s: torch.zeros(*s).half()), torch.zeros(3, dtype=torch.int32)
    for d_latent in (-8, 0, 200):
        with pytest.raises(_lib.SpecDiffError, match="d_latent = "):
            _lib.sd_latent_attention(h(1, 1, 2, 192), h(3, 16, 192), i[:1], d_latent, scale=0.1)
    with pytest.raises(_lib.SpecDiffError, match="d_nope = 0"):
        _lib.sd_latent_attention_expanded(h(5, 2, 0), h(9, 2, 0), None, h(9, 2, 128), i, i)


def test_an_absorbed_call_without_a_scale_warns():
    """The default, (d_latent + d_rope)^-1/2, is not the scale of any model's expanded form."""
    q, c, n = torch.zeros(1, 1, 2, 192).half(), torch.zeros(3, 16, 192).half(), torch.ones(1, dtype=torch.int32)
    with pytest.warns(UserWarning, match="d_nope"), pytest.raises(_lib.SpecDiffError):
        _lib.sd_latent_attention(q, c, n, 128)
    with warnings.catch_warnings(), pytest.raises(_lib.SpecDiffError, match="not on the current GPU"):
        warnings.simplefilter("error")
        _lib.sd_latent_attention(q, c, n, 128, scale=192 ** -0.5)


def test_the_readmes_absorbed_call_has_a_scale():
    with open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")) as f:
        calls = [line for line in f if "sd_latent_attention(" in line]
    assert calls and all("scale=" in line for line in calls)
