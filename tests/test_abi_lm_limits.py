"""Views and sizes of the language-model calls that no launch may get; none reaches a HIP call."""
import pytest

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
