"""sd_latent_attention_expanded with many short sequences: each workgroup finds its own
among them in steps of 64 ways, so that the work grows with the rows and not with the
square of the sequences.
"""
import pytest
import torch

import test_gpu_latent_expanded as expanded
from paper_2606_13426_amd import _lib

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("n", [63, 64, 65, 128, 129, 4095, 4096, 4097, 70000])
@pytest.mark.parametrize("first", [0, 300])
def test_every_sequence_is_found(n, first):
    # lengths 0, 1, 2 and, at both ends and inside, a few of more than a tile of rows
    nq = [(i * 7) % 3 for i in range(n)]
    for i in (0, 1, n // 2, n - 2, n - 1):
        nq[i] = 130 + i % 5
    nk = [a + (i % 4) for i, a in enumerate(nq)]
    q, k, kr, v, cq, ck = expanded._case(nq, nk, 1, 16, 8, 16, "bf16", n, extra=first)
    out = torch.full((q.shape[0], 1, 16), 5.0, dtype=q.dtype, device=DEV)
    got = _lib.sd_latent_attention_expanded(q, k, kr, v, cq, ck, out=out)
    some = sorted({0, 1, 2, 62, n // 2 - 1, n // 2, n - 3, n - 2, n - 1} | {(n * i) // 23 for i in range(23)})
    expanded._check(q, k, kr, v, cq, ck, 24 ** -0.5, got, "bf16", seqs=some)
    # every row of a sequence was written (rows without a key are 0), the others were not
    a, b = int(cq[0]), int(cq[-1])
    assert not (out[a:b] == 5.0).all(-1).any()
    assert (out[:a] == 5.0).all() and (out[b:] == 5.0).all()


def test_the_time_grows_with_the_sequences():
    def us(n):
        x = torch.randn(n, 1, 64, device=DEV).half()
        cu = torch.arange(n + 1, device=DEV, dtype=torch.int32)
        out, lse = _lib.sd_latent_attention_expanded(x, x, None, x, cu, cu)
        best = float("inf")
        for _ in range(3):
            e = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
            e[0].record()
            _lib.sd_latent_attention_expanded(x, x, None, x, cu, cu, out=out, lse=lse)
            e[1].record()
            torch.cuda.synchronize()
            best = min(best, e[0].elapsed_time(e[1]) * 1e3)
        return best

    # 16 times the sequences: 16 times the work, and one more step of the search; a scan of all
    # sequences by every workgroup took 256 times as long
    assert us(1 << 17) <= 64 * us(1 << 13)
