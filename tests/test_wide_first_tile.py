"""The attention kernel of 128 rows a workgroup: a wavefront's weights take the place of a tile's rotary parts.

All wavefronts have to have read those as keys by then.  From the second tile on the barrier of the tile before says so;
the first tile of a run has one of its own: in the assembly, between the first scores' products (then O is zeroed) and
the products of the first tile.
"""
import os
import re
import subprocess

import pytest

from paper_2606_13426_amd import build

CSRC = os.path.join(build.HERE, "csrc")


@pytest.mark.parametrize("name", ["latent_wide_bf16.hip", "latent_wide_f16.hip"])
def test_a_barrier_before_the_first_tile(name, tmp_path):
    out = tmp_path / "kernel.s"
    subprocess.run([build._hipcc(), *build.FLAGS, *build.MORE_FLAGS[name], "-I", os.path.join(build.ROOT, "include"), "-I", CSRC,
                    "--cuda-device-only", "-S", os.path.join(CSRC, name), "-o", str(out)], check=True, capture_output=True)
    code, kernel = [], False
    for line in out.read_text().splitlines():
        text = line.split(";")[0].strip()
        if re.match(r"_ZN2sd6latent18latent_wide_kernel\w*:", text):
            kernel = True
        elif text.startswith(".section") or text.startswith("s_endpgm"):
            kernel = False
        elif kernel and re.match(r"v_mfma|s_barrier|ds_write_b128", text):
            code.append(text)
    zeroed = [i for i, text in enumerate(code) if re.match(r"v_mfma\S* a\[\w+:\w+\],.*, 0$", text)]
    assert len(zeroed) == 16
    behind = code[zeroed[-1] + 1:]
    assert behind[0] == "s_barrier" and any(text.startswith("ds_write_b128") for text in behind)
