"""The attention kernel of 128 rows a workgroup keeps its sums in the accumulation registers by name.

The compiler is told that they are overwritten, not what they hold, so it must not use them for anything of its
own: in the assembly that it makes, every mention of one lies in a statement of the source's.  And the loop
must not reload registers from memory: such a load would wait for the tile loads before it.
"""
import os
import re
import subprocess

import pytest

from paper_2606_13426_amd import build

CSRC = os.path.join(build.HERE, "csrc")


@pytest.mark.parametrize("name", ["latent_wide_bf16.hip", "latent_wide_f16.hip"])
def test_accumulation_registers_are_named_by_the_source_alone(name, tmp_path):
    out = tmp_path / "kernel.s"
    subprocess.run([build._hipcc(), *build.FLAGS, *build.MORE_FLAGS[name], "-I", os.path.join(build.ROOT, "include"), "-I", CSRC,
                    "--cuda-device-only", "-S", os.path.join(CSRC, name), "-o", str(out)], check=True, capture_output=True)
    kernel, own, products, blocks, block = False, False, 0, [], None
    for line in out.read_text().splitlines():
        text = line.strip()
        if re.match(r"_ZN2sd6latent18latent_wide_kernel\w*:", text):
            kernel = True
        if text.startswith(".section") or text.startswith("s_endpgm"):
            kernel = False
        if not kernel:
            continue
        if "#ASMSTART" in text or "#ASMEND" in text:
            own = "#ASMSTART" in text
            continue
        if line.startswith(".LBB"):
            block = dict(products=0, scratch=0)
            blocks.append(block)
        code = text.split(";")[0]
        if not own:
            assert "accvgpr" not in code and not re.search(r"\ba(\d+|\[)", code), line
        elif "v_mfma" in code:
            products += 1
        if block is not None:
            block["products"] += "v_mfma" in code
            block["scratch"] += "scratch_" in code
    assert products >= 16 + 3 * 32  # O zeroed, and three copies of a tile's products
    assert all(b["scratch"] == 0 for b in blocks if 5 <= b["products"] < 36)
    assert re.search(r"\.agpr_count:\s+256", out.read_text())
