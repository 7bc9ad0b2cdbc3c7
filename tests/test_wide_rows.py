"""The attention kernel of 128 rows a workgroup: how many rows of a block each of its four wavefronts stores.

A wavefront without a row stores nothing: it has no address for one.
"""
import os
import subprocess

from paper_2606_13426_amd import build

MAIN = """
#include "latent_wide.hpp"
#include <cstdio>
int main() {
  for (int rows = 0; rows <= sd::latent::kWideRows; ++rows)
    for (int w = 0; w < 4; ++w) std::printf("%d\\n", sd::latent::rows_of_wave(rows, w));
}
"""


def test_rows_of_a_block_by_wavefronts(tmp_path):
    src, exe = tmp_path / "rows.hip", tmp_path / "rows"
    src.write_text(MAIN)
    subprocess.run([build._hipcc(), "--cuda-host-only", "-std=c++17", "-I", os.path.join(build.ROOT, "include"), "-I",
                    os.path.join(build.HERE, "csrc"), str(src), "-o", str(exe)], check=True, capture_output=True)
    got = [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    assert got == [len(range(w, rows, 4)) for rows in range(129) for w in range(4)]
