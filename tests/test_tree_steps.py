"""The steps of tree verification: one wavefront of a workgroup finds its list of nodes.

Nodes are decided by other workgroups while a step runs, and the wavefronts of one meet in barriers at every node
of their list: with lists of their own, taken from states that they read at different times, they would put slices of two nodes
into one.  In the assembly that the compiler makes of every step kernel, what comes before the first barrier is then the
list alone: one load of the states (past the caches), by the first 64 threads, and no element of a row yet.
"""
import os
import re
import subprocess

from paper_2606_13426_amd import build

CSRC = os.path.join(build.HERE, "csrc")


def test_one_wavefront_reads_the_states_before_the_first_barrier(tmp_path):
    out = tmp_path / "tree.s"
    subprocess.run([build._hipcc(), *build.FLAGS, "-I", os.path.join(build.ROOT, "include"), "-I", CSRC, "--cuda-device-only", "-S",
                    os.path.join(CSRC, "tree.hip"), "-o", str(out)], check=True, capture_output=True)
    kernels, name = {}, None
    for line in out.read_text().splitlines():
        text = line.split(";")[0].strip()
        start = re.match(r"(_ZN2sd\w*tree_step_kernel\w*):", text)
        if start:
            name = start.group(1)
            kernels[name] = []
        elif text.startswith(".section"):
            name = None
        elif name:
            kernels[name].append(text)
    assert len(kernels) == 3 * 2 * 3  # types, elements a thread, sums
    for name, code in kernels.items():
        before = code[:next(i for i, text in enumerate(code) if text.startswith("s_barrier"))]
        loads = [text for text in before if re.match(r"(global|flat|buffer)_load", text)]
        assert sorted(text.split()[0] for text in loads) == ["global_load_dword", "global_load_dwordx2"], (name, loads)
        state = next(i for i, text in enumerate(before) if text.startswith("global_load_dword "))
        assert before[state].endswith("sc1"), name
        assert any(re.match(r"v_cmp_(gt|lt)_u32\w*\s+.*\b(64|63)\b, v0$", text) for text in before[:state]), name
        assert any(text.startswith("ds_write") for text in before[state:]), name
