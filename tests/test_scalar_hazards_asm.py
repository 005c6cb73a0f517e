"""Loads into LDS are inline assembly in every kernel file that has them, so the
compiler does not keep their distance: no load or store reads a scalar register
in the 5 wait states after a vector instruction wrote it, in any compiled kernel
of the files beside the 8-bit GEMM's, over every path."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2606_13501_amd import build as B
from test_gemm_i8_asm import scalar_hazards

FILES = ["gemm.hip", "attention.hip", "cached_attention.hip"]


def test_the_files_with_such_loads():
    """gemm.hip and gemm_i8.hip take theirs from gemm_tiles.hpp too."""
    own = {f for f in os.listdir(B.CSRC) if re.search(r'asm[^;]*buffer_load', open(os.path.join(B.CSRC, f)).read())}
    assert own == {"gemm_tiles.hpp", "gemm_i8.hip", "attention.hip", "cached_attention.hip"}
    users = {f for f in os.listdir(B.CSRC) if '"gemm_tiles.hpp"' in open(os.path.join(B.CSRC, f)).read()}
    assert users == {"gemm.hip", "gemm_i8.hip"}


@pytest.mark.parametrize("source", FILES)
def test_loads_keep_their_distance_from_vector_written_scalars(source, tmp_path):
    if not os.path.exists(B.HIPCC) and shutil.which(B.HIPCC) is None:
        pytest.skip("hipcc not available")
    out = tmp_path / "kernels.s"
    flags = [f for f in B.FLAGS if f != "-fPIC"] + B.EXTRA.get(source, [])
    cmd = [B.HIPCC] + flags + ["-x", "hip", "--cuda-device-only", "-S", os.path.join(B.CSRC, source), "-o", str(out)]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    lines, kernels, loads = out.read_text().split("\n"), 0, 0
    for h in [i for i, l in enumerate(lines) if re.match(r"^_Z\S+:", l)]:
        end = next((i for i in range(h, len(lines)) if lines[i].startswith(".Lfunc_end")), None)
        body = lines[h:end]
        if end is None or not any(l.strip().startswith(("buffer_", "global_")) for l in body):
            continue
        kernels, loads = kernels + 1, loads + sum(l.strip().endswith("lds") for l in body)
        problems = scalar_hazards(body)
        assert not problems, f"{lines[h]}:\n" + "\n".join(f"line {i}: {l}" for i, l in problems[:10])
    assert kernels >= 4 and loads > 8
