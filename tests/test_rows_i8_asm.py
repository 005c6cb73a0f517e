"""The kernels of rows in 8 bits hold a row in registers: no compiled instance
keeps any of it in scratch memory."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2606_13501_amd import build as B


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    if not os.path.exists(B.HIPCC) and shutil.which(B.HIPCC) is None:
        pytest.skip("hipcc not available")
    out = tmp_path_factory.mktemp("asm") / "rows_i8.s"
    flags = [f for f in B.FLAGS if f != "-fPIC"] + B.EXTRA.get("rows_i8.hip", [])
    cmd = [B.HIPCC] + flags + ["-x", "hip", "--cuda-device-only", "-S", os.path.join(B.CSRC, "rows_i8.hip"), "-o", str(out)]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    lines = out.read_text().split("\n")
    found = {}
    for h in [i for i, l in enumerate(lines) if re.match(r"^_Z\S*(rows_i8|modulate_i8|add_rms)\S*:", l)]:
        end = next(i for i in range(h, len(lines)) if lines[i].startswith(".Lfunc_end"))
        found[lines[h].split(":")[0]] = lines[h:end]
    return found


def test_every_kernel_is_compiled(kernels):
    # 12 counts of a wave's vectors, 6 of a workgroup's, rows read twice; two types
    for name, count in (("modulate_i8_kernel", 24), ("add_rms_kernel", 24), ("rows_i8_kernel", 36), ("rows_i8_wide_kernel", 2)):
        assert sum(name in k for k in kernels) == count, name


def test_no_kernel_spills(kernels):
    spilled = {name: sum("scratch_" in l for l in body) for name, body in kernels.items()}
    assert not {name: n for name, n in spilled.items() if n}
