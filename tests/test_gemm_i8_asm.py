"""The tiled 8-bit GEMM issues its MFMAs as inline assembly on the accumulation
registers, as the bf16 one does: the same checks of every compiled instance.  No
instruction but the next MFMA touches an accumulator within the wait states after
an MFMA that writes it, no MFMA reads a register that a vector instruction wrote
in the 2 wait states before it, and the K loop neither copies accumulators nor
spills nor waits for all loads in flight.  The loads into LDS are assembly too:
the register with their LDS address is theirs, and no scalar register that a
vector instruction wrote is read by a load in the 5 wait states after it (in both
kernels, over every path)."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2606_13501_amd import build as B
from test_attention_asm import _blocks, scan
from test_gemm_asm import _flat

SHAPES = ["ILi8ELi8ELi2E", "ILi8ELi6ELi2E", "ILi4ELi8ELi2E", "ILi4ELi6ELi3E", "ILi4ELi4ELi4E"]


@pytest.fixture(scope="module")
def every_kernel(tmp_path_factory):
    if not os.path.exists(B.HIPCC) and shutil.which(B.HIPCC) is None:
        pytest.skip("hipcc not available")
    out = tmp_path_factory.mktemp("asm") / "gemm_i8.s"
    flags = [f for f in B.FLAGS if f != "-fPIC"] + B.EXTRA.get("gemm_i8.hip", [])
    cmd = [B.HIPCC] + flags + ["-x", "hip", "--cuda-device-only", "-S", os.path.join(B.CSRC, "gemm_i8.hip"), "-o", str(out)]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    lines = out.read_text().split("\n")
    found = {}
    for h in [i for i, l in enumerate(lines) if re.match(r"^_Z\S*gemm_i8_(nt|few)\S*:", l)]:
        end = next(i for i in range(h, len(lines)) if lines[i].startswith(".Lfunc_end"))
        found[lines[h].split(":")[0]] = lines[h:end]
    return found


@pytest.fixture(scope="module")
def kernels(every_kernel):
    return {name: body for name, body in every_kernel.items() if "gemm_i8_nt" in name}


def test_every_shape_epilogue_and_type_is_compiled(kernels):
    for shape in SHAPES:
        assert sum(shape in name for name in kernels) == 8, shape


def test_accumulators_keep_their_distance(kernels):
    for name, body in kernels.items():
        problems = scan([_flat(l) for l in body])
        assert not problems, f"{name}:\n" + "\n".join(f"line {i}: {m}" for i, m in problems[:10])


def test_k_loop_has_no_copies_and_no_full_waits(kernels):
    """The halves of the steps: no copies of accumulators, no spills in the kernel, waits that leave loads in flight."""
    for name, body in kernels.items():
        assert not [l for l in body if "scratch_" in l], name
        halves = [b for b in _blocks(body) if any("v_mfma" in l for _, l, _ in b["ins"])]
        assert len(halves) >= 4, name
        ins = [l for b in halves for _, l, _ in b["ins"]]
        assert not [l for l in ins if l.startswith(("v_accvgpr", "v_writelane"))], name
        steady = [b for b in halves if not any(l.startswith("buffer_load_dword ") for _, l, _ in b["ins"])]
        assert len(steady) == len(halves) - 1, name     # a tile's last half also loads the scales
        assert not [l for b in steady for _, l, _ in b["ins"] if l.startswith("v_readlane")], name
        waits = [int(m.group(1)) for l in ins for m in re.finditer(r"vmcnt\((\d+)\)", l)]
        assert waits and min(waits) >= 6, f"{name}: vmcnt waits {waits}"


def test_the_lds_address_of_a_load_is_the_one_set_for_it(kernels):
    """Between the instruction that sets m0 and its load, which are separate statements, nothing else writes m0."""
    for name, body in kernels.items():
        writer, loads = None, 0
        for l in body:
            l = l.strip()
            if re.match(r"s_\w+ m0\b", l):
                writer = l
            elif l.startswith(("s_", "v_")) and re.search(r"\bm0\b", l.split(",")[0]):
                raise AssertionError(f"{name}: {l}")
            elif l.startswith("buffer_load") and l.endswith("lds"):
                assert writer is not None, f"{name}: {l} without its own address"
                writer, loads = None, loads + 1
        assert loads > 8, name


def _scalars(text):
    out = set()
    for m in re.finditer(r"\bs\[(\d+):(\d+)\]", text):
        out.update(range(int(m.group(1)), int(m.group(2)) + 1))
    out.update(int(m.group(1)) for m in re.finditer(r"\bs(\d+)\b", text))
    return out


def _vector_writes(l):
    """Scalar registers that a vector instruction writes."""
    op = l.split()[0]
    if op.startswith(("v_readlane", "v_readfirstlane")):
        return _scalars(l.split(",")[0])
    if op.startswith("v_cmp") and not op.startswith("v_cmpx"):
        return _scalars(l.split(",")[0])
    if op.startswith(("v_add_co", "v_sub_co", "v_addc_co", "v_subb_co", "v_mad_u64", "v_mad_i64", "v_div_scale")):
        return _scalars(l.split(",")[1])
    return set()


def scalar_hazards(body, need=5):
    """Loads and stores that read a scalar register less than `need` wait states after a vector instruction wrote it."""
    blocks, bad = _blocks(body), []
    entry, work = [None] * len(blocks), [0]
    entry[0] = {}                       # register -> wait states since the write, where fewer than needed
    while work:
        k = work.pop()
        age = dict(entry[k])
        for i, l, _ in blocks[k]["ins"]:
            if l.startswith(("buffer_", "global_", "scratch_", "flat_")):
                bad += [(i, l) for r in _scalars(l) if r in age]
            m = re.match(r"s_nop (\d+)", l)
            n = int(m.group(1)) + 1 if m else 1
            age = {r: a + n for r, a in age.items() if a + n < need}
            written = _vector_writes(l)
            if not written and re.match(r"s_(?!cmp|bitcmp|cbranch|branch|waitcnt|nop|barrier|endpgm)", l):
                for r in _scalars(l.split(",")[0]):
                    age.pop(r, None)    # written anew by the scalar unit
            age.update((r, 0) for r in written)
        for s in blocks[k]["succ"]:
            joined = dict(age) if entry[s] is None else {r: min(entry[s].get(r, need), age.get(r, need)) for r in {*entry[s], *age}}
            if joined != entry[s]:
                entry[s] = joined
                work.append(s)
    return bad


def test_the_hazard_scan_finds_one():
    lines = ["v_readlane_b32 s7, v1, 0", "s_mov_b32 m0, s2", "s_nop 0", "buffer_load_dword v0, s[4:7], 0 offen lds", "s_endpgm"]
    assert scalar_hazards(lines)
    assert not scalar_hazards(lines[:2] + ["s_nop 3"] + lines[3:])
    assert not scalar_hazards(["v_readlane_b32 s7, v1, 0", "s_mov_b32 s7, s2"] + lines[3:])


def test_loads_keep_their_distance_from_vector_written_scalars(every_kernel):
    assert len(every_kernel) == 72
    for name, body in every_kernel.items():
        problems = scalar_hazards(body)
        assert not problems, f"{name}:\n" + "\n".join(f"line {i}: {l}" for i, l in problems[:10])
