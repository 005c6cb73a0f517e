"""Rows in 8 bits on the GPU against the 64-bit oracle: the quantiser, the
modulated LayerNorm and the RMS norm with its residual.

Tolerances.  A code rounds 127 y / m, computed as fma(y, hi, y lo) with hi + lo
= 127 / m to 2^-47 and one rounding to fp32 (up to 2^-24 x 127 = 2^-17 steps),
or, of a norm's y, as y hi alone (hi off by 2^-24: 2^-17 steps) inside the
rounding.  So a code c is right if |c - 127 y / m| <= 1/2 + 2^-16 for the y that
the kernel has.  Of bf16 rows as they are the codes are exact.  A scale has the
roundings of one division.  A norm's own y is off by its fp32 statistics: a
lane sums up to 128 values one by one and 6 more steps join the lanes, so with
n = 136 roundings of 2^-24 a sum of positive numbers is off by n 2^-24 of
itself and a mean by that of the mean magnitude; the square root halves the
error of the variance; the products that follow add 6 roundings."""
import numpy as np
import pytest
import torch

from gpu_util import host, log, require_gpu
from oracle import rows_i8 as R

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
N_SUM = 136
TD = {"bf16": torch.bfloat16, "fp32": torch.float32}


@pytest.fixture(scope="module")
def B():
    return require_gpu()


def rows(seed, n, width, dtype, spread=0):
    """Normal values of per-row magnitudes 2^-spread .. 2^spread, a few channels larger, off centre."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((n, width)) + 0.25
    x[:, rng.integers(0, width, max(1, width // 100))] *= 7
    x *= 2.0 ** rng.integers(-spread, spread + 1, (n, 1))
    return torch.from_numpy(x).to(TD[dtype]).cuda()


def empty_codes(x, fill=99):
    return (torch.full(x.shape, fill, dtype=torch.int8, device="cuda"),
            torch.full((x.shape[0],), -1.0, dtype=torch.float32, device="cuda"))


def check_codes(codes, scales, y, err, what):
    """codes and scales against the row y in 64 bits, itself known to err (per row, absolute)."""
    c, s = codes.cpu().numpy().astype(np.float64), host(scales)
    m = np.maximum(np.abs(y).max(1), R.LEAST)
    off = np.abs(c - 127.0 * y / m[:, None]).max(1, initial=0.0)
    # m itself may be off by err: 127 y / m then by up to 127 (err / m) more
    allowed = 0.5 + 2.0 ** -16 + 254.0 * err / m
    log(f"  {what}: worst code {np.max(off, initial=0.0):.6f} steps off, worst scale {np.max(np.abs(s * 127 / m - 1), initial=0.0):.2e}")
    assert (off <= allowed).all(), (what, off.max(), np.argmax(off - allowed))
    assert (np.abs(s - m / 127) <= m / 127 * 2 * E + err / 127).all(), what


WIDTHS = [16, 32, 80, 512, 528, 1040, 1536, 2064, 2560, 3088, 3584, 4096, 5120, 6000, 7168, 8192,   # a wave's row
          8208, 11264, 13824, 16384, 20000, 32768,                                                  # a workgroup's
          32784, 65552]                                                                             # read twice


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("width", WIDTHS)
def test_quantize_rows(B, width, dtype):
    x = rows(width, 7, width, dtype, 20)
    codes, scales = empty_codes(x)
    B.quantize_rows(x, codes, scales)
    want, _ = R.quantize(host(x))
    check_codes(codes, scales, host(x), 0.0, f"rows {width} {dtype}")
    if dtype == "bf16":
        assert (codes.cpu().numpy() == want).all()


def test_values_in_the_middle_between_two_codes_go_to_the_even_one(B):
    """127 y / m = y / 2 exactly, with y the whole numbers up to 254."""
    x = torch.arange(-254, 255, dtype=torch.float32)
    x = torch.cat([x, x[:3]]).repeat(3, 1) * torch.tensor([[1.0], [2.0 ** -60], [2.0 ** 90]])
    for dtype in TD.values():
        d = x.to(dtype).cuda()
        codes, scales = empty_codes(d)
        B.quantize_rows(d, codes, scales)
        assert torch.equal(codes.cpu(), torch.round(x[0] / 2).to(torch.int8).repeat(3, 1))   # rounds to even


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n", [0, 1, 2, 3, 4, 5, 63, 1025])
def test_rows_behind_the_last_and_strided_rows(B, n, dtype):
    wide = rows(n + 1, n + 2, 320, dtype)
    x = wide[:n, 64:208]                                    # 144 wide, 320 apart
    buf = torch.full((n + 2, 256), 99, dtype=torch.int8, device="cuda")
    scales = torch.full((n + 3,), -1.0, device="cuda")
    B.quantize_rows(x, buf[:n, 16:160], scales[1:n + 1])    # scales at an address that is 4-byte aligned only
    want, s = R.quantize(host(x))
    if dtype == "bf16":
        assert (buf[:n, 16:160].cpu().numpy() == want).all()
    assert np.allclose(host(scales[1:n + 1]), s, rtol=2 * E, atol=0)
    buf[:n, 16:160] = 99
    assert (buf == 99).all() and scales[0] == -1 and (scales[n + 1:] == -1).all()


@pytest.mark.parametrize("width", [64, 5120, 13824, 40000])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_special_rows(B, width, dtype):
    """Zeros, tiny and huge values, infinities and NaN: each row by itself."""
    x = rows(3, 9, width, dtype)
    top = torch.finfo(TD[dtype]).max
    x[0] = 0
    x[1] = 0
    x[1, width - 1] = -torch.finfo(TD[dtype]).tiny / 2      # not a normal number
    x[2, 5] = float("inf")
    x[3, width - 1] = float("-inf")
    x[4, 0] = float("nan")
    x[5, :] = float("nan")
    x[6] = x[6].clamp(-1, 1) * top
    x[7, 0], x[7, 1:] = top, 1e-3
    # a NaN with every payload bit
    x[8].view(torch.int16 if dtype == "bf16" else torch.int32)[3] = -1
    codes, scales = empty_codes(x)
    B.quantize_rows(x, codes, scales)
    want, s = R.quantize(host(x))
    got, gs = codes.cpu().numpy(), host(scales)
    for r in (2, 3, 4, 5, 8):
        assert np.isnan(gs[r]) and (got[r] == 0).all()
    assert gs[0] == gs[1] == 2.0 ** -100 and (got[:2] == 0).all()
    for r in (6, 7):
        assert np.isclose(gs[r], s[r], rtol=2 * E, atol=0) and np.abs(got[r].astype(int) - want[r]).max() <= (dtype == "fp32")
    assert (got[7, 1:] == 0).all() and got[7, 0] == 127


def test_a_row_does_not_depend_on_the_others(B):
    for width in (1040, 13824):
        x = rows(11, 37, width, "fp32", 5)
        codes, scales = empty_codes(x)
        B.quantize_rows(x, codes, scales)
        for r in (0, 17, 36):
            c, s = empty_codes(x[:1])
            B.quantize_rows(x[r:r + 1], c, s)
            assert torch.equal(c[0], codes[r]) and torch.equal(s[0], scales[r])


def test_more_rows_than_a_launch_has_waves_and_offsets_past_32_bits(B):
    """17 million rows of 16 (a launch holds 16.8 million), and rows that begin behind 2^32 bytes."""
    n = (1 << 24) + 12345
    x = torch.zeros(n, 16, dtype=torch.bfloat16, device="cuda")
    x[:, 3] = (torch.arange(n, device="cuda") % 251 + 1).bfloat16()
    x[:, 4] = -x[:, 3] / 2
    codes, scales = empty_codes(x)
    B.quantize_rows(x, codes, scales)
    assert bool((codes[:, 3] == 127).all()) and bool((codes[:, 4] == -64).all())          # 63.5 to even
    assert int(codes.abs().long().sum()) == n * 191
    assert torch.allclose(scales, x[:, 3].float() / 127, rtol=2 * E, atol=0)
    gain = torch.ones(16, dtype=torch.bfloat16, device="cuda")
    codes.fill_(99)
    B.add_rms_norm(x, None, gain, 1e-6, codes=codes, scales=scales)
    assert bool((codes[:, 3] == 127).all()) and int((codes[:, 5] != 0).sum()) == 0
    codes.fill_(99)
    z = torch.zeros(1, 16, device="cuda")
    B.adaln_modulate_i8(x, z, z, 16, [0, n], 1e-6, codes, scales)
    assert bool((codes[:, 3] == 127).all()) and bool((codes != 99).all())
    del x, codes, scales
    far = torch.empty((1 << 31) + (1 << 20), dtype=torch.bfloat16, device="cuda")[:].view(-1, 1 << 20)
    x = far[:, 1024:1056]                                     # 2,049 rows, 2 MB apart
    x.copy_(rows(4, x.shape[0], 32, "bf16"))
    codes, scales = empty_codes(x)
    B.quantize_rows(x, codes, scales)
    assert (codes.cpu().numpy() == R.quantize(host(x))[0]).all()


CUS = {"one": [9], "packed": [3, 0, 1, 4, 1], "long": [130, 5, 66]}


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("lens", CUS)
@pytest.mark.parametrize("width", [16, 64, 384, 1040, 2048, 3584, 4096, 5120, 8192])
def test_adaln_modulate_i8(B, width, lens, dtype):
    if dtype == "fp32" and width > 4096:
        width = 4000
    lens = CUS[lens]
    cu = [0] + np.cumsum(lens).tolist()
    x = rows(width, cu[-1], width, dtype, 3)
    rng = np.random.default_rng(width + 1)
    mod = torch.from_numpy(rng.standard_normal((len(lens), 6, width)) * 0.4).float().cuda()
    codes, scales = empty_codes(x)
    eps = 1e-6
    B.adaln_modulate_i8(x, mod[:, 2], mod[:, 4], mod.stride(0), cu, eps, codes, scales)
    h, sh, sc = host(x), host(mod[:, 2]), host(mod[:, 4])
    y = R.modulate(h, sh, sc, cu, eps)
    # a mean off by N_SUM E mean|x|, an inverse deviation by (N_SUM / 2 + 2) E of itself and the mean's error once more
    # (squared, so nothing), 6 roundings of products and sums
    r = np.repeat(np.arange(len(lens)), lens)
    std = np.sqrt(h.var(1) + eps)
    mul = np.abs(1 + sc).max(1)[r]
    err = E * (N_SUM * np.abs(h).mean(1) / std * mul + (N_SUM / 2 + 8) * np.abs(y).max(1) + (N_SUM / 2 + 8) * np.abs(sh).max(1)[r])
    check_codes(codes, scales, y, err, f"modulate {width} {lens} {dtype}")
    # the values are those of the entry that writes them in the rows' type, before its rounding
    out = torch.empty_like(x)
    B.adaln_modulate(x, mod[:, 2], mod[:, 4], mod.stride(0), cu, eps, out)
    if dtype == "fp32":
        assert np.abs(codes.cpu().numpy() - R.steps(host(out))).max() <= 0.5 + 2.0 ** -16


def test_adaln_modulate_i8_rows_of_one_value_and_not_finite(B):
    """A row of one value has no deviation: it is shift alone; NaN and infinities stay in their row."""
    x = rows(2, 8, 512, "bf16")
    x[1], x[3, 4], x[5, 511] = 3.0, float("nan"), float("inf")
    mod = torch.from_numpy(np.random.default_rng(3).standard_normal((2, 512))).float().cuda()
    codes, scales = empty_codes(x)
    B.adaln_modulate_i8(x, mod[:1], mod[1:], 512, [0, 8], 1e-6, codes, scales)
    c, s = codes.cpu().numpy(), host(scales)
    for r in (3, 5):
        assert np.isnan(s[r]) and (c[r] == 0).all()
    sh = host(mod[:1])
    check_codes(codes[1:2], scales[1:2], sh, np.array([1e-6 * np.abs(sh).max()]), "shift alone")
    assert np.isfinite(s[[0, 1, 2, 4, 6, 7]]).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("mode", ["codes", "out", "both"])
@pytest.mark.parametrize("add", ["no", "new", "into_x", "into_z"])
@pytest.mark.parametrize("n,width", [(1, 16), (5, 64), (64, 384), (3, 1040), (9, 4096), (7, 5120), (2, 8192)])
def test_add_rms_norm(B, n, width, add, mode, dtype):
    if dtype == "fp32" and width > 4096:
        width = 3984
    x, z = rows(n, n, width, dtype, 3), rows(n + 50, n, width, dtype, 3)
    gain = (1 + 0.3 * rows(99, 1, width, dtype)[0]).to(TD[dtype])
    hx, hz, td = host(x), host(z), TD[dtype]
    total = torch.from_numpy(hx + hz).to(td) if add != "no" else x.cpu()   # fp32 sums: see below
    if add != "no":
        total = (x.cpu().float() + z.cpu().float()).to(td)
    sm = {"no": None, "new": torch.empty_like(x), "into_x": x, "into_z": z}[add]
    out = torch.empty_like(x) if mode != "codes" else None
    codes, scales = empty_codes(x) if mode != "out" else (None, None)
    B.add_rms_norm(x, None if add == "no" else z, gain, 1e-5, sm, out, codes, scales)
    s = (x if sm is None else sm).cpu()
    assert torch.equal(s, total)                       # the sum: one rounding of an fp32 addition
    y = R.rms(s.double().numpy(), host(gain), 1e-5)
    err = E * (N_SUM / 2 + 6) * np.abs(y).max(1)
    if codes is not None:
        check_codes(codes, scales, y, err, f"rms {n} x {width} {dtype} {add}")
    if out is not None:
        # one rounding to the type: half a step, relative to the value
        assert (np.abs(host(out) - y) <= np.abs(y) * (torch.finfo(td).eps / 2 + E * (N_SUM / 2 + 6))).all()


def test_add_rms_norm_may_write_its_norm_over_an_input(B):
    for n, width in ((5, 64), (40, 5120)):
        x, z, gain = rows(1, n, width, "bf16"), rows(2, n, width, "bf16"), rows(3, 1, width, "bf16")[0]
        s, o = torch.empty_like(x), torch.empty_like(x)
        B.add_rms_norm(x, z, gain, 1e-6, s, o)
        x1, z1 = x.clone(), z.clone()
        B.add_rms_norm(x1, z1, gain, 1e-6, x1, z1)
        assert torch.equal(x1, s) and torch.equal(z1, o)
        x2, z2 = x.clone(), z.clone()
        B.add_rms_norm(x2, z2, gain, 1e-6, z2, x2)
        assert torch.equal(z2, s) and torch.equal(x2, o)
        x3 = x.clone()
        B.add_rms_norm(x3, None, gain, 1e-6, out=x3)
        B.add_rms_norm(x, None, gain, 1e-6, out=o)
        assert torch.equal(x3, o)


@pytest.mark.parametrize("n,width,dtype", [(1, 8, "bf16"), (6, 24, "bf16"), (5, 1000, "bf16"), (3, 8184, "bf16"),
                                           (1, 4, "fp32"), (7, 20, "fp32"), (5, 1004, "fp32"), (3, 4092, "fp32")])
def test_add_rms_norm_without_codes_takes_widths_of_whole_vectors(B, n, width, dtype):
    """Rows beside each other whose ends lie inside a wave's vectors; the row behind the last stays as it was."""
    td = TD[dtype]
    x, z = rows(n, n, width, dtype, 3), rows(n + 50, n, width, dtype, 3)
    gain = (1 + 0.3 * rows(99, 1, width, dtype)[0]).to(td)
    sums, outs = torch.full((n + 1, width), 7.0, dtype=td, device="cuda"), torch.full((n + 1, width), 7.0, dtype=td, device="cuda")
    B.add_rms_norm(x, z, gain, 1e-5, sums[:n], outs[:n])
    assert torch.equal(sums[:n].cpu(), (x.cpu().float() + z.cpu().float()).to(td))
    y = R.rms(host(sums[:n]), host(gain), 1e-5)
    # one rounding to the type: half a step, relative to the value
    assert (np.abs(host(outs[:n]) - y) <= np.abs(y) * (torch.finfo(td).eps / 2 + E * (N_SUM / 2 + 6))).all()
    assert bool((sums[n] == 7).all()) and bool((outs[n] == 7).all())


def test_add_rms_norm_rows_that_are_not_finite(B):
    x, z = rows(1, 6, 256, "fp32"), rows(2, 6, 256, "fp32")
    x[1, 3], z[2, 0], x[4, 255], z[4, 255] = float("nan"), float("inf"), float("inf"), float("-inf")
    codes, scales = empty_codes(x)
    sm = torch.empty_like(x)
    B.add_rms_norm(x, z, torch.ones(256, device="cuda"), 1e-6, sm, None, codes, scales)
    bad = torch.tensor([False, True, True, False, True, False])
    assert torch.equal(scales.isnan().cpu(), bad) and bool((codes[bad.cuda()] == 0).all())
    assert bool((codes[~bad.cuda()] != 0).any(1).all())


def test_streams_graphs_and_two_calls_at_once(B):
    """Each entry captured, replayed with other inputs and eager calls between; two streams at once."""
    n, w = 333, 5120
    mod = torch.randn(1, 2 * w, device="cuda")
    gain = rows(4, 1, w, "bf16")[0]

    def calls(x, z, out):
        B.quantize_rows(x, *out[0])
        B.adaln_modulate_i8(x, mod[:, :w], mod[:, w:], 2 * w, [0, n], 1e-6, *out[1])
        B.add_rms_norm(x, z, gain, 1e-6, out[3], None, *out[2])

    def fresh():
        x = rows(0, n, w, "bf16")
        return [empty_codes(x), empty_codes(x), empty_codes(x), torch.empty_like(x)]

    x, z = rows(1, n, w, "bf16"), rows(2, n, w, "bf16")
    held, want = fresh(), fresh()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls(x, z, held)
    flat = lambda o: [t for p in o[:3] for t in p] + [o[3]]
    for k in range(4):
        x.copy_(rows(10 + k, n, w, "bf16"))
        z.copy_(rows(20 + k, n, w, "bf16"))
        graph.replay()
        calls(x, z, want)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(flat(held), flat(want))), k
    a, b = fresh(), fresh()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(5):
        with torch.cuda.stream(s1):
            calls(x, z, a)
        with torch.cuda.stream(s2):
            calls(x, z, b)
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) and torch.equal(p, r) for p, q, r in zip(flat(want), flat(a), flat(b)))


@pytest.mark.parametrize("add", [True, False])
def test_codes_of_the_rms_norm_of_bf16_rows_are_exact(B, add):
    """1 / rms is a factor of the whole row, so a code rounds 127 (s g) / max|s g|, and s g of bf16 numbers has 16 bits.
    In 64 bits 127 s g is exact and its quotient is rounded once, so rint sees a middle between two codes exactly where
    there is one; any other quotient z is z / (254 x 65025) from it at least, more than half a step of fp32 at z."""
    n, width = 300, 5120
    x, z = rows(21, n, width, "bf16", 3), rows(22, n, width, "bf16", 3)
    gain = (1 + 0.2 * rows(23, 1, width, "bf16")[0]).bfloat16()
    total = torch.empty_like(x) if add else None
    codes, scales = empty_codes(x)
    B.add_rms_norm(x, z if add else None, gain, 1e-6, total, None, codes, scales)
    s = host(total if add else x)
    steps = R.steps(s * host(gain))
    ties = np.abs(steps) % 1 == 0.5
    log(f"  {int(ties.sum())} values in the middle between two codes, of {ties.size}")
    assert ties.sum() >= 5
    wrong = codes.cpu().numpy() != np.rint(steps).astype(np.int8)
    assert not wrong.any(), f"{int(wrong.sum())} codes, {int((wrong & ties).sum())} of them ties"
    both, more = empty_codes(x)
    out = torch.empty_like(x)
    B.add_rms_norm(x, z if add else None, gain, 1e-6, total, out, both, more)
    assert torch.equal(both, codes) and torch.equal(more, scales)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_middles_of_the_rms_norm_go_to_the_even_code(B, dtype):
    """s = the whole numbers up to 254 and gains of powers of two: 127 y / m = s / 2 exactly."""
    x = torch.arange(-254, 255, dtype=torch.float32)
    x = torch.cat([x, x[:3]]).repeat(3, 1) * torch.tensor([[1.0], [2.0 ** -30], [2.0 ** 40]])
    d = x.to(TD[dtype]).cuda()
    for g in (1.0, 0.25, -4096.0):
        gain = torch.full((512,), g, dtype=TD[dtype], device="cuda")
        codes, scales = empty_codes(d)
        B.add_rms_norm(d, None, gain, 1e-30, codes=codes, scales=scales)
        assert torch.equal(codes.cpu(), torch.round(x[0] / 2 * np.sign(g)).to(torch.int8).repeat(3, 1)), g
        y = R.rms(x.double().numpy(), np.full(512, g), 1e-30)
        assert np.allclose(host(scales), R.quantum(y), rtol=E * (N_SUM / 2 + 6), atol=0)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rms_norm_rows_at_the_ends_of_the_range(B, dtype):
    """Rows of zeros and of products below the least scale; a norm that passes the largest number in its last factor."""
    x = torch.zeros(4, 64, dtype=TD[dtype], device="cuda")
    x[1], x[2], x[3] = 1.0, 3.0, 1.0
    gain = torch.full((64,), 2.0 ** -110, dtype=TD[dtype], device="cuda")
    codes, scales = empty_codes(x)
    B.add_rms_norm(x, None, gain, 1e-6, codes=codes, scales=scales)
    assert bool((scales == 2.0 ** -100).all()) and bool((codes == 0).all())
    # y = 1.5 sqrt(64 / 9) x the largest power of two: above the range, though both factors of it are inside
    x[1], x[1, 9:] = 1.5, 0
    gain.fill_(2.0 ** 127)
    out = torch.empty_like(x)
    B.add_rms_norm(x, None, gain, 1e-6, None, out, codes, scales)
    assert bool(out[1, :9].isinf().all()) and bool(scales[1].isnan()) and bool((codes[1] == 0).all())
    assert bool((codes[0] == 0).all()) and bool((codes[2:] == 127).all()) and bool(scales[2:].isfinite().all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("width", [16, 64, 528, 1040, 2064, 3600])
def test_adaln_modulate_i8_large_rows_of_one_value(B, width, dtype):
    """2^112 throughout: the sums and the mean are exact, the deviations 0 and the row is its shift, though 2^112 over the
    deviation's floor of 1e-6, which a place behind the row could come to, is above the largest number."""
    x = torch.full((5, width), 2.0 ** 112, dtype=TD[dtype], device="cuda")
    mod = torch.from_numpy(np.random.default_rng(width).standard_normal((2, 2, width))).float().cuda()
    codes, scales = empty_codes(x)
    B.adaln_modulate_i8(x, mod[:, 0], mod[:, 1], 2 * width, [0, 2, 5], 1e-12, codes, scales)
    sh = host(mod[:, 0])[[0, 0, 1, 1, 1]]
    check_codes(codes, scales, sh, np.zeros(5), f"shift alone {width} {dtype}")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_the_affine_layer_norm_as_codes(B, dtype):
    """One request with the gains less 1 and the offsets in fp32: the norm of layer_norm_affine."""
    n, width = 37, 1040
    x, g, b = rows(31, n, width, dtype, 3), rows(32, 1, width, dtype)[0], rows(33, 1, width, dtype)[0]
    codes, scales = empty_codes(x)
    B.adaln_modulate_i8(x, b.float()[None], (g.float() - 1)[None], 0, [0, n], 1e-6, codes, scales)
    h, hg, hb = host(x), host(g), host(b)
    d = h - h.mean(1, keepdims=True)
    std = np.sqrt((d * d).mean(1, keepdims=True) + 1e-6)
    y = d / std * hg + hb
    # the errors of test_adaln_modulate_i8, and the two roundings of 1 + (g - 1), each up to E of 1 + |g|
    err = E * (N_SUM * np.abs(h).mean(1) / std[:, 0] * np.abs(hg).max() + (N_SUM / 2 + 8) * (np.abs(y).max(1) + np.abs(hb).max()) +
               2 * np.abs(d / std).max(1) * (1 + np.abs(hg).max()))
    check_codes(codes, scales, y, err, f"affine {dtype}")
    out = torch.empty_like(x)
    B.layer_norm_affine(x, g, b, 1e-6, out)
    assert (np.abs(host(out) - y) <= err[:, None] + torch.finfo(x.dtype).eps / 2 * (np.abs(y) + err[:, None])).all()
