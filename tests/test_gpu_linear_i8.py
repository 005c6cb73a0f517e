"""dit_linear_i8 on the GPU against the 64-bit oracle, whose sums are exact.

Tolerances.  The 32-bit sum S is exact; z = fma(fl(fl(S) sa), sw, bias) has three
roundings of up to E = 2^-24 of |S sa sw| or of z, a residual and a gate one
rounding each; one rounding to the output's type follows, half a step of it
relative to the value.  GELU's factor 1 / (1 + e^t), t = -2 u: t and its scaling
to base 2 are off by up to 6 E |t|, the exponential and the reciprocal by 2
steps each, so the factor by (6 |t| + 8) E of itself where e^t counts; its value
moves by 1.13 of the error of z at most."""
import numpy as np
import pytest
import torch

from gpu_util import host, log, require_gpu
from oracle import rows_i8 as R

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
TD = {"bf16": torch.bfloat16, "fp32": torch.float32}
TILES = [(256, 256), (256, 192), (128, 256), (128, 192), (128, 128), (64, 64), (32, 64), (32, 32), (16, 16)]


@pytest.fixture(scope="module")
def B():
    return require_gpu()


@pytest.fixture
def tile(B):
    yield lambda m, n: B._check(B.lib().dit_debug_linear_i8_tile(m, n), "tile")
    B._check(B.lib().dit_debug_linear_i8_tile(0, 0), "tile")


class Case:
    def __init__(self, B, M, N, K, epi="none", dtype="bf16", lens=None, bias=True, pad=(0, 0, 0, 0), seed=0):
        """pad: values by which the rows of a, w, out and res are apart beyond their width."""
        self.B, self.epi = B, epi
        rng = np.random.default_rng([seed, M, N, K])
        td = TD[dtype]
        codes = lambda n, p: torch.from_numpy(rng.integers(-128, 128, (n, K + p)).astype(np.int8)).cuda()[:, :K]
        f = lambda *s: torch.from_numpy(rng.standard_normal(s)).float().cuda()
        self.a, self.w = codes(M, pad[0]), codes(N, pad[1])
        # z is about 1: sums of K products of about 74 x 74
        self.sa = f(M).abs() * (1 / 74) + 1e-4
        self.sw = f(N).abs() * (K ** -0.5 / 74) + 1e-6
        self.bias = f(N).to(td) if bias else None
        self.buf = torch.full((M + 2, N + pad[2]), 7.0, dtype=td, device="cuda")
        self.out = self.buf[1:M + 1, :N]
        self.res = f(M, N + pad[3]).to(td)[:, :N] if epi in ("residual", "gated") else None
        self.lens = lens or [M]
        self.cu = [0] + np.cumsum(self.lens).tolist()
        self.gate = f(len(self.lens), 2 * N)[:, :N] if epi == "gated" else None

    def run(self, out=None, rows=slice(None), res=None, stream=None):
        B, g = self.B, self.gate
        epi = {"none": B.EPI_NONE, "gelu": B.EPI_GELU_TANH, "residual": B.EPI_RESIDUAL, "gated": B.EPI_GATED_RESIDUAL}[self.epi]
        cu = self.cu
        if rows != slice(None):   # rows of one request alone
            r = int(np.searchsorted(self.cu, rows.start, side="right")) - 1
            cu, g = [0, rows.stop - rows.start], None if g is None else g[r:r + 1]
        out = self.out if out is None else out
        res = self.res[rows] if res is None and self.res is not None else res
        B.linear_i8(self.a[rows], self.sa[rows], self.w, self.sw, self.bias, out, epi, res, g,
                    0 if g is None else g.stride(0), None if g is None else cu, stream=stream)
        return out

    def check(self, out, what, rows=slice(None)):
        h = lambda t: None if t is None else host(t)
        zz = R.linear(h(self.a)[rows], h(self.sa)[rows], h(self.w), h(self.sw))
        b = h(self.bias) if self.bias is not None else np.zeros(self.w.shape[0])
        z = zz + b
        err = E * (2 * np.abs(zz) + np.abs(z))
        if self.epi == "gelu":
            t = np.abs(2 * np.sqrt(2 / np.pi) * (z + 0.044715 * z ** 3))
            y = R.gelu_tanh(z)
            err = 1.13 * err + np.abs(y) * E * (6 * np.minimum(t, 90) + 12)
        else:
            y = z
            if self.epi == "gated":
                g = h(self.gate)[np.repeat(np.arange(len(self.lens)), self.lens)][rows]
                y, err = z * g, err * np.abs(g)
            if self.res is not None:
                y = h(self.res)[rows] + y
                err = err + E * np.abs(y)
        half = torch.finfo(out.dtype).eps / 2
        got = host(out)
        assert np.isfinite(got).all(), what
        over = np.abs(got - y) - (err + half * (np.abs(y) + err))
        log(f"  {what}: worst error {np.abs(got - y).max():.2e}, {over.max():.2e} over what the roundings allow")
        assert (over <= 0).all(), (what, np.unravel_index(np.argmax(over), over.shape))

    def untouched(self):
        m, n = self.out.shape
        self.buf[1:m + 1, :n] = 7.0
        return bool((self.buf == 7.0).all())


SIZES = [(1, 8, 16), (1, 64, 128), (2, 24, 112), (3, 5120, 5120), (15, 72, 144), (16, 16, 64), (17, 200, 1040), (32, 384, 1536),
         (33, 136, 2064), (63, 264, 13824), (64, 1000, 272), (65, 8, 16), (77, 10240, 640), (127, 392, 128), (129, 520, 4112),
         (300, 264, 384), (513, 1288, 1552), (800, 2048, 512)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("epi", ["none", "gelu", "residual", "gated"])
@pytest.mark.parametrize("M,N,K", SIZES)
def test_linear_i8(B, M, N, K, epi, dtype):
    lens = None
    if M > 2:   # requests of one row, no rows, and the rest
        lens = [1, 0, M // 2, M - 1 - M // 2]
    c = Case(B, M, N, K, epi, dtype, lens, bias=(M + N) % 3 != 0, pad=(16 * (M % 3), 32 * (M % 2), 8 * (M % 5), 16 * (K % 3)))
    c.check(c.run(), f"{M} x {N} x {K} {epi} {dtype}")
    assert c.untouched()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("epi", ["none", "gelu", "residual", "gated"])
@pytest.mark.parametrize("M,N,K", [(300, 456, 1040), (520, 648, 112), (257, 264, 5136)])
def test_every_tile_gives_the_same_bits(B, tile, M, N, K, epi, dtype):
    c = Case(B, M, N, K, epi, dtype, [100, M - 171, 1, 70], pad=(16, 0, 8, 8))
    first = None
    for t in TILES:
        tile(*t)
        c.buf.fill_(7.0)
        got = c.run().clone()
        if first is None:
            first = got
            c.check(got, f"tile {t} {M} x {N} x {K} {epi} {dtype}")
        assert torch.equal(got, first), t
        assert c.untouched()


@pytest.mark.parametrize("t", TILES)
def test_many_tiles_per_workgroup_and_steps_of_every_count(B, tile, t):
    """More tiles than compute units (a sequence of several tiles per workgroup), K of 1 to 5 steps, not whole ones."""
    tile(*t)
    for M, N, K in ((2100, 8200, 48), (4090, 6152, 128), (1800, 9000, 144), (3000, 7000, 368), (2000, 7784, 624)):
        c = Case(B, M, N, K, "none", "bf16")
        got = c.run()
        want = (c.a.double() @ c.w.double().T).float() * c.sa[:, None]          # exact sums, then the kernel's own roundings
        want = torch.addcmul(c.bias.double(), want.double(), c.sw.double()).float().bfloat16()
        # the fused multiply-add rounds once; in 64 bits, rounded to fp32 and then to bf16, twice: the same or a neighbour
        far = (got.float() - want.float()).abs() > want.float().abs() * 2.0 ** -7
        assert not bool(far.any()), (t, M, N, K)
        assert float((got != want).double().mean()) < 1e-4
        assert c.untouched()


@pytest.mark.parametrize("epi", ["none", "gelu", "residual", "gated"])
def test_a_row_has_the_same_bits_alone(B, epi):
    lens = [40, 1, 0, 300, 59, 120]
    for dtype in TD:
        c = Case(B, 520, 1032, 2064, epi, dtype, lens)
        whole = c.run().clone()
        for r, n in enumerate(lens):
            if n:
                rows = slice(c.cu[r], c.cu[r + 1])
                assert torch.equal(c.run(torch.empty_like(whole[rows]), rows), whole[rows]), (dtype, r)


@pytest.mark.parametrize("M", [5, 300])
@pytest.mark.parametrize("epi", ["residual", "gated"])
def test_in_place_and_columns_of_one_buffer(B, M, epi):
    c = Case(B, M, 264, 640, epi, "bf16", [2, M - 2])
    want = c.run().clone()
    x = c.res.clone()
    c.run(x, res=x)
    assert torch.equal(x, want)
    both = torch.full((M, 2 * 264 + 8), 3.0, dtype=torch.bfloat16, device="cuda")   # the residual beside the output
    both[:, 264:528] = c.res
    c.run(both[:, :264], res=both[:, 264:528])
    assert torch.equal(both[:, :264], want) and torch.equal(both[:, 264:528], c.res) and bool((both[:, 528:] == 3).all())


@pytest.mark.parametrize("M", [2, 70, 300])
def test_the_largest_sums(B, M):
    """K = 131,056 products of -128 and -128, or 127 and -128: next to the ends of 32-bit integers."""
    K, N = 131056, 24
    a = torch.full((M, K), -128, dtype=torch.int8, device="cuda")
    w = torch.full((N, K), -128, dtype=torch.int8, device="cuda")
    a[1::2] = 127
    w[3] = 127
    w[4] = 0
    w[4, K - 1] = 1
    one, ones = torch.ones(M, device="cuda"), torch.ones(N, device="cuda")
    out = torch.empty(M, N, device="cuda")
    B.linear_i8(a, one, w, ones, None, out)
    want = torch.tensor(R.sums(a[:2].cpu().numpy(), w.cpu().numpy())).float().repeat(-(-M // 2), 1)[:M]
    assert torch.equal(out.cpu(), want)


@pytest.mark.parametrize("M", [7, 200])
def test_scales_that_are_not_finite_and_rows_of_zeros(B, M):
    for epi in ("none", "gelu", "residual"):
        c = Case(B, M, 136, 256, epi, "fp32")
        clean = c.run().clone()
        c.sa[3] = float("nan")
        c.sa[5] = 0.0
        got = c.run()
        assert bool(got[3].isnan().all())
        rest = [r for r in range(M) if r not in (3, 5)]
        assert torch.equal(got[rest], clean[rest])
        b = host(c.bias)
        want = R.gelu_tanh(b) if epi == "gelu" else b if epi == "none" else host(c.res[5]) + b
        assert np.allclose(host(got[5]), want, rtol=1e-5, atol=1e-6)
        c.sa[3] = 1.0
        c.sw[9] = float("nan")
        got = c.run()
        assert bool(got[:, 9].isnan().all()) and int(got.isnan().sum()) == M


def test_offsets_past_32_bits(B):
    # rows of a 1 MB apart: the last begins behind 4 GiB
    M, N, K = 4200, 72, 208
    far = torch.empty(M << 20, dtype=torch.int8, device="cuda").view(M, 1 << 20)
    c = Case(B, M, N, K)
    far[:, 4096:4096 + K] = c.a
    want = c.run().clone()
    c.a = far[:, 4096:4096 + K]
    got = c.run()
    assert torch.equal(got, want)
    c.a, c.sa, M = c.a[-40:], c.sa[-40:], 40                       # few rows, from there
    c.cu = [0, 40]
    few = torch.empty(40, N, dtype=torch.bfloat16, device="cuda")
    c.run(few)
    assert torch.equal(few, want[-40:])
    del far, c, got, want
    # an output of more than 2^32 values
    M, N, K = 530000, 8200, 16
    c = Case(B, 2, N, K)
    codes = torch.randint(-128, 128, (M, K), dtype=torch.int8, device="cuda")
    sa = torch.rand(M, device="cuda")
    out = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    B.linear_i8(codes, sa, c.w, c.sw, c.bias, out)
    for lo in (0, 261900, 523776, M - 300):
        part = torch.empty(300, N, dtype=torch.bfloat16, device="cuda")
        B.linear_i8(codes[lo:lo + 300].contiguous(), sa[lo:lo + 300].contiguous(), c.w, c.sw, c.bias, part)
        assert torch.equal(out[lo:lo + 300], part)


def test_weights_far_apart(B):
    M, K, ld = 130, 160, 1 << 22
    w = torch.empty(1100 * ld, dtype=torch.int8, device="cuda").view(1100, ld)   # rows of 4 MB, the largest stride
    c = Case(B, M, 1096, K)
    want = c.run().clone()
    w[:1096, 64:64 + K] = c.w
    c.w = w[:1096, 64:64 + K]
    assert torch.equal(c.run(), want)
    c.a, c.sa, c.cu = c.a[:9], c.sa[:9], [0, 9]
    assert torch.equal(c.run(torch.empty(9, 1096, dtype=torch.bfloat16, device="cuda")), want[:9])


@pytest.mark.parametrize("M", [3, 700])
def test_streams_graphs_and_two_calls_at_once(B, M):
    c = Case(B, M, 1304, 1040, "gated", "bf16", [1, M - 1])
    held = torch.empty(M, 1304, dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run(held)
    for k in range(4):
        c.a.copy_(torch.randint(-128, 128, c.a.shape, dtype=torch.int8, device="cuda"))
        c.sa.mul_(1.25)
        graph.replay()
        want = c.run().clone()
        torch.cuda.synchronize()
        assert torch.equal(held, want), k
    outs = [torch.empty_like(held) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(8):
        for s, o in zip(streams, outs):
            c.run(o, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want) and torch.equal(outs[1], want)


def test_empty_calls(B):
    c = Case(B, 4, 64, 128, "gated", "bf16", [1, 3])
    before = c.buf.clone()
    B.linear_i8(c.a[:0], c.sa[:0], c.w, c.sw, c.bias, c.out[:0], B.EPI_GATED_RESIDUAL, c.res[:0], c.gate, c.gate.stride(0), [0, 0, 0])
    assert torch.equal(c.buf, before)


@pytest.mark.parametrize("rows,D,F", [([64], 384, 1536), ([100, 0, 1, 411], 1024, 2816), ([3, 2], 5120, 13824)])
def test_the_mlp_of_a_block_in_8_bits(B, rows, D, F):
    """The operators as a block uses them: modulated norm, up projection with GELU, quantiser, gated down projection into
    the residual stream; weights from the quantiser.  Each stage against the 64-bit one on the stage's own inputs, and
    the whole against the MLP in 64 bits, within half a step of every code that was rounded on the way."""
    rng = np.random.default_rng(D)
    cu = [0] + np.cumsum(rows).tolist()
    n, td = cu[-1], torch.bfloat16
    f = lambda std, *s: torch.from_numpy(rng.standard_normal(s) * std).float().cuda()
    x, mod = f(1.0, n, D).to(td), f(0.3, len(rows), 6, D)
    wu, wd, bu, bd = f(D ** -0.5, F, D).to(td), f(F ** -0.5, D, F).to(td), f(0.1, F).to(td), f(0.1, D).to(td)

    def coded(t):
        c, s = torch.empty(t.shape, dtype=torch.int8, device="cuda"), torch.empty(t.shape[0], device="cuda")
        B.quantize_rows(t, c, s)
        return c, s

    cwu, cwd = coded(wu), coded(wd)
    cx, ch = (torch.empty(n, k, dtype=torch.int8, device="cuda") for k in (D, F))
    sx, sh = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    hidden, y = torch.empty(n, F, dtype=td, device="cuda"), x.clone()
    B.adaln_modulate_i8(x, mod[:, 3], mod[:, 4], mod.stride(0), cu, 1e-6, cx, sx)
    B.linear_i8(cx, sx, *cwu, bu, hidden, B.EPI_GELU_TANH)
    B.quantize_rows(hidden, ch, sh)
    B.linear_i8(ch, sh, *cwd, bd, y, B.EPI_GATED_RESIDUAL, y, mod[:, 5], mod.stride(0), cu)

    h, half = host, 2.0 ** -8
    mid = R.linear(h(cx), h(sx), h(cwu[0]), h(cwu[1]), h(bu), "gelu")
    assert (np.abs(h(hidden) - mid) <= half * np.abs(mid) + 1e-5).all()
    assert (h(ch) == R.quantize(h(hidden))[0]).all()
    end = R.linear(h(ch), h(sh), h(cwd[0]), h(cwd[1]), h(bd), "gated", h(x), h(mod[:, 5]), cu)
    assert (np.abs(h(y) - end) <= half * np.abs(end) + 1e-5).all()

    # the MLP without codes, and how far the codes' roundings may take it: a code is off by half a step (and 2^-16 of it)
    step = lambda t: R.quantum(t)[:, None] * 0.5001
    v = R.modulate(h(x), h(mod[:, 3]), h(mod[:, 4]), cu, 1e-6)
    z = v @ h(wu).T + h(bu)
    dv, dwu = step(v), step(h(wu))
    dz = dv * np.abs(h(wu)).sum(1) + np.abs(v).sum(1)[:, None] * dwu.T + dv * D * dwu.T
    u = R.gelu_tanh(z)
    du = 1.13 * dz + half * (np.abs(u) + 1.13 * dz)
    du = du + (np.abs(u) + du).max(1)[:, None] / 127 * 0.5001
    dwd = step(h(wd))
    dy = du @ np.abs(h(wd)).T + (np.abs(u) + du).sum(1)[:, None] * dwd.T
    gate = h(mod[:, 5])[np.repeat(np.arange(len(rows)), rows)]
    true = h(x) + gate * (u @ h(wd).T + h(bd))
    bound = np.abs(gate) * dy
    bound = bound + half * (np.abs(true) + bound) + 1e-5
    assert (np.abs(h(y) - true) <= bound).all()
    rel = np.linalg.norm(h(y) - true) / np.linalg.norm(true - h(x))
    log(f"  MLP {rows} {D} {F}: {rel:.4f} of its result off")


TILED = [t for t in TILES if t[0] >= 128]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("epi", ["none", "gelu", "residual", "gated"])
@pytest.mark.parametrize("M,N,K", [(2100, 8200, 48), (4090, 6152, 256), (1800, 9000, 368), (3000, 7000, 512), (2600, 8200, 624)])
def test_every_epilogue_and_type_over_several_tiles_of_a_workgroup(B, tile, M, N, K, epi, dtype):
    """Every tiled shape with more tiles than compute units and K of 1 to 5 steps: an epilogue's stores (twice as many in
    fp32), its reads of the residual and of the gates of requests that end inside a wave's rows lie between a tile's loads
    and the next one's waits.  Against the sums in 64 bits on the device, within the roundings counted above; the same bits
    for every shape and in place."""
    assert all(-(-M // m) * -(-N // n) > 256 for m, n in TILED)
    c = Case(B, M, N, K, epi, dtype, [100, 0, 1, M // 2 + 3, M - M // 2 - 104], pad=(16, 0, 8, 16), seed=7)
    S = (c.a.double() @ c.w.double().T.contiguous()) * c.sa.double()[:, None] * c.sw.double()
    z = S + c.bias.double()
    err = E * (2 * S.abs() + z.abs())
    y = z
    if epi == "gelu":
        u = (2 / np.pi) ** 0.5 * (z + 0.044715 * z ** 3)
        y = 0.5 * z * (1 + torch.tanh(u))
        # tanh near -1 leaves 2^-53 of z in 1 + tanh
        err = 1.13 * err + y.abs() * E * (6 * (2 * u).abs().clamp(max=90) + 12) + z.abs() * 2.0 ** -52
    elif epi == "gated":
        g = c.gate.double().repeat_interleave(torch.tensor(c.lens, device="cuda"), 0)
        y, err = z * g, err * g.abs()
    if c.res is not None:
        y = c.res.double() + y
        err = err + E * y.abs()
    allowed = err + torch.finfo(TD[dtype]).eps / 2 * (y.abs() + err)
    first = None
    for t in TILED:
        tile(*t)
        c.buf.fill_(7.0)
        got = c.run().clone()
        over = (got.double() - y).abs() - allowed
        assert bool((over <= 0).all()), (t, float(over.max()), divmod(int(over.argmax()), N))
        first = got if first is None else first
        assert torch.equal(got, first), t
        assert c.untouched()
        if c.res is not None:
            x = c.res.clone()
            c.run(x, res=x)
            assert torch.equal(x, first), t
