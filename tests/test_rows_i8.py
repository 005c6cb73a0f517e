"""The Linears on 8-bit integers on the CPU: every refusal of the C entries
before a launch, the binding's own checks, calls without rows, and the rule that
chooses a product's tile."""
import ctypes

import numpy as np
import pytest
import torch

B = pytest.importorskip("paper_2606_13501_amd.binding")


@pytest.fixture(scope="module")
def L():
    import os
    if not os.path.exists(B.LIB_PATH):
        pytest.skip("libditblock.so not built")
    return B.lib()


BAD, NOT = B.DIT_ERR_INVALID_ARG, B.DIT_ERR_UNSUPPORTED
S = None
# aligned addresses, far apart, never read: each call fails on the host or has no rows
X, Z, G, C, SC, O, SUM, W, WS, RES, GATE = (0x100000000 * i for i in range(1, 12))


def cu(*a):
    a = np.asarray(a, np.int32)
    cu.keep = a
    return a.ctypes.data


def quantize(L, x=X, xs=64, rows=4, width=64, c=C, cs=64, s=SC, dt=B.DIT_BF16):
    return L.dit_quantize_rows(x, xs, rows, width, c, cs, s, dt, S)


def modulate(L, x=X, shift=G, scale=W, stride=64, cus=(0, 4), n=1, width=64, eps=1e-6, c=C, s=SC, dt=B.DIT_BF16):
    return L.dit_adaln_modulate_i8(x, shift, scale, stride, cu(*cus), n, width, eps, c, s, dt, S)


def rms(L, x=X, z=Z, gain=G, rows=4, width=64, eps=1e-6, sm=SUM, out=O, c=C, s=SC, dt=B.DIT_BF16):
    return L.dit_add_rms_norm(x, z, gain, rows, width, eps, sm, out, c, s, dt, S)


def linear(L, a=X, lda=64, sa=SC, w=W, ldw=64, sw=WS, bias=G, out=O, ldo=64, M=4, N=64, K=64, epi=B.EPI_NONE, res=RES, ldr=64,
           gate=GATE, gs=64, cus=(0, 1, 4), n=2, dt=B.DIT_BF16):
    return L.dit_linear_i8(a, lda, sa, w, ldw, sw, bias, out, ldo, M, N, K, epi, res, ldr, gate, gs, cu(*cus), n, dt, S)


@pytest.mark.parametrize("call,args,status,words", [
    (quantize, dict(dt=5), BAD, b"dtype"),
    (quantize, dict(rows=-1), BAD, b"n_rows"),
    (quantize, dict(rows=1 << 31), BAD, b"n_rows"),
    (quantize, dict(width=0), BAD, b"multiple of 16"),
    (quantize, dict(width=40), BAD, b"multiple of 16"),
    (quantize, dict(width=(1 << 22) + 16, xs=1 << 23, cs=1 << 23), NOT, b"too large"),
    (quantize, dict(xs=56), BAD, b"x_row_stride"),
    (quantize, dict(xs=68), BAD, b"x_row_stride"),
    (quantize, dict(xs=66, dt=B.DIT_F32), BAD, b"x_row_stride"),
    (quantize, dict(cs=48), BAD, b"codes_row_stride"),
    (quantize, dict(cs=72), BAD, b"codes_row_stride"),
    (quantize, dict(x=None), BAD, b"x is NULL"),
    (quantize, dict(c=None), BAD, b"codes is NULL"),
    (quantize, dict(s=None), BAD, b"scales is NULL"),
    (quantize, dict(x=X + 8), BAD, b"x is not 16"),
    (quantize, dict(c=C + 8), BAD, b"codes is not 16"),
    (quantize, dict(s=SC + 2), BAD, b"scales is not 4"),
    (quantize, dict(c=X + 496), BAD, b"codes overlaps x"),
    (quantize, dict(s=X + 508), BAD, b"scales overlaps x"),
    (quantize, dict(s=C + 252), BAD, b"codes overlaps scales"),
    (modulate, dict(dt=-1), BAD, b"dtype"),
    (modulate, dict(n=0), BAD, b"n_req"),
    (modulate, dict(n=65), BAD, b"n_req"),
    (modulate, dict(cus=(0, 4, 2), n=2), BAD, b"decreases"),
    (modulate, dict(cus=(1, 4)), BAD, b"must be 0"),
    (modulate, dict(width=24), BAD, b"multiple of 16"),
    (modulate, dict(width=8208), NOT, b"too large"),
    (modulate, dict(width=4112, dt=B.DIT_F32), NOT, b"too large"),
    (modulate, dict(eps=0.0), BAD, b"eps"),
    (modulate, dict(eps=float("nan")), BAD, b"eps"),
    (modulate, dict(eps=float("inf")), BAD, b"eps"),
    (modulate, dict(stride=66), BAD, b"mod_stride"),
    (modulate, dict(stride=-4), BAD, b"mod_stride"),
    (modulate, dict(shift=None), BAD, b"shift is NULL"),
    (modulate, dict(scale=W + 4), BAD, b"scale is not 16"),
    (modulate, dict(c=X), BAD, b"codes overlaps x"),
    (modulate, dict(s=G + 4), BAD, b"scales overlaps shift"),
    (modulate, dict(c=W + 64), BAD, b"codes overlaps scale"),
    (rms, dict(dt=2), BAD, b"dtype"),
    (rms, dict(width=72), BAD, b"multiple of 16"),
    (rms, dict(width=68, c=None, s=None), BAD, b"multiple of 8"),
    (rms, dict(width=66, c=None, s=None, dt=B.DIT_F32), BAD, b"multiple of 4"),
    (rms, dict(width=8208), NOT, b"too large"),
    (rms, dict(eps=-1.0), BAD, b"eps"),
    (rms, dict(x=None), BAD, b"x is NULL"),
    (rms, dict(gain=None), BAD, b"gain is NULL"),
    (rms, dict(z=None), BAD, b"z and sum"),
    (rms, dict(sm=None), BAD, b"z and sum"),
    (rms, dict(c=None), BAD, b"codes and scales"),
    (rms, dict(s=None), BAD, b"codes and scales"),
    (rms, dict(out=None, c=None, s=None), BAD, b"neither"),
    (rms, dict(sm=O), BAD, b"sum overlaps out"),
    (rms, dict(sm=X + 16), BAD, b"sum overlaps an input"),
    (rms, dict(out=Z - 16), BAD, b"out overlaps an input"),
    (rms, dict(out=G), BAD, b"out overlaps gain"),
    (rms, dict(c=SUM), BAD, b"codes overlaps sum"),
    (rms, dict(s=Z), BAD, b"scales overlaps z"),
    (linear, dict(dt=3), BAD, b"dtype"),
    (linear, dict(M=-1), BAD, b"bad GEMM size"),
    (linear, dict(N=0), BAD, b"bad GEMM size"),
    (linear, dict(K=0), BAD, b"bad GEMM size"),
    (linear, dict(K=56), NOT, b"K % 16"),
    (linear, dict(N=60, ldo=64), NOT, b"N % 8"),
    (linear, dict(K=131072, lda=131072, ldw=131072), NOT, b"K <="),
    (linear, dict(M=(1 << 28) + 1), NOT, b"too many tiles"),
    (linear, dict(M=1 << 28, N=1 << 20, ldo=1 << 20), NOT, b"too many tiles"),
    (linear, dict(epi=4), BAD, b"epilogue"),
    (linear, dict(lda=48), BAD, b"lda"),
    (linear, dict(ldw=72), BAD, b"lda"),
    (linear, dict(lda=(1 << 22) + 16), BAD, b"lda"),
    (linear, dict(N=(1 << 24) + 8, ldo=1 << 25), NOT, b"N <="),
    (linear, dict(ldo=(1 << 24) + 8), BAD, b"ldo"),
    (linear, dict(epi=B.EPI_RESIDUAL, ldr=(1 << 24) + 8), BAD, b"ldr"),
    (linear, dict(ldo=56), BAD, b"ldo"),
    (linear, dict(ldo=68), BAD, b"ldo"),
    (linear, dict(epi=B.EPI_RESIDUAL, ldr=56), BAD, b"ldr"),
    (linear, dict(epi=B.EPI_RESIDUAL, res=None), BAD, b"res is NULL"),
    (linear, dict(epi=B.EPI_RESIDUAL, res=O + 16), BAD, b"out overlaps res"),
    (linear, dict(epi=B.EPI_RESIDUAL, res=O, ldr=72), BAD, b"out overlaps res"),
    (linear, dict(epi=B.EPI_RESIDUAL, res=O + 126 + 2, ldr=128, ldo=128 + 8), BAD, b"out overlaps res"),
    (linear, dict(epi=B.EPI_RESIDUAL, res=O + 112, ldr=128, ldo=128), BAD, b"out overlaps res"),
    (linear, dict(epi=B.EPI_GATED_RESIDUAL, gate=None), BAD, b"gate is NULL"),
    (linear, dict(epi=B.EPI_GATED_RESIDUAL, gs=62), BAD, b"gate_stride"),
    (linear, dict(epi=B.EPI_GATED_RESIDUAL, cus=(0, 1, 5)), BAD, b"cu_seqlens ends"),
    (linear, dict(epi=B.EPI_GATED_RESIDUAL, gate=O), BAD, b"out overlaps gate"),
    (linear, dict(a=None), BAD, b"a is NULL"),
    (linear, dict(w=W + 4), BAD, b"w is not 16"),
    (linear, dict(sa=None), BAD, b"a_scales is NULL"),
    (linear, dict(sw=WS + 1), BAD, b"w_scales is not 4"),
    (linear, dict(bias=G + 8), BAD, b"bias is not 16"),
    (linear, dict(out=X), BAD, b"out overlaps a"),
    (linear, dict(out=W + 16), BAD, b"out overlaps w"),
    (linear, dict(out=SC), BAD, b"out overlaps a_scales"),
    (linear, dict(out=G), BAD, b"out overlaps bias"),
])
def test_refusals(L, call, args, status, words):
    assert call(L, **args) == status
    assert words in L.dit_last_error(), L.dit_last_error()


def test_calls_without_rows_do_nothing(L):
    assert quantize(L, rows=0, x=None, c=None, s=None) == B.DIT_OK
    assert modulate(L, cus=(0, 0, 0), n=2, x=None, shift=None, scale=None, c=None, s=None) == B.DIT_OK
    assert rms(L, rows=0, x=None, z=None, gain=None, sm=None, out=None, c=None, s=None) == B.DIT_OK
    for epi in range(4):
        assert linear(L, M=0, cus=(0, 0, 0), epi=epi, a=None, sa=None, out=None, res=None) == B.DIT_OK
    # their sizes are checked all the same
    assert quantize(L, rows=0, width=8) == BAD and linear(L, M=0, cus=(0, 0, 0), K=8) == NOT


def _cpu(*shape, dt=torch.bfloat16):
    return torch.zeros(shape, dtype=dt)


def test_binding_checks():
    i8, f32 = torch.int8, torch.float32
    x, codes, scales = _cpu(4, 64), _cpu(4, 64, dt=i8), _cpu(4, dt=f32)
    with pytest.raises(ValueError, match="codes"):
        B.quantize_rows(x, _cpu(4, 64), scales)
    with pytest.raises(ValueError, match="codes"):
        B.quantize_rows(x, _cpu(4, 80, dt=i8), scales)
    with pytest.raises(ValueError, match="scales"):
        B.quantize_rows(x, codes, _cpu(5, dt=f32))
    with pytest.raises(ValueError, match="rows of 64 dense"):
        B.quantize_rows(_cpu(64, 4).T, codes, scales)
    with pytest.raises(ValueError, match="cpu"):
        B.quantize_rows(x, codes, scales)
    mod = _cpu(2, 6, 64, dt=f32)
    call = lambda x=x, sh=mod[:, 0], sc=mod[:, 1], st=384, cus=(0, 1, 4), c=codes: B.adaln_modulate_i8(x, sh, sc, st, cus, 1e-6, c, scales)
    with pytest.raises(ValueError, match="cu_seqlens ends at 5"):
        call(cus=(0, 1, 5))
    with pytest.raises(ValueError, match="shift"):
        call(st=448)                       # the second request's vector would end behind the tensor
    with pytest.raises(ValueError, match="scale"):
        call(sc=mod[:1, 1])
    with pytest.raises(ValueError, match="shift"):
        call(sh=mod[:, 0].double())
    with pytest.raises(ValueError, match="not dense"):
        call(x=_cpu(4, 128)[:, :64])
    with pytest.raises(ValueError, match="cpu"):
        call()
    norm = lambda z=None, gain=_cpu(64), **kw: B.add_rms_norm(x, z, gain, 1e-6, **kw)
    for bad in (dict(z=_cpu(4, 64, dt=f32)), dict(gain=_cpu(32)), dict(sum=_cpu(5, 64)), dict(out=_cpu(4, 64, dt=f32)),
                dict(codes=_cpu(4, 64)), dict(scales=_cpu(3, dt=f32))):
        with pytest.raises(ValueError, match="needed"):
            norm(**bad)
    a, w, out = _cpu(4, 64, dt=i8), _cpu(24, 64, dt=i8), _cpu(4, 24)
    ws, bias, gate = _cpu(24, dt=f32), _cpu(24), _cpu(2, 24, dt=f32)

    def lin(a=a, sa=scales, w=w, sw=ws, bias=bias, out=out, **kw):
        B.linear_i8(a, sa, w, sw, bias, out, **kw)

    for bad in (dict(a=_cpu(4, 64)), dict(w=_cpu(24, 48, dt=i8)), dict(out=_cpu(4, 32)), dict(sa=_cpu(5, dt=f32)),
                dict(sw=_cpu(24)), dict(bias=_cpu(24, dt=f32)), dict(res=_cpu(4, 24, dt=f32)), dict(res=_cpu(5, 24)),
                dict(gate=gate, gate_stride=32, cu_seqlens=(0, 1, 4)), dict()):
        with pytest.raises(ValueError):
            lin(**bad)


TILES = [(256, 256), (256, 192), (128, 256), (128, 192), (128, 128), (64, 64), (32, 64), (32, 32), (16, 16)]


def test_a_forced_tile_is_one_of_the_kernel_s(L):
    for bad in ((256, 128), (0, 256), (64, 16), (-1, -1)):
        assert L.dit_debug_linear_i8_tile(*bad) == BAD and b"output tile" in L.dit_last_error()
    try:
        for t in TILES:
            assert L.dit_debug_linear_i8_tile(*t) == B.DIT_OK
            assert plan(L, 300, 640, 512) == t
            assert (plan(L, 4097, 640, 512) == t) == (t[0] >= 128)      # few rows: up to 4,096
    finally:
        assert L.dit_debug_linear_i8_tile(0, 0) == B.DIT_OK


def plan(L, M, N, K, cus=256):
    m, n = ctypes.c_int(), ctypes.c_int()
    assert L.dit_debug_linear_i8_plan(M, N, K, cus, ctypes.byref(m), ctypes.byref(n)) == B.DIT_OK, L.dit_last_error()
    return m.value, n.value


def test_the_choice_of_tiles(L):
    assert plan(L, 1, 5120, 5120) == (16, 16) and plan(L, 64, 5120, 5120) == (32, 64)
    assert plan(L, 128, 5120, 13824) == (64, 64) and plan(L, 256, 15360, 5120)[0] >= 128
    assert {plan(L, M, N, K) for M in (1, 20, 100, 600, 1000, 4000, 30000) for N in (384, 2048, 5120, 15360)
            for K in (384, 5120, 13824)} >= {(256, 256), (256, 192), (128, 128), (64, 64), (32, 64), (32, 32), (16, 16)}
    assert plan(L, 75600, 15360, 5120) == (256, 256)
    m, n = ctypes.c_int(), ctypes.c_int()
    f = L.dit_debug_linear_i8_plan
    assert f(0, 64, 64, 256, ctypes.byref(m), ctypes.byref(n)) == BAD
    assert f(1, 64, 64, 0, ctypes.byref(m), ctypes.byref(n)) == BAD
    assert f(1, 60, 64, 256, ctypes.byref(m), ctypes.byref(n)) == NOT
    assert f(1, 64, 64, 256, None, ctypes.byref(n)) == BAD


@pytest.mark.parametrize("last", [2 ** 32 + 4, -2 ** 32 + 4, 2 ** 31])
@pytest.mark.parametrize("of", [list, np.array, torch.tensor])
def test_offsets_outside_32_bits_are_refused(of, last):
    """Cut to 32 bits, [0, 2^32 + 4] would be the offsets of four rows."""
    i8, f32 = torch.int8, torch.float32
    cu = of([0, last])
    mod, scales = _cpu(1, 64, dt=f32), _cpu(4, dt=f32)
    with pytest.raises(ValueError, match="32-bit"):
        B.adaln_modulate_i8(_cpu(4, 64), mod, mod, 64, cu, 1e-6, _cpu(4, 64, dt=i8), scales)
    with pytest.raises(ValueError, match="32-bit"):
        B.linear_i8(_cpu(4, 64, dt=i8), scales, _cpu(24, 64, dt=i8), _cpu(24, dt=f32), None, _cpu(4, 24), B.EPI_GATED_RESIDUAL,
                    _cpu(4, 24), _cpu(1, 24, dt=f32), 24, cu)
    with pytest.raises((ValueError, OverflowError)):
        B._i32(cu)
    for fits in ([0, 4], [0, 2 ** 31 - 1], [-2 ** 31, 0]):
        assert B._i32(of(fits)).tolist() == fits and B._offsets(of(fits)).tolist() == fits


def test_the_largest_product(L):
    """M N = 2^44 is the most; the tiles of every shape then have 32-bit indices."""
    m, n = ctypes.c_int(), ctypes.c_int()
    f = lambda M, N: L.dit_debug_linear_i8_plan(M, N, 64, 256, ctypes.byref(m), ctypes.byref(n))
    for M, N in ((1 << 28, 1 << 16), (1 << 20, 1 << 24), ((1 << 28) - 1, (1 << 16) - 8)):
        assert f(M, N) == B.DIT_OK
        for bm, bn in TILES[:5]:
            assert -(-M // bm) * -(-N // bn) <= 0x7FFFFFF8
    for M, N in ((1 << 28, (1 << 16) + 8), ((1 << 20) + 1, 1 << 24), (1 << 28, 3 << 15)):
        assert f(M, N) == NOT and b"too many tiles" in L.dit_last_error()
