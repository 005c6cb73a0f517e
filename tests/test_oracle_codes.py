"""The cache oracle's codes against torch's own e4m3."""
import numpy as np
import torch

from oracle import cache as C

F8 = torch.float8_e4m3fn


def test_code_table_is_torchs():
    want = torch.arange(256, dtype=torch.uint8).view(F8).double().numpy()
    assert np.array_equal(C.VALUES, want, equal_nan=True)
    assert np.array_equal(np.signbit(C.VALUES[[0, 128]]), [False, True])


def test_rounding_is_torchs():
    """Every code, every middle, their fp32 neighbours, every bf16 value up to 448
    and random fp32 numbers of every octave."""
    pos = C.VALUES[:127].astype(np.float32)
    mid = (pos[1:] + pos[:-1]) / 2
    near = np.concatenate([pos, mid, np.nextafter(mid, np.float32(0)), np.nextafter(mid, np.float32(1e9))])
    bf16 = torch.arange(1 << 15, dtype=torch.int16).view(torch.bfloat16).float().numpy()
    rng = np.random.default_rng(1)
    octaves = (rng.random((40, 2000)) + 1).astype(np.float32) * np.exp2(np.arange(-31, 9, dtype=np.float32))[:, None]
    x = np.concatenate([near, bf16, octaves.ravel()])
    x = x[np.isfinite(x) & (x <= 448)]
    x = np.concatenate([x, -x])
    want = torch.from_numpy(x).to(F8).view(torch.uint8).numpy()
    assert np.array_equal(C.codes(x), want)
