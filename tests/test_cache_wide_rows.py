"""Query rows whose heads do not have 32-bit places in them (no HIP call: these
run without a GPU)."""
import ctypes

from test_cache import B, BAD, Q, UNSUP, _attn, _cache, _cu, _lib, _refused

WIDE = 1 << 33   # a row stride past either width


def test_rows_past_32_bits_are_refused():
    L = _lib()
    for dim, most in ((128, (1 << 24) - 1), (64, (1 << 25) - 1)):
        c = _cache(n_kv_heads=1, head_dim=dim)
        for n in (most + 1, 1 << 30, 2 ** 31 - 1):
            for dt in (B.DIT_BF16, B.DIT_F32):
                _refused(_attn(c, cu=(0, 1), n_heads=n, qs=WIDE, os_=WIDE, dt=dt), UNSUP, "query rows of")
                a, pa = _cu([0, 1])
                assert L.dit_attention_cached_workspace_size(ctypes.byref(c), pa, 1, n, 0, dt) == 0
        # the widest row goes on to the checks behind this one
        _refused(_attn(c, cu=(0, 1), n_heads=most, qs=WIDE, os_=WIDE, o=Q), BAD, "o overlaps q")
