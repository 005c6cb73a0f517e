"""Lengths that another stream writes while the attention runs: the rows of such
a call are undefined, but it writes nothing but its own rows and workspace, it
ends, and the next call is right again."""
import numpy as np
import pytest
import torch

from gpu_util import log, require_gpu
from test_gpu_cache import TYPES, _bits, _check_attention, _fill_real, _i32, _request_pages

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,dim", TYPES)
@pytest.mark.parametrize("qlens", [[1, 3, 2, 1], [150, 1, 40, 33], [2000, 0, 700, 1]])
def test_lengths_written_during_calls(dtype, dim, qlens):
    B = require_gpu()
    log(f"case lengths written during calls {dtype} dim {dim} q {qlens}")
    rng = np.random.default_rng(1)
    most = 6000
    cache = B.KvCache.empty(4 * 94 + 1, 2, dim, 64, 4, 94)
    _fill_real(cache, rng)
    _request_pages(cache, rng, [most] * 4)   # every row of the table is whole, so any length up to 6,000 names pages
    lens = [_i32(x) for x in ([most, 3, 0, 700], [0, most, 64, 5], [1, 0, most, most], [-1, 2 ** 31 - 1, 130, 0])]
    cu = [0] + np.cumsum(qlens).tolist()
    T, w = cu[-1], 4 * dim
    q, _ = _bits(rng.standard_normal((T, w)), dtype)
    held = torch.full((T + 16, w), 3.0, dtype=dtype, device="cuda")
    o = held[8:8 + T]
    n = B.attention_cached_workspace_size(cache, cu, 4, dtype)
    space = torch.full((n + 8192,), 0xA5, dtype=torch.uint8, device="cuda")
    ws = space[4096:4096 + n] if n else None
    pools = [t.clone() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale, cache.table)]
    call = lambda s: B.attention_cached(cache, q, o, cu, 4, ws, stream=s)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for rep in range(20):
        call(streams[0])
        with torch.cuda.stream(streams[1]):
            for x in lens:
                cache.lens.copy_(x)
    torch.cuda.synchronize()
    assert (held[:8] == 3).all() and (held[8 + T:] == 3).all()
    assert (space[:4096] == 0xA5).all() and (space[4096 + n:] == 0xA5).all()
    for a, b in zip(pools, (cache.k, cache.v, cache.k_scale, cache.v_scale, cache.table)):
        assert torch.equal(a, b)
    cache.lens.copy_(lens[0])
    torch.cuda.synchronize()
    call(streams[0])
    torch.cuda.synchronize()
    _check_attention(cache, q, o, cu, 4, rows=6)
