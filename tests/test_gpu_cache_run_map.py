"""The slot map at the largest size that an int holds."""
import pytest
import torch

from gpu_util import log, require_gpu

pytestmark = pytest.mark.gpu


def test_largest_slot_map():
    """2^31 - 1 entries (34 GB): the entries that are there, and zeros to the last one."""
    B = require_gpu()
    n = 2 ** 31 - 1
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("the slot map takes 34 GB")
    log("case slot map of 2^31 - 1 entries")
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")
    cache = B.KvCache.empty(4, 1, 64, 32, 2, 4)
    runs = torch.empty((n, 4), dtype=torch.int32, device="cuda")
    for part in (runs[:8], runs[2 ** 30 - 4:2 ** 30 + 4], runs[-8:]):
        part.fill_(7)
    counts = i32(0, 0, 0, 0)
    B.cache_tables(cache, None, i32(40, 3), i32(2, 0, 3), runs, counts, 43)
    torch.cuda.synchronize()
    assert counts.tolist() == [3, 3, 0, 43] and cache.lens.tolist() == [40, 3]
    assert runs[:4].tolist() == [[2, 0, 0, 32], [0, 32, 0, 8], [3, 40, 0, 3], [0, 0, 0, 0]]
    for part in (runs[4:8], runs[2 ** 30 - 4:2 ** 30 + 4], runs[-8:]):
        assert (part == 0).all()
    del runs
    torch.cuda.empty_cache()
