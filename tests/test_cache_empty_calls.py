"""Calls on the cache with nothing to do -- no request grows, no request has
queries, no prompt has rows -- where an empty tensor's address is 0."""
import ctypes

import pytest
import torch

from gpu_util import log, require_gpu
from test_cache import B, BAD, P, RUNS, S, TAB, _attn, _cache, _lib, _model, _refused, _store, W

I32 = torch.int32


def test_entries_without_rows():
    """No HIP call: these run without a GPU."""
    _lib()
    c = _cache()
    assert _store(c, k=0, v=0, n_rows=0) == B.DIT_OK
    assert _store(c, k=0, v=0, n_rows=0, runs=0, n_runs=0) == B.DIT_OK
    assert _attn(c, q=0, o=0, cu=(0, 0)) == B.DIT_OK and _attn(c, q=0, o=0, cu=(0, 0, 0, 0)) == B.DIT_OK
    # the other arguments are still looked at, and rows still need their tensors
    _refused(_store(c, k=0, v=0, n_rows=0, block=2), BAD, "block 2")
    _refused(_store(c, k=0, n_rows=1), BAD, "k is NULL")
    _refused(_attn(c, q=0, o=0, cu=(0, 0), n_heads=6), BAD, "6 query heads")
    _refused(_attn(c, o=0, cu=(0, 0, 1)), BAD, "o is NULL")


def test_text_without_rows():
    L = _lib()
    m, c = _model(), _cache()
    vl = B.Varlen([0, 6, 12], [0, 0, 0], [(1, 2, 3)] * 2)
    blocks = (B.CWeights * 2)()
    for b in blocks:
        for n in B.WEIGHT_FIELDS:
            setattr(b, n, W)
    mw = B.CModelWeights(*([W] * len(B.MODEL_FIELDS)), ctypes.cast(blocks, ctypes.POINTER(B.CWeights)))
    ref = ctypes.byref
    assert L.dit_text_kv_cached_workspace_size(ref(m.c), ref(vl.c)) == 0
    text = lambda cache: L.dit_text_kv_cached(ref(m.c), ref(mw), ref(vl.c), P(0), ref(cache), P(RUNS), 4, P(0), 0, S)
    assert text(c) == B.DIT_OK
    _refused(text(_cache(k=TAB + 8)), BAD, "cache k")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_a_round_in_which_nothing_grows(dtype):
    B = require_gpu()
    log(f"case empty calls {dtype}")
    cache = B.KvCache.empty(4, 2, 64, 32, 3, 4)
    cache.lens.copy_(torch.tensor([5, 0, 32]))
    before = [t.clone() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale, cache.table, cache.lens)]
    i32 = lambda *a: torch.tensor(a, dtype=I32, device="cuda")
    runs, counts = torch.full((B.cache_run_bound(32, 3, 0), 4), 9, dtype=I32, device="cuda"), i32(9, 9, 9, 9)
    B.cache_tables(cache, cache.lens.clone(), i32(0, 0, 0), i32()[:0], runs, counts, 0)
    kv = torch.empty(7, 3 * 128, dtype=dtype, device="cuda")
    for x in (kv[0:0], torch.empty(0, 256, dtype=dtype, device="cuda")):
        B.cache_store(cache, x[:, :128], x[:, 128:256], runs)
        B.cache_store(cache, x[:, :128], x[:, 128:256], runs[:0])
        B.attention_cached(cache, x[:, :256], x[:, :256].clone(), [0, 0, 0, 0], 4)
    torch.cuda.synchronize()
    assert counts.tolist() == [0, 0, 0, 0] and (runs == 0).all()
    for a, b in zip(before, (cache.k, cache.v, cache.k_scale, cache.v_scale, cache.table, cache.lens)):
        assert torch.equal(a, b)


@pytest.mark.gpu
def test_text_of_empty_prompts():
    from test_gpu_cached_step import CachedStep
    log("case text of empty prompts")
    s = CachedStep("step_tiny_fp32")
    before = s.cache.k.clone()
    B = s.B
    vl = B.Varlen([0, 0, 0], [0, 0, 0], [(1, 1, 1)] * 2)
    txt = torch.empty(0, s.mw.block.hidden, device="cuda")
    runs = torch.zeros(4, 4, dtype=I32, device="cuda")
    B.text_kv_cached(s.cfg, s.w, vl, txt, s.cache, runs, torch.empty(0, dtype=torch.uint8, device="cuda"))
    B.text_kv_cached(s.cfg, s.w, vl, txt, s.cache, runs, None)
    torch.cuda.synchronize()
    assert torch.equal(s.cache.k, before)
