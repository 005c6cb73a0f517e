"""The cache's entry points on the CPU: what they refuse, before any HIP call."""
import ctypes
import os

import numpy as np
import pytest
import torch

B = pytest.importorskip("paper_2606_13501_amd.binding")

S = ctypes.c_void_p(0)
P = lambda a: ctypes.c_void_p(a)
BAD, UNSUP, WS = B.DIT_ERR_INVALID_ARG, B.DIT_ERR_UNSUPPORTED, B.DIT_ERR_WORKSPACE
# distinct, aligned, never dereferenced device addresses, 16 GiB apart
K, V, KS, VS, TAB, LENS, RUNS, CNT, BEF, ADD, FREE, Q, O, W = (i << 34 for i in range(1, 15))


def _lib():
    if not os.path.exists(B.LIB_PATH):
        pytest.skip("libditblock.so not built")
    return B.lib()


def _cache(**kw):
    f = dict(n_blocks=2, n_pages=10, n_kv_heads=4, head_dim=128, page_tokens=64, max_pages=8, table_rows=3, k=K, v=V,
             k_scale=KS, v_scale=VS, table=TAB, lens=LENS)
    f.update(kw)
    return B.CKvCache(*(f[n] for n, _ in B.CKvCache._fields_))


def _cu(a):
    a = np.asarray(a, np.int32)
    return a, a.ctypes.data_as(ctypes.POINTER(ctypes.c_int32))


def _refused(st, want, text):
    assert st == want, (st, B.lib().dit_last_error())
    assert text in B.lib().dit_last_error().decode(), B.lib().dit_last_error()


BAD_CACHES = [
    (dict(head_dim=96), UNSUP, "head_dim"), (dict(page_tokens=16), UNSUP, "page of 16"), (dict(page_tokens=96), UNSUP, "page"),
    (dict(page_tokens=512), UNSUP, "page"), (dict(n_pages=0), BAD, "pages"), (dict(n_kv_heads=0), BAD, "heads"),
    (dict(n_blocks=0), BAD, "blocks"), (dict(n_pages=1 << 30), UNSUP, "groups"),
]
BAD_POOLS = [(dict(k=0), BAD, "cache k is NULL"), (dict(v=V + 8), BAD, "cache v is not"), (dict(k_scale=0), BAD, "k_scale"),
             (dict(v_scale=0), BAD, "v_scale")]
BAD_TABLES = [(dict(table_rows=1), BAD, "table has 1 rows"), (dict(max_pages=0), BAD, "table of 0"),
              (dict(max_pages=1 << 25), BAD, "cache table of"), (dict(max_pages=(1 << 24) + 1), BAD, "cache table of"), (dict(table=0), BAD, "cache table"),
              (dict(lens=0), BAD, "cache lens")]


def _tables(cache, n_req=2, before=BEF, added=ADD, per=0, n_rows=100, free=FREE, n_free=4, runs=RUNS, n_runs=5, counts=CNT):
    return B.lib().dit_cache_tables(ctypes.byref(cache) if cache else None, n_req, P(before), P(added), per, n_rows, P(free),
                                    n_free, P(runs), n_runs, P(counts), S)


def test_tables_refusals():
    _lib()
    _refused(_tables(None), BAD, "cache is NULL")
    for kw, st, text in BAD_CACHES + BAD_TABLES:
        _refused(_tables(_cache(**kw)), st, text)
    c = _cache()
    for kw, text in [(dict(n_req=0), "n_req"), (dict(n_req=65), "n_req"), (dict(n_req=4), "3 rows"), (dict(added=0), "added"),
                     (dict(before=BEF + 2), "lens_before"), (dict(free=FREE + 1), "free_pages"), (dict(runs=RUNS + 8), "runs"), (dict(free=0), "free_pages"), (dict(n_free=-1), "n_free"),
                     (dict(runs=0), "runs"), (dict(counts=0), "counts"), (dict(n_rows=-1), "n_rows"),
                     (dict(n_rows=1 << 31), "n_rows"), (dict(per=-1), "rows_per_req"), (dict(per=49), "padded"),
                     (dict(n_runs=4), "5 needed"), (dict(n_runs=-1), "needed")]:
        _refused(_tables(c, **kw), BAD, text)
    # what is written must not meet anything else that is read or written
    for kw, text in [(dict(before=LENS), "cache lens overlaps lens_before"), (dict(added=LENS), "cache lens overlaps added"),
                     (dict(free=TAB + 32), "cache table overlaps free_pages"), (dict(runs=TAB), "cache table overlaps runs"),
                     (dict(counts=RUNS + 64), "runs overlaps counts"), (dict(added=RUNS + 16), "runs overlaps added"),
                     (dict(counts=BEF), "counts overlaps lens_before")]:
        _refused(_tables(c, **kw), BAD, text)


def test_run_bound():
    L = _lib()
    f = L.dit_cache_run_bound
    assert f(64, 2, 100) == 5 and f(32, 1, 0) == 2 and f(32, 64, 4096) == 256
    assert f(0, 1, 1) == f(32, 0, 1) == f(32, 65, 1) == f(32, 1, -1) == 0
    # enough for every split of the rows over requests that start anywhere in a page
    for page in (32, 64):
        for before in range(page):
            for a, b in ((1, page - 1), (2, 2 * page), (page + 1, page + 2), (page, 0)):
                touched = sum(-(-(s + n) // page) - s // page for s, n in ((before, a), (page - 1, b)) if n)
                assert touched <= f(page, 2, a + b)


def _store(cache, block=0, k=Q, v=O, ks=512, vs=512, n_rows=100, runs=RUNS, n_runs=5, dt=B.DIT_BF16):
    return B.lib().dit_cache_store(ctypes.byref(cache) if cache else None, block, P(k), P(v), ks, vs, n_rows, P(runs), n_runs,
                                   dt, S)


def test_store_refusals():
    _lib()
    _refused(_store(None), BAD, "cache is NULL")
    for kw, st, text in BAD_CACHES + BAD_POOLS:
        _refused(_store(_cache(**kw)), st, text)
    c = _cache()
    for kw, st, text in [(dict(dt=7), BAD, "dtype"), (dict(block=2), BAD, "block 2"), (dict(block=-1), BAD, "block -1"),
                         (dict(k=0), BAD, "k is NULL"), (dict(v=O + 8), BAD, "v is not"), (dict(ks=504), BAD, "stride"),
                         (dict(vs=516), BAD, "stride"), (dict(vs=518, dt=B.DIT_F32), BAD, "stride"), (dict(n_rows=-1), BAD, "n_rows"),
                         (dict(n_runs=-1), BAD, "slot map"), (dict(runs=0), BAD, "runs"), (dict(n_runs=1 << 29), UNSUP, "slot map")]:
        _refused(_store(c, **kw), st, text)
    for kw, text in [(dict(k=K + 64), "cache k overlaps k"), (dict(v=VS), "v_scale overlaps v"), (dict(runs=V), "cache v overlaps runs"),
                     (dict(k=K - 512), "cache k overlaps k")]:
        _refused(_store(c, **kw), BAD, text)
    _refused(_store(_cache(v=K + 64)), BAD, "cache k overlaps cache v")
    assert _store(c, n_runs=0) == B.DIT_OK and _store(c, n_runs=0, runs=0, n_rows=0) == B.DIT_OK   # nothing to do


def _attn(cache, block=0, q=Q, o=O, qs=1024, os_=1024, cu=(0, 5, 9), n_heads=8, max_len=0, scale=0.0, dt=B.DIT_BF16, ws=0, n=0):
    a, pa = _cu(cu)
    return B.lib().dit_attention_cached(ctypes.byref(cache) if cache else None, block, P(q), P(o), qs, os_, pa, len(cu) - 1,
                                        n_heads, max_len, scale, dt, P(ws), n, S)


def test_attention_refusals():
    L = _lib()
    _refused(_attn(None), BAD, "cache is NULL")
    for kw, st, text in BAD_CACHES + BAD_POOLS + BAD_TABLES:
        _refused(_attn(_cache(**kw)), st, text)
    c = _cache()
    for kw, st, text in [(dict(dt=7), BAD, "dtype"), (dict(block=2), BAD, "block 2"), (dict(q=0), BAD, "q is NULL"),
                         (dict(o=O + 4), BAD, "o is not"), (dict(qs=1016), BAD, "stride"), (dict(os_=1028), BAD, "stride"),
                         (dict(cu=(1, 5)), BAD, "must be 0"), (dict(cu=(0, 5, 4)), BAD, "decreases"), (dict(cu=(0, 1, 2, 3, 4)), BAD, "3 rows"),
                         (dict(n_heads=6), BAD, "6 query heads"), (dict(n_heads=0), BAD, "0 query heads"), (dict(max_len=-1), BAD, "max_len"),
                         (dict(scale=float("inf")), BAD, "softmax_scale"), (dict(scale=float("nan")), BAD, "softmax_scale"),
                         (dict(cu=(0, 1 << 29), o=O << 4), UNSUP, "work items")]:
        _refused(_attn(c, **kw), st, text)
    for kw, text in [(dict(o=Q + 1024), "o overlaps q"), (dict(o=K), "o overlaps cache k"), (dict(o=VS), "o overlaps cache v_scale"),
                     (dict(o=TAB), "o overlaps cache table"), (dict(o=LENS), "o overlaps cache lens")]:
        _refused(_attn(c, **kw), BAD, text)
    # single queries over a long table are divided: a workspace is needed
    long = _cache(max_pages=4000)
    a, pa = _cu([0, 1, 2])
    need = L.dit_attention_cached_workspace_size(ctypes.byref(long), pa, 2, 8, 0, B.DIT_BF16)
    assert need > 0
    _refused(_attn(long, cu=(0, 1, 2)), WS, "NULL")
    _refused(_attn(long, cu=(0, 1, 2), ws=W + 16, n=need), WS, "aligned")
    _refused(_attn(long, cu=(0, 1, 2), ws=W, n=need - 1), WS, "needed")
    _refused(_attn(long, cu=(0, 1, 2), ws=O, n=need), BAD, "o overlaps the workspace")
    _refused(_attn(long, cu=(0, 1, 2), ws=Q, n=need), BAD, "the workspace overlaps q")
    f = lambda cache, cu, n, h, m, dt: L.dit_attention_cached_workspace_size(ctypes.byref(cache), cu, n, h, m, dt)
    assert f(long, pa, 2, 8, 512, B.DIT_BF16) == 0      # few tokens at most: not divided
    assert f(long, pa, 2, 7, 0, B.DIT_BF16) == f(long, pa, 4, 8, 0, B.DIT_BF16) == f(long, pa, 2, 8, 0, 7) == 0


def _model(dtype=torch.bfloat16, heads=4):
    return B.ModelConfig(B.BlockConfig(128 * heads, heads, 128, 256, 64, (44, 42, 42), dtype), 2, 16, (1, 2, 2))


def test_model_entry_refusals():
    L = _lib()
    m, c = _model(), _cache()
    vl = B.Varlen([0, 6], [0, 7], [(1, 2, 3)])
    blocks = (B.CWeights * 2)()
    for b in blocks:
        for n in B.WEIGHT_FIELDS:
            setattr(b, n, W)
    mw = B.CModelWeights(*([W] * len(B.MODEL_FIELDS)), ctypes.cast(blocks, ctypes.POINTER(B.CWeights)))
    ref = ctypes.byref
    need = L.dit_text_kv_cached_workspace_size(ref(m.c), ref(vl.c))
    assert need == 7 * 2 * 512 * 2
    text = lambda cache=c, txt=Q, runs=RUNS, n=4, ws=O, nb=need: L.dit_text_kv_cached(
        ref(m.c), ref(mw), ref(vl.c), P(txt), ref(cache), P(runs), n, P(ws), nb, S)
    _refused(text(cache=_cache(n_kv_heads=2)), BAD, "cache of 2 heads")
    _refused(text(cache=_cache(head_dim=64)), BAD, "heads of 64")
    _refused(text(cache=_cache(n_blocks=3)), BAD, "cache of 3 blocks")
    _refused(text(cache=_cache(k=0)), BAD, "cache k")
    _refused(text(txt=0), BAD, "txt")
    _refused(text(runs=0), BAD, "runs")
    _refused(text(n=-1), BAD, "slot map")
    _refused(text(ws=0), WS, "NULL")
    _refused(text(nb=need - 1), WS, "needed")
    no_txt = B.Varlen([0, 6], None, [(1, 2, 3)])
    need = L.dit_denoise_cached_workspace_size(ref(m.c), ref(no_txt.c), ref(c))
    assert need >= L.dit_denoise_workspace_size(ref(m.c), ref(vl.c)) > 0
    step = lambda cache=c, lat=Q, out=O, ws=FREE, nb=need: L.dit_denoise_step_cached(
        ref(m.c), ref(mw), ref(no_txt.c), P(lat), P(ADD), P(BEF), ref(cache) if cache else None, P(out), P(ws), nb, S)
    _refused(step(cache=_cache(n_kv_heads=8)), BAD, "cache of 8 heads")
    _refused(step(cache=_cache(n_blocks=1)), BAD, "cache of 1 blocks")
    _refused(step(cache=_cache(table_rows=0)), BAD, "0 rows")
    _refused(step(cache=None), BAD, "cache is NULL")
    _refused(step(lat=0), BAD, "latent")
    _refused(step(out=0), BAD, "latent_out")
    _refused(step(ws=0), WS, "NULL")
    _refused(step(nb=need - 1), WS, "needed")
    assert L.dit_denoise_cached_workspace_size(ref(m.c), ref(no_txt.c), ref(_cache(head_dim=64))) == 0


def test_binding_checks_layouts():
    _lib()
    c = B.KvCache.empty(3, 2, 64, 64, 4, 5, device="cpu")
    assert (c.c.n_blocks, c.c.n_pages, c.c.n_kv_heads, c.c.head_dim, c.c.page_tokens, c.c.max_pages, c.c.table_rows) == (
        1, 3, 2, 64, 64, 5, 4)
    parts = [c.k, c.v, c.k_scale, c.v_scale, c.table, c.lens]
    for i, t in [(1, c.v[:, :2]), (0, c.k.to(torch.int8)), (2, c.k_scale[..., :1]), (3, c.v_scale.float()), (4, c.table.long()),
                 (5, c.lens[:3]), (1, c.v.transpose(-1, -2)), (4, c.table.T), (4, c.lens), (0, c.k[0, 0, 0, 0])]:
        with pytest.raises(ValueError):
            B.KvCache(*(t if j == i else x for j, x in enumerate(parts)))
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    with pytest.raises(ValueError):
        B.cache_tables(c, i32(3), i32(2), i32(4), i32(9, 4), i32(4), 10)
    with pytest.raises(ValueError):
        B.cache_tables(c, None, i32(2), i32(4).long(), i32(9, 4), i32(4), 10)
    with pytest.raises(ValueError):
        B.cache_tables(c, None, i32(2), i32(4), i32(9, 3), i32(4), 10)
    kv = torch.zeros(6, 128)
    for k, v in [(kv[:, :64], kv), (kv, kv.bfloat16()), (kv[:5], kv), (kv.T, kv.T)]:
        with pytest.raises(ValueError):
            B.cache_store(c, k, v, i32(4, 4))
    with pytest.raises(ValueError):
        B.attention_cached(c, kv, kv.clone(), [0, 7], 2)
    with pytest.raises(ValueError):
        B.attention_cached(c, kv, kv[:5].clone(), [0, 6], 2)
    with pytest.raises(ValueError):
        B.attention_cached(c, kv, kv.bfloat16(), [0, 6], 2)


def test_binding_checks_places():
    """A cache in host memory is made but not used; its tensors lie in one place."""
    _lib()
    c = B.KvCache.empty(3, 2, 64, 64, 4, 5, device="cpu")
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    kv = torch.zeros(6, 128)
    for call in (lambda: B.cache_tables(c, i32(2), i32(2), i32(4), i32(9, 4), i32(4), 10),
                 lambda: B.cache_store(c, kv, kv, i32(4, 4)),
                 lambda: B.attention_cached(c, kv, kv.clone(), [0, 6], 2)):
        with pytest.raises(ValueError, match="not on a GPU"):
            call()
    with pytest.raises(ValueError, match="meta"):
        B.KvCache(c.k, c.v, c.k_scale, c.v_scale, c.table.to("meta"), c.lens)
