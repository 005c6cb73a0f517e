"""The denoising step on a paged 8-bit text cache: pages from dit_cache_tables,
text keys and values by dit_text_kv_cached, dit_denoise_step_cached.

A cached value is a code times a power of two, exact in bf16 and fp32, so
dit_denoise_step on the cache's own values as a packed cache computes the same
step; the two differ by the order of sums and roundings inside the
cross-attention (the framework's tolerances for a step)."""
import dataclasses

import numpy as np
import pytest
import torch

import synth
from gpu_util import check, host, log, require_gpu
from oracle import cache as C
from test_gpu_cache import _check_attention
from test_gpu_step import DeviceStep

pytestmark = pytest.mark.gpu
STEPS = ["step_tiny_fp32", "step_small_bf16"]


def _i32(a):
    return torch.tensor(a, dtype=torch.int32, device="cuda")


class CachedStep(DeviceStep):
    def __init__(self, name, page=32, rows=6, n_pages=40, width=8):
        super().__init__(synth.get_model_workload(name) if isinstance(name, str) else name)
        B, wl = self.B, self.mw.block
        self.page = page
        self.cache = B.KvCache.empty(n_pages, wl.n_heads, wl.head_dim, page, rows, width, n_blocks=self.n_blocks)
        for t in (self.cache.k, self.cache.v):
            t.fill_(0x7F)   # NaN wherever nothing is stored
        self.no_txt = B.Varlen(wl.cu_seqlens(), None, list(wl.grids))
        self.ws_step = torch.empty(B.denoise_cached_workspace_size(self.cfg, self.no_txt, self.cache), dtype=torch.uint8,
                                   device="cuda")

    def admit(self, txt, lens, free):
        """Places for packed prompts, their keys and values, the pages taken."""
        B, n = self.B, len(lens)
        runs = torch.empty((B.cache_run_bound(self.page, n, sum(lens)), 4), dtype=torch.int32, device="cuda")
        counts = _i32([0] * 4)
        B.cache_tables(self.cache, None, _i32(lens), _i32(free), runs, counts, sum(lens))
        vl = B.Varlen([0] * (n + 1), [0] + np.cumsum(lens).tolist(), [(1, 1, 1)] * n)
        ws = torch.empty(B.text_kv_cached_workspace_size(self.cfg, vl), dtype=torch.uint8, device="cuda")
        B.text_kv_cached(self.cfg, self.w, vl, txt, self.cache, runs, ws)
        kv = torch.empty(B.text_kv_elems(self.cfg, vl), dtype=self.kv.dtype, device="cuda")
        B.text_kv(self.cfg, self.w, vl, txt, kv)
        torch.cuda.synchronize()
        assert counts.tolist()[2:] == [0, sum(lens)]
        return counts.tolist()[0], kv.view(self.n_blocks, sum(lens), -1), runs

    def values(self, lens):
        """The cached values as a packed text cache [n_blocks, rows, 2 D]."""
        c, wl = self.cache, self.mw.block
        out = torch.empty(self.n_blocks, sum(lens), 2 * wl.hidden, dtype=self.kv.dtype)
        table = c.table.cpu().numpy()
        for b in range(self.n_blocks):
            parts = [t[b].cpu().numpy() for t in (c.k, c.v, c.k_scale, c.v_scale)]
            at = 0
            for r, n in enumerate(lens):
                for h in range(wl.n_heads):
                    K, V, there = C.gather(*parts, table[r], n, h)
                    assert there.all()
                    d = wl.head_dim
                    out[b, at:at + n, h * d:(h + 1) * d] = torch.from_numpy(K)
                    out[b, at:at + n, wl.hidden + h * d:wl.hidden + (h + 1) * d] = torch.from_numpy(V)
                at += n
        return out.cuda()

    def cached(self, out=None, stream=None):
        out = torch.empty_like(self.dm["latent"]) if out is None else out
        self.B.denoise_step_cached(self.cfg, self.w, self.no_txt, self.dm["latent"], self.dm["t"], self.dm["dt"], self.cache,
                                   out, self.ws_step, stream)
        return out

    def packed(self, kv, lens):
        """dit_denoise_step on a packed text cache of these prompt lengths."""
        B, wl = self.B, self.mw.block
        vl = B.Varlen(wl.cu_seqlens(), [0] + np.cumsum(lens).tolist(), list(wl.grids))
        ws = torch.empty(B.denoise_workspace_size(self.cfg, vl), dtype=torch.uint8, device="cuda")
        out = torch.empty_like(self.dm["latent"])
        B.denoise_step(self.cfg, self.w, vl, self.dm["latent"], self.dm["t"], self.dm["dt"], kv.contiguous(), out, ws)
        return out

    def agree(self, lens, what):
        g, r = host(self.cached()), host(self.packed(self.values(lens), lens))
        lat = host(self.dm["latent"])
        check(g, r, self.mw.block.dtype, f"{what} latent_out")
        check(g - lat, r - lat, self.mw.block.dtype, f"{what} update")


def _prompts(s, lens, seed):
    return torch.randn(sum(lens), s.mw.block.hidden, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).to(
        s.kv.dtype)


@pytest.mark.parametrize("name", STEPS)
@pytest.mark.parametrize("page", [32, 64])
def test_text_into_the_cache(name, page):
    """Every block's cached values are the packed text cache's, rounded to e4m3
    at their page's scale."""
    log(f"case text cache {name} page {page}")
    s = CachedStep(name, page)
    lens = [77, 5]
    _, kv, _ = s.admit(_prompts(s, lens, 1), lens, [7, 3, 30, 21, 5, 6])
    got = host(s.values(lens))
    want = host(kv)
    d, H = s.mw.block.head_dim, s.mw.block.n_heads
    at = 0
    for n in lens:
        for t in range(0, n, page):
            rows = slice(at + t, at + min(n, t + page))
            for b in range(s.n_blocks):
                for h in range(2 * H):
                    x = want[b, rows, h * d:(h + 1) * d]
                    scale = 2.0 ** (C.scale_byte(x) - 127)
                    assert np.array_equal(got[b, rows, h * d:(h + 1) * d], C.VALUES[C.codes(x / scale)] * scale)
        at += n


@pytest.mark.parametrize("name", STEPS)
def test_cached_step_vs_packed_step(name):
    log(f"case cached step {name}")
    s = CachedStep(name)
    lens = [77, 40]
    s.admit(_prompts(s, lens, 2), lens, [9, 2, 31, 4, 17, 6])
    s.agree(lens, name)
    # the cache stands for the oracle's text to within e4m3's rounding; the bf16 bar holds for the step's latent
    txt = s.dm["txt"]
    cut = s.mw.block.cu_txt()
    lens = [b - a for a, b in zip(cut, cut[1:])]
    s.admit(txt, lens, [20, 21, 22, 23, 24, 25, 26])
    g, r = host(s.cached()), s.oracle()
    assert np.dot(g.ravel(), r.ravel()) / np.linalg.norm(g) / np.linalg.norm(r) >= 0.9999


@pytest.mark.parametrize("name", STEPS)
def test_prompts_of_length_zero_and_one(name):
    log(f"case cached step {name}, empty prompts")
    s = CachedStep(name)
    lens = [1, 0]
    s.admit(_prompts(s, lens, 3), lens, [9])
    out = s.cached()
    assert torch.isfinite(out).all()
    s.agree(lens, f"{name} {lens}")


@pytest.mark.parametrize("grids", [[(3, 4, 6), (1, 6, 10)], [(1, 4, 6), (1, 5, 6)]])
@pytest.mark.parametrize("lens,width", [([77, 40], 4), ([2500, 700], 128)])
def test_long_texts_and_small_latents(grids, lens, width):
    """Requests of more and of fewer than 32 tokens, on texts whose tokens one
    workgroup takes and on texts divided among workgroups."""
    log(f"case cached step, latents {grids}, texts {lens}")
    mw = synth.get_model_workload("step_small_bf16")
    rows = tuple(f * h * w for f, h, w in grids)
    mw = dataclasses.replace(mw, block=dataclasses.replace(mw.block, grids=tuple(grids), rows=rows))
    s = CachedStep(mw, n_pages=120, width=width)
    assert (s.B.attention_cached_workspace_size(s.cache, [0, *np.cumsum(rows)], mw.block.n_heads, torch.bfloat16) > 0) == (width > 4)
    free = np.random.default_rng(5).permutation(120).tolist()
    s.admit(_prompts(s, lens, 6), lens, free)
    s.agree(lens, f"{grids} {lens}")


@pytest.mark.parametrize("name", STEPS)
def test_requests_come_and_go(name):
    """Pages that one batch gives back serve the next one, and a captured step
    serves both: it reads the table and lengths as they are at the replay."""
    log(f"case cached step {name}, captured, other prompts")
    s = CachedStep(name, n_pages=6)
    s.admit(_prompts(s, [33, 64], 4), [33, 64], [0, 1, 2, 3])
    first = s.cached()
    torch.cuda.synchronize()
    out = torch.empty_like(first)
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        s.cached(out, stream)
    for rep, (lens, free) in enumerate([([33, 64], [3, 2, 1, 0]), ([90, 10], [5, 1, 4, 0]), ([2, 31], [2, 3]), ([33, 64], [1, 5, 0, 4])]):
        s.admit(_prompts(s, lens, 4 if lens == [33, 64] else rep), lens, free)
        out.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, s.cached()), rep
        if lens == [33, 64]:
            assert torch.equal(out, first), "the same prompts on other pages"
        else:
            assert not torch.equal(out, first)
            s.agree(lens, f"{name} {lens}")


def test_tables_store_attention_together():
    """A video's history grows frame by frame: lengths from the last call, new
    pages and places, the frame's keys and values, attention of the next frame
    to all of them; the codes, lengths and outputs of the oracle's own run."""
    B = require_gpu()
    log("case history of frames")
    rng = np.random.default_rng(9)
    P, H, d, n = 64, 2, 128, 3
    cache = B.KvCache.empty(30, H, d, P, n, 10)
    free = rng.permutation(30).astype(np.int32)
    lens = [_i32([0] * n), _i32([0] * n)]
    table, at = cache.table.cpu().numpy(), 0
    have = [0] * n
    for frame in range(4):
        add = [rng.integers(0, 150) if frame else 40 + r for r in range(n)]
        rows = int(sum(add))
        k, v = (torch.from_numpy(rng.standard_normal((rows, H * d)).astype(np.float32)).bfloat16().cuda() for _ in range(2))
        runs = torch.empty((B.cache_run_bound(P, n, rows), 4), dtype=torch.int32, device="cuda")
        counts = _i32([0] * 4)
        before = cache.lens.clone()
        B.cache_tables(cache, before, _i32([int(a) for a in add]), _i32(free[at:].tolist()), runs, counts, rows)
        held = [t[0].cpu().numpy() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale)]
        B.cache_store(cache, k, v, runs)
        table, have, want_runs, cnt = C.tables(P, table, have, add, free[at:], rows)
        assert counts.tolist() == cnt and cache.lens.tolist() == [int(x) for x in have]
        assert np.array_equal(cache.table.cpu().numpy(), table)
        at += cnt[0]
        for p, row, off, m in want_runs:
            for i, (x, place) in enumerate(((k, C.k_place), (v, C.v_place))):
                x = x.double().cpu().numpy()
                for h in range(H):
                    held[i][p, h], held[2 + i][p, h] = C.store(held[i][p, h], held[2 + i][p, h], x[row:row + m, h * d:(h + 1) * d], off,
                                                           place)
        for t, w in zip((cache.k, cache.v, cache.k_scale, cache.v_scale), held):
            got = t[0].cpu().numpy()
            same = np.array_equal(got, w) if w.ndim == 2 else np.array_equal(C.VALUES[got], C.VALUES[w], equal_nan=True)
            assert same, frame
        q = torch.from_numpy(rng.standard_normal((3 * 20, H * d)).astype(np.float32)).bfloat16().cuda()
        cu = [0, 20, 40, 60]
        o = torch.empty_like(q)
        B.attention_cached(cache, q, o, cu, H)
        _check_attention(cache, q, o, cu, H)
