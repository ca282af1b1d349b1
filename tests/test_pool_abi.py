"""Calls of the pool of cache blocks, of the attention over shared prefixes and of sampling that are refused before anything reaches a GPU, and the arithmetic that their
kernels decide by, compiled for the host."""
import ctypes as C
import os
import subprocess

import pytest
import torch

from paper_2205_10350_b200 import binding, build
from tests.test_cache_abi import ATTEND, BAD_CACHE, NVCC, P, _cache, _OnDevice, _refused

HUGE = 1 << 40


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load()


def _pool(**kw):
    f = dict(table=P, refs=P, rows=6, table_stride=4, n_blocks=8, block=32)
    f.update(kw)
    return C.byref(binding.KvPoolStruct(*(f[n] for n, _ in binding.KvPoolStruct._fields_)))


def _caches(*kw):
    caches = [_cache(**{"k_codes": P + 4096 * i, "v_codes": P + 4096 * i + 2048, **k}) for i, k in enumerate(kw)]
    return (binding.KvCacheStruct * len(caches))(*caches)


SHARED = {**{k: v for k, v in ATTEND.items() if k in ("q", "dtype", "stride", "heads", "off", "len", "B", "M", "max_new", "max_keys")}, "group": P, "shared": P, "G": 1, "max_shared": 90,
          "causal": 1, "scale": 0.125, "out": P, "scratch": P, "nbytes": HUGE}
SAMPLE = dict(scores=P, stride=1000, dtype=0, vocab=1000, M=5, t=P, k=P, p=P, min_p=P, r=P, tokens=P, logp=P, out=HUGE, out_stride=1000)
BAD_POOL = [dict(table=None), dict(refs=None), dict(rows=0), dict(rows=8193), dict(rows=-1), dict(table_stride=0), dict(n_blocks=0), dict(block=0), dict(block=24),
            dict(block=256), dict(table_stride=1 << 27), dict(rows=8192, table_stride=1 << 19), dict(rows=2)]


@pytest.mark.parametrize("bad", BAD_POOL)
def test_pools_that_cannot_be(lib, bad):
    pool, B = _pool(**bad), 3
    _refused(lib, lib.ad_cache_fork(pool, P, P, B, None, None))
    _refused(lib, lib.ad_cache_reserve(pool, None, 0, P, P, B, P, HUGE, None, None))
    assert lib.ad_cache_reserve_scratch_bytes(pool, B) == 0
    if bad != dict(rows=2):
        _refused(lib, lib.ad_cache_compact(pool, None, 0, P, P, HUGE, None))
        assert lib.ad_cache_compact_scratch_bytes(pool) == 0


def test_pool_refusals(lib):
    pool, caches = _pool(), _caches({}, {})
    for args in ((None, P, 3), (P, None, 3), (P, P, 0), (P, P, -1), (P, P, 7)):
        _refused(lib, lib.ad_cache_fork(pool, *args, None, None))
        _refused(lib, lib.ad_cache_reserve(pool, caches, 2, *args, P, HUGE, None, None))
    _refused(lib, lib.ad_cache_fork(None, P, P, 3, None, None))
    _refused(lib, lib.ad_cache_compact(pool, caches, 2, None, P, HUGE, None))
    need, needed = lib.ad_cache_reserve_scratch_bytes(pool, 3), lib.ad_cache_compact_scratch_bytes(pool)
    assert need > 0 and needed > 0
    for scratch, n, m, want in ((None, need, needed, binding.AD_ERR_ARG), (P + 128, need, needed, binding.AD_ERR_ARG), (P, need - 1, needed - 1, binding.AD_ERR_CAPACITY)):
        _refused(lib, lib.ad_cache_reserve(pool, caches, 2, P, P, 3, scratch, n, None, None), want)
        _refused(lib, lib.ad_cache_compact(pool, caches, 2, P, scratch, m, None), want)


@pytest.mark.parametrize("bad", [b for b in BAD_CACHE if "table" not in b] + [dict(table=None), dict(table=P + 4), dict(table_stride=5), dict(n_blocks=9), dict(block=64), dict(k_codes=P), dict(v_codes=P + 2048)])
def test_caches_that_are_not_the_pools(lib, bad):
    """The second of two caches cannot be, has other blocks or another table than the pool, or is the first one again."""
    pool, caches = _pool(), _caches({}, bad)
    _refused(lib, lib.ad_cache_reserve(pool, caches, 2, P, P, 3, P, HUGE, None, None))
    _refused(lib, lib.ad_cache_compact(pool, caches, 2, P, P, HUGE, None))
    for n in (-1, 65):
        _refused(lib, lib.ad_cache_reserve(pool, caches, n, P, P, 3, P, HUGE, None, None))
    _refused(lib, lib.ad_cache_compact(pool, None, 1, P, P, HUGE, None))


@pytest.mark.parametrize("bad", [dict(q=None), dict(q=P + 2), dict(out=None), dict(out=P + 4), dict(dtype=7), dict(stride=255), dict(stride=260), dict(heads=3), dict(heads=0), dict(off=None),
                                 dict(len=None), dict(B=0), dict(B=8193, G=1), dict(M=-5), dict(M=1 << 29), dict(max_new=0), dict(max_keys=-1), dict(scale=0.0), dict(scale=float("nan")),
                                 dict(group=None), dict(shared=None), dict(G=0), dict(G=3), dict(max_shared=-1), dict(scratch=P + 128, max_shared=1 << 30, max_keys=1 << 30)])
def test_shared_attention_refusals(lib, bad):
    _refused(lib, lib.ad_cache_attention_shared(C.byref(_cache(table_stride=1 << 20)), *{**SHARED, **bad}.values(), None, None))


@pytest.mark.parametrize("bad", BAD_CACHE)
def test_shared_attention_over_caches_that_cannot_be(lib, bad):
    _refused(lib, lib.ad_cache_attention_shared(C.byref(_cache(**bad)), *SHARED.values(), None, None))


def test_shared_attention_scratch(lib):
    """What is asked for is enough, whichever way the positions are read, and a byte less is refused."""
    c = C.byref(_cache(table_stride=1 << 20))
    sizes = lambda n: (c, 1, 4, 2, 5, 3, n, 1, n)
    short, long = lib.ad_cache_attention_shared_scratch_bytes(*sizes(100)), lib.ad_cache_attention_shared_scratch_bytes(*sizes(1 << 25))
    assert short == lib.ad_cache_attention_scratch_bytes(c, 1, 4, 2, 3, 100) and long > short
    a = {**SHARED, "max_keys": 1 << 25, "max_shared": 1 << 25}
    _refused(lib, lib.ad_cache_attention_shared(c, *{**a, "nbytes": long - 1}.values(), None, None), binding.AD_ERR_CAPACITY)
    _refused(lib, lib.ad_cache_attention_shared(c, *{**a, "scratch": None}.values(), None, None))
    for bad in (dict(n=-1), dict(G=0), dict(G=3), dict(shared=-1), dict(M=-1), dict(dtype=9), dict(new=0)):
        f = {**dict(dtype=1, heads=4, B=2, M=5, new=3, n=100, G=1, shared=90), **bad}
        assert lib.ad_cache_attention_shared_scratch_bytes(c, *f.values()) == 0
    # as many tokens, heads, rows and groups as there may be: counted in 64 bits
    wide = C.byref(_cache(table_stride=1 << 23, head_dim=128, n_kv_heads=16, n_blocks=1 << 30))
    assert lib.ad_cache_attention_shared_scratch_bytes(wide, 0, 64, 8192, 1 << 24, 1 << 15, (1 << 31) - 1, 1, (1 << 31) - 1) > 3 << 39
    assert lib.ad_cache_attention_shared(c, *{**SHARED, "M": 0, "q": None, "out": None}.values(), None, None) == binding.AD_OK


@pytest.mark.parametrize("bad", [dict(scores=None), dict(scores=P + 2), dict(out=P + 1), dict(stride=999), dict(out_stride=999), dict(dtype=3), dict(vocab=0),
                                 dict(vocab=(1 << 20) + 1, stride=1 << 21, out_stride=1 << 21), dict(M=-1), dict(M=1 << 29), dict(r=None), dict(tokens=None),
                                 dict(out=P + 4000), dict(out=P + 4 * 4999), dict(out=P - 4 * 4999), dict(out=P, out_stride=1001)])
def test_sample_refusals(lib, bad):
    _refused(lib, lib.ad_sample(*{**SAMPLE, **bad}.values(), None, None))


def test_sampling_no_rows_is_no_error(lib):
    assert lib.ad_sample(*{**SAMPLE, "M": 0, "scores": None, "r": None, "tokens": None}.values(), None, None) == binding.AD_OK


def test_struct_layout():
    assert C.sizeof(binding.KvPoolStruct) == 2 * 8 + 4 * 4


def test_pool_without_a_gpu_is_refused():
    with pytest.raises(binding.AdError, match="CUDA"):
        binding.KvPool(2, 4, 8, device="cpu")


class _NoLaunch:
    def __getattr__(self, name):
        if name.endswith("scratch_bytes"):
            return lambda *_: 0
        def reached(*a):
            raise AssertionError("reached the library")
        return reached


def test_tensors_that_sampling_refuses(monkeypatch):
    """Scores that do not lie next to each other, parameters of other types, lengths or places, and sizes that 32 bits do not hold."""
    monkeypatch.setattr(binding, "_lib", _NoLaunch())
    monkeypatch.setattr(binding, "_call_on", lambda dev, call, *a: call(*a, None))
    on = _OnDevice
    r, x = on(torch.zeros(3)), on(torch.zeros(3, 40))
    full = lambda n=3, dtype=torch.float32: on(torch.zeros(n, dtype=dtype))
    for scores in (torch.zeros(3, 80)[:, ::2], torch.zeros(3, 1).expand(3, 40), torch.zeros(40), torch.zeros(3, 40, dtype=torch.float64), torch.zeros(3, 40, dtype=torch.float16)):
        with pytest.raises(binding.AdError, match="next to each other|scores are"):
            binding.sample(on(scores), r)
    with pytest.raises(binding.AdError, match="scores are"):
        binding.sample(torch.zeros(3, 40), torch.zeros(3))
    for kw in (dict(temperature=full(2)), dict(temperature=full(3, torch.float64)), dict(top_k=full(3)), dict(top_p=full(3, torch.int32)), dict(min_p=torch.zeros(3)),
               dict(temperature=on(torch.zeros(6)[::2]))):
        with pytest.raises(binding.AdError, match="contiguous"):
            binding.sample(x, r, **kw)
    for out in (full(), on(torch.zeros(3, 41)), on(torch.zeros(3, 40, dtype=torch.bfloat16)), torch.zeros(3, 40)):
        with pytest.raises(binding.AdError, match="like them"):
            binding.sample(x, r, filtered=out)
    with pytest.raises(binding.AdError, match="next to each other"):
        binding.sample(x, r, filtered=on(torch.zeros(3, 80)[:, ::2]))
    with pytest.raises(binding.AdError, match="2\\^31|large|32"):
        binding.sample(on(torch.empty((1, (1 << 32) + 5), device="meta")), on(torch.zeros(1)))
    with pytest.raises(AssertionError, match="reached"):
        binding.sample(x, r, full(), full(3, torch.int32), full(), full(), filtered=x)


HOST = """
#include <stdio.h>
#include "block_pool.cuh"
#include "shared_attention.cuh"
using namespace ad;
#define CHECK(x) do { if (!(x)) { printf("line %d: %s\\n", __LINE__, #x); return 1; } } while (0)
int main() {
  pool::Pool p = {nullptr, nullptr, 6, 4, 8, 32};
  int fault;
  auto heir = [&](int parent, int len) { return pool::heir(p, 5, parent, len, fault); };
  CHECK(p.there(0) && p.there(7) && !p.there(8) && !p.there(-1) && !p.there(INT_MIN));
  // blocks of a length, rows that are to be empty (whatever their length), parents and lengths that make no sense
  CHECK(heir(4, 0).held == 0 && heir(4, 1).held == 1 && heir(4, 32).held == 1 && heir(4, 33).held == 2 && heir(4, 128).held == 4 && fault == AD_OK);
  CHECK(heir(-1, 5).parent == pool::EMPTY && fault == AD_OK && heir(INT_MIN, -9).parent == pool::EMPTY && fault == AD_OK);
  CHECK(heir(5, 1).parent == pool::AS_IT_WAS && fault == AD_ERR_ARG && heir(0, -1).parent == pool::AS_IT_WAS && fault == AD_ERR_ARG);
  CHECK(heir(0, 129).parent == pool::AS_IT_WAS && fault == AD_ERR_CAPACITY && heir(INT_MAX, 1).parent == pool::AS_IT_WAS && fault == AD_ERR_ARG);
  pool::Span s;
  auto span = [&](int o0, int o1, int len) { return pool::span_of(p, o0, o1, len, s, fault); };
  CHECK(!span(3, 3, 500) && fault == AD_OK && !span(3, 3, -1) && fault == AD_OK);      // (a row without new tokens is left alone)
  CHECK(span(0, 1, 0) && s.first == 0 && s.last == 0 && s.live == 0);
  CHECK(span(2, 34, 31) && s.first == 0 && s.last == 1 && s.live == 31);
  CHECK(span(2, 3, 64) && s.first == 2 && s.last == 2 && s.live == 0);
  CHECK(span(0, 128, 0) && s.last == 3 && !span(0, 129, 0) && fault == AD_ERR_CAPACITY && !span(0, 1, 128) && fault == AD_ERR_CAPACITY);
  CHECK(!span(4, 3, 0) && fault == AD_ERR_ARG && !span(-1, 3, 0) && fault == AD_ERR_ARG && !span(0, 1, -1) && fault == AD_ERR_ARG);
  CHECK(!span(0, INT_MAX, INT_MAX) && fault == AD_ERR_CAPACITY && !span(INT_MIN, INT_MAX, 0) && fault == AD_ERR_ARG);
  // the longest rows and the largest tables that calls accept do not wrap around
  p.stride = (INT_MAX - (1 << 19)) / 128; p.block = 128;
  CHECK(heir(0, p.stride * 128).held == p.stride && heir(0, p.stride * 128 - 1).held == p.stride && fault == AD_OK);
  CHECK(heir(0, INT_MAX).parent == pool::AS_IT_WAS && fault == AD_ERR_CAPACITY);
  CHECK(span(0, 1 << 19, p.stride * 128 - (1 << 19)) && s.last == p.stride - 1);
  // rows that begin at a later block
  int table[8] = {0, 7, 8, -1, 5, 6, 3, 2}, first[2] = {1, 2};
  kv::Cache c = {};
  c.table = table; c.table_stride = 4; c.n_blocks = 8; c.block = 32; c.first = first;
  CHECK(c.find(0, 0) == 7 && c.find(0, 1) == -1 && c.find(1, 0) == 3 && c.find(1, 1) == 2);
  // wherever an item's granules are cut, every tile of keys belongs to one part
  for (int weight = 1; weight <= 2; ++weight)
    for (int kt = 1; kt < 40; ++kt) {
      const int per = kt * weight + shr::FIXED;
      for (int a = 0; a < per; ++a)
        for (int b = a + 1; b <= per; ++b) {
          auto cut = [&](int x) { const int t = shr::tile_at(x, weight); return t < kt ? t : kt; };
          CHECK(cut(0) == 0 && cut(a) <= cut(b) && cut(per) == kt);
        }
    }
  // keys and values take turns, and none of the places twice
  int seen[256] = {};
  for (int g = 0; g < 60; ++g) { ++seen[shr::keys_fill(g)]; ++seen[shr::values_fill(g)]; }
  for (int i = 0; i < 119; ++i) CHECK(seen[i] == 1);
  return 0;
}
"""


@pytest.mark.skipif(not os.path.exists(NVCC), reason="no CUDA compiler")
def test_what_kernels_decide_by(tmp_path):
    src, exe = tmp_path / "pool.cu", tmp_path / "pool"
    src.write_text(HOST)
    subprocess.run([NVCC, "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-I", build.CSRC, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout


APPEND_POOLED = dict(k=P, v=P, dtype=1, stride=128, off=P, len=P, B=3, M=5, max_new=3)


@pytest.mark.parametrize("bad", [dict(off=None), dict(len=None), dict(B=0), dict(B=7), dict(M=-1), dict(max_new=0), dict(max_new=1 << 20), dict(dtype=2), dict(k=None), dict(v=P + 8),
                                 dict(stride=120), dict(stride=130)])
def test_pooled_append_refusals(lib, bad):
    _refused(lib, lib.ad_cache_append_pooled(_pool(), C.byref(_cache()), *{**APPEND_POOLED, **bad}.values(), None, None))


def test_pooled_append_of_pools_and_caches_that_do_not_belong_together(lib):
    for bad in BAD_POOL:
        _refused(lib, lib.ad_cache_append_pooled(_pool(**bad), C.byref(_cache()), *APPEND_POOLED.values(), None, None))
    for bad in [b for b in BAD_CACHE if "table" not in b] + [dict(table=None), dict(table=P + 4), dict(table_stride=5), dict(n_blocks=9), dict(block=64)]:
        _refused(lib, lib.ad_cache_append_pooled(_pool(), C.byref(_cache(**bad)), *APPEND_POOLED.values(), None, None))
    _refused(lib, lib.ad_cache_append_pooled(None, C.byref(_cache()), *APPEND_POOLED.values(), None, None))
    _refused(lib, lib.ad_cache_append_pooled(_pool(), None, *APPEND_POOLED.values(), None, None))
    assert lib.ad_cache_append_pooled(_pool(), C.byref(_cache()), *{**APPEND_POOLED, "M": 0, "k": None, "v": None}.values(), None, None) == binding.AD_OK


@pytest.mark.parametrize("heads,B,max_new", [(4, 17, 1), (2, 65, 8), (8, 7, 64)])
def test_rows_own_positions_are_planned_for_whatever_others_share(lib, heads, B, max_new):
    """A row may share nothing and be as long as any (max_keys): the attention over its own positions is planned, and given scratch, as cache_attention's would be, whatever the longest
    prefix is."""
    c, M, keys = C.byref(_cache(table_stride=1 << 20)), B * max_new, 1 << 24
    need = {n: lib.ad_cache_attention_shared_scratch_bytes(c, 1, heads, B, M, max_new, keys, 2, n) for n in (keys, keys - 300, keys - 5000, keys // 2)}
    own = lib.ad_cache_attention_scratch_bytes(c, 1, heads, B, max_new, keys)
    assert own > 0 and len(set(need.values())) == 1 and need[keys] > own, (need, own)


def test_a_prefix_that_nobody_named_is_not_planned_for(monkeypatch):
    """Without max_shared the call does not take max_keys for the longest prefix: rows of many positions of their own would go the way that pays for long prefixes."""
    seen = []

    class Lib:
        def ad_cache_attention_shared_scratch_bytes(self, *a):
            return 0

        def ad_cache_attention_shared(self, *a):
            seen.append(a)
            return binding.AD_OK
    monkeypatch.setattr(binding, "_lib", Lib())
    monkeypatch.setattr(binding, "_call_on", lambda dev, call, *a: call(*a, None))
    monkeypatch.setattr(binding, "_BF16", torch.bfloat16)
    monkeypatch.setattr(binding, "_FP32", torch.float32)
    monkeypatch.setattr(binding, "_INT32", torch.int32)
    cache = object.__new__(binding.KvCache)
    cache._dev, cache.device, cache._table_rows, cache.n_kv_heads, cache.head_dim, cache._scratch, cache._ref = 0, "cuda:0", 4, 2, 64, {}, None
    i32 = lambda n: _OnDevice(torch.zeros(n, dtype=torch.int32))
    q, out = (_OnDevice(torch.zeros(3, 4, 64, dtype=torch.bfloat16)) for _ in range(2))
    for kw, want in (({}, 0), (dict(max_shared=None), 0), (dict(max_shared=0), 0), (dict(max_shared=4000), 4000), (dict(max_shared=20000), 20000)):
        binding.cache_attention_shared(cache, q, i32(3), i32(2), i32(2), i32(1), 3, 20000, out=out, **kw)
        args = dict(zip("cache q dtype stride heads off len B M max_new max_keys group shared G max_shared".split(), seen.pop()))
        assert (args["max_keys"], args["G"], args["max_shared"]) == (20000, 1, want)


def test_pools_of_more_blocks_than_32_bits_can_number(lib):
    """The planning kernels count holes and movers behind one another, and walk the counts some way beyond the last one."""
    for n in ((1 << 30) - 511, 1 << 30, (1 << 31) - 257, (1 << 31) - 1):
        pool = _pool(n_blocks=n)
        _refused(lib, lib.ad_cache_fork(pool, P, P, 3, None, None))
        _refused(lib, lib.ad_cache_reserve(pool, None, 0, P, P, 3, P, HUGE, None, None))
        _refused(lib, lib.ad_cache_append_pooled(pool, C.byref(_cache(n_blocks=n)), *APPEND_POOLED.values(), None, None))
        _refused(lib, lib.ad_cache_compact(pool, None, 0, P, P, HUGE, None))
        assert lib.ad_cache_reserve_scratch_bytes(pool, 3) == 0 and lib.ad_cache_compact_scratch_bytes(pool) == 0
    most = (1 << 30) - 512
    # claims, lists and moves of as many blocks as there may be, counted in 64 bits
    assert lib.ad_cache_reserve_scratch_bytes(_pool(n_blocks=most), 3) > 12 * most and lib.ad_cache_compact_scratch_bytes(_pool(n_blocks=most)) > 18 * most - 4096
    # the last index of either list, and the last step of a walk
    assert 2 * most - 1 < 2 ** 31 and most + 2 * 256 < 2 ** 31


OVERLAP = """
#include <stdio.h>
#include "cache_checks.h"
int main() {
  for (size_t element = 2; element <= 4; element += 2)
    for (size_t vocab = 1; vocab <= 3; ++vocab)
      for (size_t M = 1; M <= 3; ++M)
        for (size_t sa = vocab; sa <= 8; ++sa)
          for (size_t sb = vocab; sb <= 8; ++sb)
            for (int d = -30; d <= 30; ++d) {
              const uintptr_t a = 4096, b = a + d * (intptr_t)element;
              bool touch = false;
              for (size_t i = 0; i < M; ++i)
                for (size_t j = 0; j < M; ++j) touch = touch || (a + i * sa * element < b + (j * sb + vocab) * element && b + j * sb * element < a + (i * sa + vocab) * element);
              const bool itself = d == 0 && (sa == sb || M == 1), said = ad::rows_overlap(a, sa, b, sb, vocab, M, element);
              // never let through what touches, and with one stride nothing else refused
              if ((touch && !itself && !said) || (itself && said) || (sa == sb && !touch && said)) { printf("%zu %zu %zu %zu %zu %d\\n", element, vocab, M, sa, sb, d); return 1; }
            }
  return 0;
}
"""


@pytest.mark.skipif(not os.path.exists(NVCC), reason="no CUDA compiler")
def test_what_overlaps(tmp_path):
    """Against every pair of rows: in place, apart, between the rows, partly over them."""
    src, exe = tmp_path / "overlap.cu", tmp_path / "overlap"
    src.write_text(OVERLAP)
    subprocess.run([NVCC, "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-I", build.CSRC, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout


def test_pairs_are_read_row_by_row(lib):
    """What a group's positions take when they are read once is nearly what two rows take: pairs are not worth it at lengths where more rows are."""
    c = C.byref(_cache(table_stride=1 << 20, n_blocks=1 << 20))
    for dtype in (0, 1):
        for G, n, once in ((1, 2, False), (8, 2, False), (1, 16, True), (8, 16, True), (1, 64, True), (4, 3, True)):
            B, new, keys = G * n, 4, 14000
            sizes = (c, dtype, 2, B, B * new, new, keys + 300, G, keys)
            alone = lib.ad_cache_attention_scratch_bytes(c, dtype, 2, B, new, keys + 300)
            got = lib.ad_cache_attention_shared_scratch_bytes(*sizes)
            assert (got > alone) == (once and (B - 1.9 * G) * 2 * (keys // 32) >= 9000 + 20 * B + 0.4 * B * new), (dtype, G, n)
            assert once or got == alone
