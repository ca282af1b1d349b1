"""Calls of the 8-bit cache and of sampled verification that are refused before anything reaches a GPU, and the checks that kernels make of what only
the device knows (offsets, lengths, tables), compiled for the host."""
import ctypes as C
import os
import subprocess

import pytest

from paper_2205_10350_b200 import binding, build

NVCC = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
P = 1 << 20          # an aligned address; nothing is launched on it


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load()


def _cache(**kw):
    f = dict(k_codes=P, v_codes=P, k_scale=P, v_scale=P, table=P, table_stride=4, n_blocks=8, n_kv_heads=2, block=32, head_dim=64, format=0)
    f.update(kw)
    return binding.KvCacheStruct(*(f[n] for n, _ in binding.KvCacheStruct._fields_))


APPEND = dict(k=P, v=P, dtype=1, stride=128, off=P, len=P, B=2, M=5, max_new=3)
ATTEND = dict(q=P, dtype=1, stride=256, heads=4, off=P, len=P, B=2, M=5, max_new=3, max_keys=100, causal=1, scale=0.125, out=P, scratch=P, nbytes=1 << 40)
ACCEPT = dict(target=P, ts=1000, draft=P, ds=1000, dtype=0, t=1.0, vocab=1000, off=P, drafts=P, kmax=5, B=2, M=5, u=P, r=P, eos=-1, tokens=P, n=P,
              scratch=P, nbytes=1 << 40)

BAD_CACHE = [dict(k_codes=None), dict(v_scale=None), dict(k_codes=P + 8), dict(table_stride=0), dict(n_blocks=0), dict(n_kv_heads=0), dict(block=48),
             dict(block=0), dict(head_dim=96), dict(head_dim=0), dict(format=2), dict(table_stride=1 << 27), dict(table=None, table_stride=5)]


def _refused(lib, rc, want=binding.AD_ERR_ARG):
    assert rc == want
    assert len(lib.ad_last_error(None)) > 10


@pytest.mark.parametrize("bad", BAD_CACHE)
def test_caches_that_cannot_be(lib, bad):
    c = C.byref(_cache(**bad))
    _refused(lib, lib.ad_cache_append(c, *APPEND.values(), None, None))
    _refused(lib, lib.ad_cache_read(c, P, P, 1, P, P, 2, 5, 3, None, None))
    _refused(lib, lib.ad_cache_attention(c, *ATTEND.values(), None, None))


@pytest.mark.parametrize("bad", [dict(off=None), dict(len=None), dict(B=0), dict(B=70000), dict(M=-1), dict(max_new=0), dict(max_new=1 << 20), dict(dtype=2),
                                 dict(k=None), dict(v=P + 8), dict(stride=120), dict(stride=130)])
def test_append_refusals(lib, bad):
    c = C.byref(_cache())
    _refused(lib, lib.ad_cache_append(c, *{**APPEND, **bad}.values(), None, None))
    if "stride" not in bad:
        a = {**APPEND, **bad}
        _refused(lib, lib.ad_cache_read(c, a["k"], a["v"], a["dtype"], a["off"], a["len"], a["B"], a["M"], a["max_new"], None, None))
    _refused(lib, lib.ad_cache_append(None, *APPEND.values(), None, None))


@pytest.mark.parametrize("bad", [dict(q=None), dict(q=P + 2), dict(out=None), dict(out=P + 4), dict(dtype=7), dict(stride=255), dict(stride=260), dict(heads=3),
                                 dict(heads=0), dict(off=None), dict(len=None), dict(B=0), dict(M=-5), dict(max_new=0), dict(max_keys=-1), dict(scale=0.0),
                                 dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=3e38), dict(heads=65534, stride=65534 * 64, max_new=600),
                                 dict(max_new=1 << 20)])
def test_attention_refusals(lib, bad):
    _refused(lib, lib.ad_cache_attention(C.byref(_cache()), *{**ATTEND, **bad}.values(), None, None))


@pytest.mark.parametrize("bad", [dict(target=None), dict(target=P + 2), dict(draft=P + 1), dict(ts=999), dict(ds=999), dict(dtype=3), dict(t=0.0), dict(t=-1.0),
                                 dict(t=float("nan")), dict(t=float("inf")), dict(t=1e-35), dict(vocab=0), dict(vocab=(1 << 20) + 1, ts=1 << 21, ds=1 << 21), dict(off=None), dict(drafts=None),
                                 dict(kmax=0), dict(B=0), dict(M=-1), dict(u=None), dict(r=None), dict(tokens=None), dict(n=None), dict(scratch=None),
                                 dict(scratch=P + 128)])
def test_sampled_verification_refusals(lib, bad):
    _refused(lib, lib.ad_accept_sampled(*{**ACCEPT, **bad}.values(), None, None))


def test_too_little_scratch(lib):
    need = lib.ad_accept_sampled_scratch_bytes(5, 1000, 1)
    assert need > lib.ad_accept_sampled_scratch_bytes(5, 1000, 0) > 0
    _refused(lib, lib.ad_accept_sampled(*{**ACCEPT, "nbytes": need - 1}.values(), None, None), binding.AD_ERR_CAPACITY)


def test_nothing_to_do_is_no_error(lib):
    c = C.byref(_cache())
    assert lib.ad_cache_append(c, *{**APPEND, "M": 0, "k": None, "v": None}.values(), None, None) == binding.AD_OK
    assert lib.ad_cache_read(c, None, None, 1, P, P, 2, 0, 3, None, None) == binding.AD_OK
    assert lib.ad_cache_attention(c, *{**ATTEND, "M": 0, "q": None, "out": None}.values(), None, None) == binding.AD_OK


def test_struct_layout():
    assert C.sizeof(binding.KvCacheStruct) == 5 * 8 + 6 * 4


def test_cache_without_a_gpu_is_refused():
    with pytest.raises(binding.AdError, match="CUDA"):
        binding.KvCache(4, 2, 64, device="cpu")
    with pytest.raises(binding.AdError, match="format"):
        binding.KvCache(4, 2, 64, fmt="fp4")


@pytest.mark.skipif(not os.path.exists(NVCC), reason="no CUDA compiler")
def test_what_kernels_check_of_rows_and_tables(tmp_path):
    src = tmp_path / "rows.cu"
    src.write_text("""
#include <stdio.h>
#include "kv_cache.cuh"
using namespace ad;
#define CHECK(x) do { if (!(x)) { printf("line %d: %s\\n", __LINE__, #x); return 1; } } while (0)
int main() {
  int table[8] = {0, 7, 8, -1, INT_MAX, INT_MIN, 3, 2};
  kv::Cache c = {};
  c.table = table; c.table_stride = 4; c.n_blocks = 8; c.block = 32;
  CHECK(c.find(0, 0) == 0 && c.find(0, 1) == 7 && c.find(0, 2) == -1 && c.find(0, 3) == -1);
  CHECK(c.find(1, 0) == -1 && c.find(1, 1) == -1 && c.find(1, 2) == 3 && c.find(1, 3) == 2);
  c.table = nullptr;
  CHECK(c.find(0, 3) == 3 && c.find(1, 3) == 7 && c.find(2, 0) == -1);
  // capacity 128 tokens a row, 10 tokens in the batch, at most 6 a row
  CHECK(kv::row_fault(c, 0, 6, 0, 10, 6, 6) == AD_OK && kv::row_fault(c, 4, 6, 122, 10, 6, 6) == AD_OK);
  CHECK(kv::row_fault(c, 4, 6, 123, 10, 6, 6) == AD_ERR_CAPACITY && kv::row_fault(c, 0, 1, INT_MAX, 10, 6, 1) == AD_ERR_CAPACITY);
  CHECK(kv::row_fault(c, 5, 6, 0, 10, 6, 6) == AD_ERR_ARG && kv::row_fault(c, -1, 2, 0, 10, 6, 2) == AD_ERR_ARG);
  CHECK(kv::row_fault(c, 0, 7, 0, 10, 6, 7) == AD_ERR_ARG && kv::row_fault(c, 0, -1, 0, 10, 6, -1) == AD_ERR_ARG);
  CHECK(kv::row_fault(c, 0, 2, -1, 10, 6, 2) == AD_ERR_ARG && kv::row_fault(c, INT_MAX, 2, 0, 10, 6, 2) == AD_ERR_ARG);
  // queries that only look at the row
  CHECK(kv::row_fault(c, 0, 6, 128, 10, 6, 0) == AD_OK && kv::row_fault(c, 0, 6, 129, 10, 6, 0) == AD_ERR_CAPACITY);
  // the longest capacity that calls accept does not wrap around
  c.table_stride = (INT_MAX - (1 << 19)) / 128; c.block = 128;
  CHECK(kv::row_fault(c, 0, 1 << 19, c.table_stride * 128 - (1 << 19), 1 << 20, 1 << 19, 1 << 19) == AD_OK);
  CHECK(kv::row_fault(c, 0, 1 << 19, c.table_stride * 128 - (1 << 19) + 1, 1 << 20, 1 << 19, 1 << 19) == AD_ERR_CAPACITY);
  return 0;
}
""")
    exe = tmp_path / "rows"
    subprocess.run([NVCC, "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-I", build.CSRC, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout


@pytest.mark.skipif(not os.path.exists(NVCC), reason="no CUDA compiler")
def test_shares_of_work_cover_it_once(tmp_path):
    """The attention's CTAs share granules of work evenly and in order; the join finds by arithmetic which of them had a part of an item."""
    src = tmp_path / "shares.cu"
    src.write_text("""
#include <stdio.h>
#include "cache_attention.cuh"
using namespace ad;
#define CHECK(x) do { if (!(x)) { printf("line %d: %s (%lld granules, %lld CTAs)\\n", __LINE__, #x, total, ctas); return 1; } } while (0)
int main() {
  const long long totals[] = {1, 2, 3, 7, 64, 147, 148, 149, 443, 444, 445, 1000, 12501, 1ll << 33, (1ll << 40) + 17};
  for (long long total : totals)
    for (long long grid = 1; grid <= 900; grid += 1 + grid / 7) {
      const long long ctas = grid < total ? grid : total;
      CHECK(kv::cta_start(total, 0, ctas) == 0 && kv::cta_start(total, ctas, ctas) == total);
      for (long long c = 0; c < ctas; ++c) {
        const long long a = kv::cta_start(total, c, ctas), e = kv::cta_start(total, c + 1, ctas);
        CHECK(a < e && e - a <= (total + ctas - 1) / ctas);
        CHECK(kv::cta_of(total, a, ctas) == c && kv::cta_of(total, e - 1, ctas) == c && kv::cta_of(total, a + (e - a) / 2, ctas) == c);
      }
    }
  return 0;
}
""")
    exe = tmp_path / "shares"
    subprocess.run([NVCC, "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-I", build.CSRC, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout


class _OnDevice:
    """A tensor of the CPU that says it lies on device 0; what would be launched on it is looked at instead."""

    def __init__(self, t):
        self.t = t

    def get_device(self):
        return 0

    def __getattr__(self, name):
        return getattr(self.t, name)

    @property
    def shape(self):
        return self.t.shape


class _NoLaunch:
    def ad_accept_sampled_scratch_bytes(self, *_):
        return 4096

    def ad_accept_sampled(self, *a):
        raise AssertionError("reached the library")


def _accept(monkeypatch, target, draft, B=1, kmax=2):
    import torch
    monkeypatch.setattr(binding, "_lib", _NoLaunch())
    monkeypatch.setattr(binding, "_call_on", lambda dev, call, *a: call(*a, None))
    i32 = lambda *s: _OnDevice(torch.zeros(s, dtype=torch.int32))
    f32 = lambda *s: _OnDevice(torch.zeros(s))
    return binding.accept_sampled(_OnDevice(target), None if draft is None else _OnDevice(draft), i32(B, kmax), i32(B + 1), f32(B, kmax), f32(B))


@pytest.mark.parametrize("M", [1, 2])
def test_scores_that_do_not_lie_next_to_each_other_are_refused(monkeypatch, M):
    """One score for a whole row (a stride of zero) is not a row of scores: kernels would read behind it."""
    import torch
    full, column, spread = torch.zeros(M, 40), torch.zeros(M, 1).expand(M, 40), torch.zeros(M, 80)[:, ::2]
    wide = torch.zeros(M * 100).as_strided((M, 40), (100, 0))
    for t, d in ((column, None), (spread, None), (wide, None), (column, full), (full, column), (wide, full), (full, wide), (full, spread), (spread, full), (wide, wide)):
        with pytest.raises(binding.AdError, match="next to each other|overlap"):
            _accept(monkeypatch, t, d)
    for t, d in ((full, None), (full, full), (torch.zeros(M, 60)[:, 7:47], full)):
        with pytest.raises(AssertionError, match="reached"):
            _accept(monkeypatch, t, d)


def test_sizes_that_32_bits_do_not_hold_are_refused(monkeypatch):
    """The library's sizes are 32-bit; a larger one would arrive as another number, a vocabulary of 2^32 + 5 as one of five."""
    import torch
    big = (1 << 32) + 5
    for M, V in ((1, big), (big, 1), (1, 1 << 31)):
        scores = torch.empty((M, V), device="meta")
        for draft in (None, scores):
            with pytest.raises(binding.AdError, match="2\\^31"):
                _accept(monkeypatch, scores, draft)
    # a cache's calls, up to where they would reach the library
    cache = object.__new__(binding.KvCache)
    cache._dev, cache.device, cache._table_rows, cache.n_kv_heads, cache.head_dim, cache._scratch, cache._ref = 0, "cuda:0", 4, 2, 64, {}, None
    i32 = lambda n: _OnDevice(torch.zeros(n, dtype=torch.int32))
    x = _OnDevice(torch.zeros(3, 2, 64, dtype=torch.bfloat16))
    monkeypatch.setattr(binding, "_BF16", torch.bfloat16)
    monkeypatch.setattr(binding, "_INT32", torch.int32)
    for bad in (big, 1 << 31, -1):
        for call in (lambda: binding.cache_append(cache, x, x, i32(2), i32(1), bad), lambda: binding.cache_attention(cache, x, i32(2), i32(1), bad, 10),
                     lambda: binding.cache_attention(cache, x, i32(2), i32(1), 3, bad), lambda: binding.cache_read(cache, i32(2), i32(1), 3, bad),
                     lambda: binding.cache_read(cache, i32(2), i32(1), bad, 3)):
            with pytest.raises(binding.AdError, match="2\\^31"):
                call()


@pytest.mark.parametrize("heads,max_new", [(4, 3), (2, 1 << 19), (64, 1 << 10)])
def test_longer_rows_than_there_can_be_are_planned_as_the_longest(lib, heads, max_new):
    """max_keys up to INT_MAX ("no bound") plans like the capacity of a row, for a single row and for the most that a batch can have."""
    for table_stride, B in ((300, 1), (300, 65535), ((2 ** 31 - 2 ** 19 - 1) // 32, 1), ((2 ** 31 - 2 ** 19 - 1) // 32, 65535)):
        c = C.byref(_cache(table_stride=table_stride))
        need = [lib.ad_cache_attention_scratch_bytes(c, 1, heads, B, max_new, n) for n in (table_stride * 32, 2 ** 31 - 1, 2 ** 31 - 31, 2 ** 31 - 32)]
        assert need[0] > 0 and len(set(need)) == 1, need
        # as many parts at the most as twice the CTAs that an SM and 4096 SMs could hold, and a place per row
        assert need[0] <= 2 * 5 * 4096 * 32 * (64 + 2) * 4 + 8 * (B + 2)
        _refused(lib, lib.ad_cache_attention(c, *{**ATTEND, "heads": heads, "stride": heads * 64, "B": B, "max_new": max_new, "max_keys": 2 ** 31 - 1,
                                                  "nbytes": need[0] - 1}.values(), None, None), binding.AD_ERR_CAPACITY)


def test_scratch_of_as_many_tokens_as_there_can_be(lib):
    """Rows of scores counted in 32 bits: a part for each, 8 bytes, and no sum on the way that passes them."""
    most = (2 ** 31 - 1) // 2
    assert lib.ad_accept_sampled_scratch_bytes(most, 8, 1) == most * 2 * 8
    assert lib.ad_accept_sampled_scratch_bytes(most, 8, 0) == most * 8
    assert lib.ad_accept_sampled_scratch_bytes(most + 1, 8, 0) == 0
