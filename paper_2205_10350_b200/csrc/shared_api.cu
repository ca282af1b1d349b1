// Operator-level entry point of attention over shared prefixes, declared in include/aggressive_decoding.h.
#include <math.h>

#include <algorithm>
#include <atomic>

#include "cache_checks.h"
#include "shared_attention.cuh"

using namespace ad;

namespace {

constexpr int kSharedRows = 8192;

size_t rounded(size_t bytes) { return (bytes + 255) / 256 * 256; }

struct Scratch { size_t total, lines, start, ml, part, bytes; long long part_rows; int grid; };
// Results: of every query and head once in its group's items and once in its row's, and as much as an item's between the CTAs' parts.
Scratch scratch_of(const ad_kv_cache* c, int32_t n_heads, int32_t B, int32_t M, int32_t G) {
  Scratch s;
  s.grid = op_num_sms();
  s.part_rows = 2ll * M * n_heads + (long long)s.grid * shr::ITEM_ROWS;
  s.total = 0;
  s.lines = 256;
  s.start = s.lines + rounded(((size_t)G + B) * sizeof(shr::Line));
  s.ml = s.start + rounded(s.grid * sizeof(shr::Start));
  s.part = s.ml + rounded(2 * (size_t)s.part_rows * sizeof(float2));
  s.bytes = s.part + rounded(2 * (size_t)s.part_rows * c->head_dim * sizeof(float));
  return s;
}
const char* shared_fault(const ad_kv_cache* c, int32_t dtype, int32_t n_heads, int32_t B, int32_t M, int32_t max_new, int32_t max_keys, int32_t G, int32_t max_shared) {
  if (const char* why = cache_fault(c, B)) return why;
  if (B < 1 || B > kSharedRows) return "1 to 8192 rows";
  if (G < 1 || G > B) return "1 to as many groups as rows";
  if (M < 0) return "negative number of tokens";
  if (max_new < 1 || max_new > kMaxNew) return "1 to 2^19 tokens of a row";
  if (!known_dtype(dtype)) return "unknown dtype";
  if (n_heads < 1 || n_heads > 65535 || n_heads % c->n_kv_heads != 0 || (int64_t)M * n_heads > (1 << 30))
    return "query heads must be a multiple of the cache's, at most 65535, and tokens times them at most 2^30";
  if ((int64_t)max_new * n_heads > (1 << 30)) return "max_new times the query heads may be 2^30 at most";
  if (max_keys < 0 || max_shared < 0) return "negative number of keys";
  return nullptr;
}

template <typename T, typename F, int DIM>
cudaError_t launch_shared(const shr::Params& a, cudaStream_t st) {
  static std::atomic<uint64_t> raised{0};              // devices on which the kernel may use its shared memory
  auto kernel = shr::shared_attention_kernel<T, F, DIM>;
  constexpr int smem = shr::smem_bytes<DIM, sizeof(T) == 4>();
  static_assert(smem <= 227 * 1024, "an SM's shared memory");
  const uint64_t bit = 1ull << op_device();
  cudaError_t e = cudaSuccess;
  if (!(raised.load(std::memory_order_relaxed) & bit)) {
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    raised.fetch_or(bit, std::memory_order_relaxed);
  }
  e = launch_op(shr::shared_plan_kernel, dim3(1), dim3(shr::PLAN_THREADS), dim3(), 0, st, a);
  if (e == cudaSuccess) e = launch_op(kernel, dim3(a.grid), dim3(shr::THREADS), dim3(), smem, st, a);
  const long long warps = (long long)a.max_new * a.n_heads, each = shr::JOIN_THREADS / 32;
  if (e == cudaSuccess) e = launch_op(shr::shared_join_kernel<T, DIM>, dim3((unsigned)((warps + each - 1) / each), a.B), dim3(shr::JOIN_THREADS), dim3(), 0, st, a);
  return e;
}
template <typename T, typename F>
cudaError_t launch_shared_dim(int dim, const shr::Params& a, cudaStream_t st) {
  return dim == 32 ? launch_shared<T, F, 32>(a, st) : dim == 64 ? launch_shared<T, F, 64>(a, st) : launch_shared<T, F, 128>(a, st);
}

}  // namespace

extern "C" size_t ad_cache_attention_shared_scratch_bytes(const ad_kv_cache* c, int32_t dtype, int32_t n_heads, int32_t B, int32_t M, int32_t max_new,
                                                          int32_t max_keys, int32_t G, int32_t max_shared) {
  if (shared_fault(c, dtype, n_heads, B, M, max_new, max_keys, G, max_shared)) return 0;
  return scratch_of(c, n_heads, B, M, G).bytes;
}

extern "C" int ad_cache_attention_shared(const ad_kv_cache* c, const void* q, int32_t dtype, int64_t q_stride, int32_t n_heads, const int32_t* off,
                                         const int32_t* len, int32_t B, int32_t M, int32_t max_new, int32_t max_keys, const int32_t* group,
                                         const int32_t* shared, int32_t G, int32_t max_shared, int32_t causal, float scale, void* out, void* scratch,
                                         size_t scratch_bytes, int32_t* status, void* stream) {
  const char* entry = "ad_cache_attention_shared";
  if (!off || !len || !group || !shared) return arg_fault(entry, "null offsets, lengths or groups");
  if (const char* why = shared_fault(c, dtype, n_heads, B, M, max_new, max_keys, G, max_shared)) return arg_fault(entry, why);
  if (!(scale > 0.f) || !(scale <= 1e30f)) return arg_fault(entry, "the scale must be positive, and 1e30 at most");
  if (M == 0) return AD_OK;
  if (!q || !out || !aligned(q, 16) || !aligned(out, 16)) return arg_fault(entry, "queries and result must be 16-byte aligned");
  if (q_stride < (int64_t)n_heads * c->head_dim || q_stride % (int64_t)(16 / dtype_bytes(dtype)))
    return arg_fault(entry, "queries must be a multiple of 16 bytes apart, and not overlap");
  const Scratch s = scratch_of(c, n_heads, B, M, G);
  if (scratch_bytes < s.bytes) return op_fail(AD_ERR_CAPACITY, entry, "scratch too small");
  if (!scratch || !aligned(scratch, 256)) return arg_fault(entry, "scratch must be 256-byte aligned");
  char* at = static_cast<char*>(scratch);
  shr::Params a = {};
  a.c = device_cache(c); a.q = q; a.q_stride = (size_t)q_stride; a.out = out; a.n_heads = n_heads; a.M = M; a.max_new = max_new; a.B = B; a.G = G;
  a.off = off; a.len = len; a.group = group; a.shared = shared; a.causal = causal != 0; a.scale = scale * (float)M_LOG2E; a.status = status;
  a.grid = s.grid; a.item_rows = dtype == AD_DTYPE_FP32 ? shr::M_ROWS : shr::ITEM_ROWS; a.part_rows = s.part_rows;
  a.total = reinterpret_cast<long long*>(at + s.total); a.lines = reinterpret_cast<shr::Line*>(at + s.lines); a.start = reinterpret_cast<shr::Start*>(at + s.start);
  a.ml = reinterpret_cast<float2*>(at + s.ml); a.part = reinterpret_cast<float*>(at + s.part);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const int dim = c->head_dim;
  cudaError_t e;
  if (dtype == AD_DTYPE_FP32) e = c->format == AD_CACHE_E4M3 ? launch_shared_dim<float, kv::E4m3>(dim, a, st) : launch_shared_dim<float, kv::Int8>(dim, a, st);
  else e = c->format == AD_CACHE_E4M3 ? launch_shared_dim<bf16, kv::E4m3>(dim, a, st) : launch_shared_dim<bf16, kv::Int8>(dim, a, st);
  return launched(entry, e);
}
