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

struct Scratch { size_t total, lines, start, first, len, ml, part, own_ml, own_part, rows, bytes; long long part_rows; int grid; };
// Results of the groups' items: of every query and head, and as much as an item's between the CTAs' parts, twice (either half of the keys); those of the rows' own
// positions; and what the attention row by row wants, which is planned for rows of max_keys of their own: groups need not share max_shared positions, nor any.  (Planned for max_keys - max_shared, a
// row of 32000 that shared nothing was not split beside 64 rows behind 32000: 729 us instead of 114, row by row 525.)  That no row is long after all is found out on the device, and nothing
// is split then.
Scratch scratch_of(const ad_kv_cache* c, int32_t n_heads, int32_t B, int32_t M, int32_t max_new, int32_t max_keys, int32_t G) {
  Scratch s;
  const size_t mh = (size_t)M * n_heads;
  s.grid = op_num_sms();
  s.part_rows = (long long)mh + (long long)s.grid * shr::ITEM_ROWS;
  s.total = 0;
  s.lines = 256;
  s.start = s.lines + rounded(((size_t)G + B) * sizeof(shr::Line));
  s.first = s.start + rounded(s.grid * sizeof(shr::Start));
  s.len = s.first + rounded(B * sizeof(int));
  s.ml = s.len + rounded(B * sizeof(int));
  s.part = s.ml + rounded(2 * (size_t)s.part_rows * sizeof(float2));
  s.own_ml = s.part + rounded(2 * (size_t)s.part_rows * c->head_dim * sizeof(float));
  s.own_part = s.own_ml + rounded(mh * sizeof(float2));
  s.rows = s.own_part + rounded(mh * c->head_dim * sizeof(float));
  s.bytes = s.rows + rounded(cache_attention_scratch(c, n_heads, B, max_new, max_keys, true));
  return s;
}
// Whether the groups' positions are read once for all rows.  Row by row they take units of 32 keys for 32 rows of queries and a key/value head; read once, a group's take about 1.9 rows' units.
// What that saves has to outweigh the plan, a second pass over the rows and the join: about 9000 units (12000 of 128 wide BF16, which the attention row by row takes less long for), ten for every row and
// key/value head, and 0.2 for every query and head, whose parts are written and read again.  Row by row / read once in us, own positions 20:
//   128 wide, 32 heads on 8, BF16: 16 rows of a query behind 4000 positions 44 / 41, 64 behind 1000 38 / 45, 8 behind 16000 62 / 47, 64 behind 16000 273 / 73, 4 behind 30000 58 / 57, 3 50 / 56, 2 38 / 56;
//   16 rows of 8 behind 4000 60 / 63, 8 groups of 16 of 8 behind 1000 130 / 133, 8 of 16 of 15 behind 330 105 / 189;
//   64 wide, 8 heads on 8: 64 rows of a query behind 1000 35 / 28, in FP32 40 / 30; 8 groups of 8 of 8 behind 1000 38 / 37, in FP32 42 / 39; 16 of 8 behind 4000 33 / 37, in FP32 37 / 38; 8 groups of 32
//   of a query behind 250 36 / 49, in FP32 41 / 50; 8 of 16 of 15 behind 330 27 / 56, in FP32 32 / 57; 4 of 2 of a query behind 14000 38 / 62; 16 heads, 8 of 2 of 4 behind 14000 100 / 170.
// Over 420 others, of 50 to 20000 positions, 1 to 8 groups of 2 to 64 rows and 1 to 25 queries, the choice takes 0.6 % longer than the faster side in the mean and 28 % at the most.
bool worth_sharing(const ad_kv_cache* c, int32_t dtype, int32_t n_heads, int32_t B, int32_t M, int32_t max_new, int32_t max_keys, int32_t G, int32_t max_shared) {
  const int64_t rows = (int64_t)max_new * (n_heads / c->n_kv_heads), keys = std::min<int64_t>(std::min(max_keys, max_shared), (int64_t)c->table_stride * c->block);
  const double saved = (B - 1.9 * G) * c->n_kv_heads * (double)((rows + 31) / 32) * (double)(keys / 32);
  return saved >= (dtype == AD_DTYPE_BF16 && c->head_dim == 128 ? 12000.0 : 9000.0) + 10.0 * B * c->n_kv_heads + 0.2 * M * (double)n_heads;
}
const char* shared_fault(int32_t n_heads, int32_t B, int32_t M, int32_t G, int32_t max_shared) {
  if (B < 1 || B > kSharedRows) return "1 to 8192 rows";
  if (G < 1 || G > B) return "1 to as many groups as rows";
  if (M < 0 || n_heads < 1 || (int64_t)M * n_heads > (1 << 30)) return "tokens times query heads may be 2^30 at most";
  if (max_shared < 0) return "negative number of shared positions";
  return nullptr;
}

// rows(): the attention row by row over what the groups do not share.
template <typename T, typename F, int DIM, typename Rows>
cudaError_t launch_shared(const shr::Params& a, cudaStream_t st, Rows rows) {
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
  if (e == cudaSuccess) e = rows();
  if (e == cudaSuccess) e = launch_op(kernel, dim3(a.grid), dim3(shr::THREADS), dim3(), smem, st, a);
  const long long warps = (long long)a.max_new * a.n_heads, each = shr::JOIN_THREADS / 32;
  if (e == cudaSuccess) e = launch_op(shr::shared_join_kernel<T, DIM>, dim3((unsigned)((warps + each - 1) / each), a.B), dim3(shr::JOIN_THREADS), dim3(), 0, st, a);
  return e;
}
template <typename T, typename F, typename Rows>
cudaError_t launch_shared_dim(int dim, const shr::Params& a, cudaStream_t st, Rows rows) {
  return dim == 32 ? launch_shared<T, F, 32>(a, st, rows) : dim == 64 ? launch_shared<T, F, 64>(a, st, rows) : launch_shared<T, F, 128>(a, st, rows);
}

}  // namespace

extern "C" size_t ad_cache_attention_shared_scratch_bytes(const ad_kv_cache* c, int32_t dtype, int32_t n_heads, int32_t B, int32_t M, int32_t max_new,
                                                          int32_t max_keys, int32_t G, int32_t max_shared) {
  if (shared_fault(n_heads, B, M, G, max_shared)) return 0;
  const size_t alone = ad_cache_attention_scratch_bytes(c, dtype, n_heads, B, max_new, max_keys);
  if (cache_fault(c, B) || !known_dtype(dtype) || max_new < 1 || max_keys < 0 || n_heads % c->n_kv_heads) return 0;
  return worth_sharing(c, dtype, n_heads, B, M, max_new, max_keys, G, max_shared) ? scratch_of(c, n_heads, B, M, max_new, max_keys, G).bytes : alone;
}

extern "C" int ad_cache_attention_shared(const ad_kv_cache* c, const void* q, int32_t dtype, int64_t q_stride, int32_t n_heads, const int32_t* off,
                                         const int32_t* len, int32_t B, int32_t M, int32_t max_new, int32_t max_keys, const int32_t* group,
                                         const int32_t* shared, int32_t G, int32_t max_shared, int32_t causal, float scale, void* out, void* scratch,
                                         size_t scratch_bytes, int32_t* status, void* stream) {
  const char* entry = "ad_cache_attention_shared";
  AttentionCall call = {q, dtype, q_stride, n_heads, off, len, B, M, max_new, max_keys, causal != 0, scale, out, status, nullptr, nullptr, nullptr, nullptr};
  if (const char* why = cache_attention_fault(c, call)) return arg_fault(entry, why);
  if (!group || !shared) return arg_fault(entry, "null groups");
  if (const char* why = shared_fault(n_heads, B, M, G, max_shared)) return arg_fault(entry, why);
  if (M == 0) return AD_OK;
  const size_t need = ad_cache_attention_shared_scratch_bytes(c, dtype, n_heads, B, M, max_new, max_keys, G, max_shared);
  if (scratch_bytes < need) return op_fail(AD_ERR_CAPACITY, entry, "scratch too small");
  if (need && (!scratch || !aligned(scratch, 256))) return arg_fault(entry, "scratch must be 256-byte aligned");
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (!worth_sharing(c, dtype, n_heads, B, M, max_new, max_keys, G, max_shared)) return launched(entry, cache_attention(c, call, scratch, st));
  const Scratch s = scratch_of(c, n_heads, B, M, max_new, max_keys, G);
  char* at = static_cast<char*>(scratch);
  shr::Params a = {};
  a.c = device_cache(c); a.q = q; a.q_stride = (size_t)q_stride; a.out = out; a.n_heads = n_heads; a.M = M; a.max_new = max_new; a.B = B; a.G = G;
  a.off = off; a.len = len; a.group = group; a.shared = shared; a.causal = causal != 0; a.scale = scale * (float)M_LOG2E; a.status = status;
  a.grid = s.grid; a.item_rows = dtype == AD_DTYPE_FP32 ? shr::M_ROWS : shr::ITEM_ROWS; a.part_rows = s.part_rows;
  a.total = reinterpret_cast<shr::Total*>(at + s.total); a.lines = reinterpret_cast<shr::Line*>(at + s.lines); a.start = reinterpret_cast<shr::Start*>(at + s.start);
  a.own_first = reinterpret_cast<int*>(at + s.first); a.own_len = reinterpret_cast<int*>(at + s.len);
  a.ml = reinterpret_cast<float2*>(at + s.ml); a.part = reinterpret_cast<float*>(at + s.part);
  a.own_ml = reinterpret_cast<float2*>(at + s.own_ml); a.own_part = reinterpret_cast<float*>(at + s.own_part);
  call.first = a.own_first; call.len = a.own_len; call.mean = a.own_part; call.weight = a.own_ml; call.whole = &a.total->own_whole;
  a.own = cache_attention_parts(c, call, at + s.rows);
  auto rows = [&] { return cache_attention(c, call, at + s.rows, st); };
  const int dim = c->head_dim;
  cudaError_t e;
  if (dtype == AD_DTYPE_FP32) e = c->format == AD_CACHE_E4M3 ? launch_shared_dim<float, kv::E4m3>(dim, a, st, rows) : launch_shared_dim<float, kv::Int8>(dim, a, st, rows);
  else e = c->format == AD_CACHE_E4M3 ? launch_shared_dim<bf16, kv::E4m3>(dim, a, st, rows) : launch_shared_dim<bf16, kv::Int8>(dim, a, st, rows);
  return launched(entry, e);
}
