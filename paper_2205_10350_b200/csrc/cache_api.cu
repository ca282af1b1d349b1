// Operator-level entry points of the 8-bit key/value cache and of sampled verification, declared in include/aggressive_decoding.h.
#include <limits.h>
#include <math.h>

#include <algorithm>
#include <atomic>

#include "accept_sampled.cuh"
#include "ad_common.cuh"
#include "cache_attention.cuh"
#include "cache_checks.h"
#include "kv_cache.cuh"
#include "op_launch.h"

using namespace ad;

namespace {

template <typename T, typename F> struct Types { typedef T Num; typedef F Fmt; };
// Calls f with the number and code types of a call.
template <typename Fn>
cudaError_t by_types(int32_t dtype, int32_t format, Fn f) {
  if (dtype == AD_DTYPE_FP32) return format == AD_CACHE_E4M3 ? f(Types<float, kv::E4m3>()) : f(Types<float, kv::Int8>());
  return format == AD_CACHE_E4M3 ? f(Types<bf16, kv::E4m3>()) : f(Types<bf16, kv::Int8>());
}

// Heads' tiles that a CTA of ad_cache_append and ad_cache_read takes one after the other, by how often one tile a CTA would fill the GPU (768 threads an
// SM, what registers allow): four beyond eight times, two beyond two and a half, else one.  Appending, one / two / four: 1.7 times (32 rows x 9-64 tokens, 64 wide)
// 6.9 / 7.9 / 11.1 us, 3.4 times (128 wide) 12.6 / 12.1 / 13.3, 4.9 times (8 rows x 100-1000) 23.9 / 19.8 / 19.6, 37 times (8 prompts) 100 / 76 / 64.
int tiles_a_cta(const ad_kv_cache* c, int32_t B, int32_t max_new) {
  const int64_t threads = (int64_t)2 * c->n_kv_heads * ((max_new + c->block - 1) / c->block) * B * std::max(32, c->block * c->head_dim / (8 * kv::VECS));
  const int64_t filled = 768 * (int64_t)op_num_sms();
  return threads >= 8 * filled ? 4 : 2 * threads >= 5 * filled ? 2 : 1;
}
dim3 tile_grid(const ad_kv_cache* c, int32_t B, int32_t max_new, int tiles) {
  return dim3((2 * c->n_kv_heads + tiles - 1) / tiles, (max_new + c->block - 2) / c->block + 1, B);
}
dim3 tile_threads(const ad_kv_cache* c) { return dim3(std::max(32, c->block * c->head_dim / (8 * kv::VECS))); }
dim3 read_threads(const ad_kv_cache* c) { return dim3(std::max(32, c->block * c->head_dim / (16 * kv::READ_VECS))); }

}  // namespace

int ad::cache_append(const char* entry, const ad_kv_cache* c, const int32_t* refs, const void* k, const void* v, int32_t dtype, int64_t token_stride, const int32_t* off,
                     const int32_t* len, int32_t B, int32_t M, int32_t max_new, int32_t* status, void* stream) {
  if (const char* why = batch_fault(off, len, B, M, max_new)) return arg_fault(entry, why);
  if (const char* why = cache_fault(c, B)) return arg_fault(entry, why);
  if (!known_dtype(dtype)) return arg_fault(entry, "unknown dtype");
  if (M == 0) return AD_OK;
  if (!k || !v || !aligned(k, 16) || !aligned(v, 16)) return arg_fault(entry, "keys and values must be 16-byte aligned");
  if (token_stride < (int64_t)c->n_kv_heads * c->head_dim || token_stride % (int64_t)(16 / dtype_bytes(dtype)))
    return arg_fault(entry, "tokens must be a multiple of 16 bytes apart, and not overlap");
  const kv::Cache d = device_cache(c);
  const int tiles = tiles_a_cta(c, B, max_new);
  return launched(entry, by_types(dtype, c->format, [&](auto t) {
    typedef typename decltype(t)::Num T;
    auto kernel = refs ? kv::cache_append_kernel<T, typename decltype(t)::Fmt, true> : kv::cache_append_kernel<T, typename decltype(t)::Fmt, false>;
    return launch_op(kernel, tile_grid(c, B, max_new, tiles), tile_threads(c), dim3(), 0,
                     static_cast<cudaStream_t>(stream), d, refs, static_cast<const T*>(k), static_cast<const T*>(v), (size_t)token_stride,
                     (int)c->head_dim, off, len, (int)M, (int)max_new, tiles, status);
  }));
}

extern "C" int ad_cache_append(const ad_kv_cache* c, const void* k, const void* v, int32_t dtype, int64_t token_stride, const int32_t* off,
                               const int32_t* len, int32_t B, int32_t M, int32_t max_new, int32_t* status, void* stream) {
  return cache_append("ad_cache_append", c, nullptr, k, v, dtype, token_stride, off, len, B, M, max_new, status, stream);
}

extern "C" int ad_cache_read(const ad_kv_cache* c, void* k, void* v, int32_t dtype, const int32_t* off, const int32_t* start, int32_t B, int32_t M,
                             int32_t max_tokens, int32_t* status, void* stream) {
  const char* entry = "ad_cache_read";
  if (const char* why = batch_fault(off, start, B, M, max_tokens)) return arg_fault(entry, why);
  if (const char* why = cache_fault(c, B)) return arg_fault(entry, why);
  if (!known_dtype(dtype)) return arg_fault(entry, "unknown dtype");
  if (M == 0) return AD_OK;
  if (!k || !v || !aligned(k, 16) || !aligned(v, 16)) return arg_fault(entry, "keys and values must be 16-byte aligned");
  const kv::Cache d = device_cache(c);
  const int tiles = tiles_a_cta(c, B, max_tokens);
  return launched(entry, by_types(dtype, c->format, [&](auto t) {
    typedef typename decltype(t)::Num T;
    return launch_op(kv::cache_read_kernel<T, typename decltype(t)::Fmt>, tile_grid(c, B, max_tokens, tiles), read_threads(c), dim3(), 0,
                     static_cast<cudaStream_t>(stream), d, static_cast<T*>(k), static_cast<T*>(v), (int)c->head_dim, off, start, (int)M,
                     (int)max_tokens, tiles, status);
  }));
}

namespace {
// Units of 32 keys that one piece of a row's keys has, and what a tile of rows costs besides its keys, in units.  Measured, with another kernel between the
// calls: pieces of 4 / 8 / 16, one query on 2000 keys 10.4 / 12.4 / 17.3 us, two rows of 25 queries on 4000 24.6 / 20.6 / 20.6, 24 rows of one on 20000
// 129 / 129 / 134; 0 / 16 / 32 for the tile, 32 rows x 17-64 queries 178 / 122 / 125, two rows of 25 on 4000 20.7 / 20.6 / 24.7.
constexpr int kGranule = 8, kItemFixed = 16;
struct AttendPlan { int nq, row_tiles, grid, granule; bool shared; };
// max_keys, but no more than a row can hold (which leaves room for roundings below 2^31).
int32_t longest_row(const ad_kv_cache* c, int32_t max_keys) { return std::min(max_keys, c->table_stride * c->block); }
// Rows of queries a CTA takes: 8 or 16 where that is all there are, else 32, which make the most of a key's codes once they are FP16.  Keys that are
// too few to be split leave the GPU to as many CTAs as there are tiles of rows: then tiles are made smaller while all are resident at once
// (8 x 25 queries in FP32 over 400 keys, 8 heads: 14.4 -> 10.3 us).  So they are where rows may be long but are likely to be short (`own`: what is left of them behind a prefix that
// others share: 2 x 8 rows of 5 queries, 32 heads on 8, of 300 keys beside the prefix's work 87 -> 83 us; with one of 16000 among them 107 both ways).
AttendPlan attend_plan(const ad_kv_cache* c, int32_t n_heads, int32_t B, int32_t max_new, int32_t max_keys, bool own) {
  AttendPlan plan;
  max_keys = longest_row(c, max_keys);
  const int rows = max_new * (n_heads / c->n_kv_heads), pieces = std::max(1, (max_keys + kv::UNIT - 1) / kv::UNIT / kGranule);
  auto items = [&](int nq) { return (int64_t)B * c->n_kv_heads * ((rows + 8 * nq - 1) / (8 * nq)); };
  auto resident = [&](int nq) { return (int64_t)op_num_sms() * kv::att_resident(c->head_dim, nq); };
  plan.nq = rows <= 8 ? 1 : rows <= 16 ? 2 : 4;
  while ((own || pieces == 1) && plan.nq > 1 && items(plan.nq / 2) <= resident(plan.nq / 2)) plan.nq /= 2;
  plan.row_tiles = (rows + 8 * plan.nq - 1) / (8 * plan.nq);
  plan.granule = pieces > 1 ? kGranule : 0;
  plan.grid = (int)std::min(resident(plan.nq), std::min(resident(plan.nq), items(plan.nq)) * pieces);     // (items times pieces alone may pass 64 bits)
  // Whether the threads of a CTA of the join share a row's parts: from six CTAs a tile of rows on (single queries on 20000 keys, four rows, 14 CTAs a tile: 41.1 -> 34.8 us,
  // eight, 7: 53.4 -> 50.5); at two to five both take the same time, and with many rows shared ones are too many CTAs (32 x 17-64 queries 122 against 191).
  plan.shared = plan.grid > 6 * items(plan.nq);
  return plan;
}
// Scratch: granules in front of every row of the batch, then the parts (16-byte aligned).
size_t attend_prefix_bytes(int32_t B) { return ((size_t)B + 2) / 2 * 2 * sizeof(long long); }
size_t attend_part_bytes(const ad_kv_cache* c, const AttendPlan& plan, int32_t B) {
  return plan.granule == 0 ? 0 : 2 * (size_t)plan.grid * 8 * plan.nq * (c->head_dim + 2) * sizeof(float) + attend_prefix_bytes(B);
}
bool attend_sizes(const ad_kv_cache* c, int32_t n_heads, int32_t max_new) {
  return n_heads >= 1 && n_heads <= 65535 && n_heads % c->n_kv_heads == 0 && (int64_t)max_new * (n_heads / c->n_kv_heads) <= (1 << 24) && (int64_t)max_new * n_heads <= (1 << 30);
}

template <typename T, typename F, int DIM, int NQ, bool TWO>
cudaError_t launch_attention_part(const kv::AttendParams& a, cudaStream_t st) {
  static std::atomic<uint64_t> raised{0};              // devices on which the kernel may use its shared memory
  auto kernel = kv::cache_attention_kernel<T, F, DIM, NQ, TWO>;
  constexpr int smem = kv::att_smem(DIM, NQ, sizeof(T) == 4);
  const uint64_t bit = 1ull << op_device();
  if (!(raised.load(std::memory_order_relaxed) & bit)) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    raised.fetch_or(bit, std::memory_order_relaxed);
  }
  return launch_op(kernel, dim3(a.grid), dim3(32 * kv::ATT_WARPS), dim3(), smem, st, a);
}
template <typename T, int DIM, int NQ>
cudaError_t launch_join(const kv::AttendParams& a, const AttendPlan& plan, cudaStream_t st) {
  if (!a.granule) return cudaSuccess;
  const int rows = plan.row_tiles * 8 * NQ, groups = 512 / DIM;
  return plan.shared ? launch_op(kv::cache_attention_join_kernel<T, DIM, NQ, true>, dim3(rows, a.c.heads, a.B), dim3(128), dim3(), a.grid * sizeof(float), st, a)
                     : launch_op(kv::cache_attention_join_kernel<T, DIM, NQ, false>, dim3((rows + groups - 1) / groups, a.c.heads, a.B), dim3(128), dim3(), 0, st, a);
}
template <typename T, typename F, int DIM, int NQ>
cudaError_t launch_attention(const kv::AttendParams& a, const AttendPlan& plan, cudaStream_t st) {
  const cudaError_t e = a.c.block == 16 ? launch_attention_part<T, F, DIM, NQ, true>(a, st) : launch_attention_part<T, F, DIM, NQ, false>(a, st);
  return e == cudaSuccess && !a.mean ? launch_join<T, DIM, NQ>(a, plan, st) : e;
}
template <typename T, typename F, int DIM>
cudaError_t launch_attention_dim(const kv::AttendParams& a, const AttendPlan& plan, cudaStream_t st) {
  return plan.nq == 1 ? launch_attention<T, F, DIM, 1>(a, plan, st) : plan.nq == 2 ? launch_attention<T, F, DIM, 2>(a, plan, st) : launch_attention<T, F, DIM, 4>(a, plan, st);
}
}  // namespace

size_t ad::cache_attention_scratch(const ad_kv_cache* c, int n_heads, int B, int max_new, int max_keys, bool own) {
  return attend_part_bytes(c, attend_plan(c, n_heads, B, max_new, max_keys, own), B);
}
kv::Parts ad::cache_attention_parts(const ad_kv_cache* c, const AttentionCall& call, void* scratch) {
  const AttendPlan plan = attend_plan(c, call.n_heads, call.B, call.max_new, call.max_keys, call.mean);
  return kv::Parts{reinterpret_cast<float*>(static_cast<char*>(scratch) + attend_prefix_bytes(call.B)), static_cast<long long*>(scratch), plan.grid, 8 * plan.nq, kItemFixed, plan.granule};
}
cudaError_t ad::cache_attention(const ad_kv_cache* c, const AttentionCall& call, void* scratch, cudaStream_t st) {
  const AttendPlan plan = attend_plan(c, call.n_heads, call.B, call.max_new, call.max_keys, call.mean);
  kv::AttendParams a;
  a.c = device_cache(c); a.c.first = call.first;
  a.q = call.q; a.q_stride = (size_t)call.q_stride; a.out = call.out; a.n_heads = call.n_heads; a.M = call.M; a.max_new = call.max_new; a.off = call.off; a.len = call.len;
  a.causal = call.causal; a.scale = call.scale * (float)M_LOG2E; a.status = call.status; a.mean = call.mean; a.weight = call.weight; a.whole = call.whole;
  // More than half of L2 would not be there any more for the next call, and drives out what others keep there (1 x 200001 keys 104 -> 91 us); tiles of
  // the same row read one another's keys from L2.
  a.stream_once = plan.row_tiles == 1 && (double)call.B * longest_row(c, call.max_keys) * c->n_kv_heads * c->head_dim * 2 > (64 << 20);
  const kv::Parts parts = cache_attention_parts(c, call, scratch);
  a.B = call.B; a.grid = plan.grid; a.granule = plan.granule; a.fixed = kItemFixed; a.prefix = const_cast<long long*>(parts.prefix); a.part = const_cast<float*>(parts.part);
  return by_types(call.dtype, c->format, [&](auto t) {
    typedef typename decltype(t)::Num T;
    typedef typename decltype(t)::Fmt F;
    return c->head_dim == 32 ? launch_attention_dim<T, F, 32>(a, plan, st) : c->head_dim == 64 ? launch_attention_dim<T, F, 64>(a, plan, st)
                                                                                              : launch_attention_dim<T, F, 128>(a, plan, st);
  });
}

extern "C" size_t ad_cache_attention_scratch_bytes(const ad_kv_cache* c, int32_t dtype, int32_t n_heads, int32_t B, int32_t max_new, int32_t max_keys) {
  if (cache_fault(c, B) || B < 1 || max_new < 1 || max_keys < 0 || !known_dtype(dtype) || !attend_sizes(c, n_heads, max_new)) return 0;
  return cache_attention_scratch(c, n_heads, B, max_new, max_keys, false);
}

const char* ad::cache_attention_fault(const ad_kv_cache* c, const AttentionCall& call) {
  if (const char* why = batch_fault(call.off, call.len, call.B, call.M, call.max_new)) return why;
  if (const char* why = cache_fault(c, call.B)) return why;
  if (!known_dtype(call.dtype)) return "unknown dtype";
  if (!attend_sizes(c, call.n_heads, call.max_new)) return "query heads must be a multiple of the cache's, at most 65535, and max_new times their ratio at most 2^24 (times them, 2^30)";
  if (call.max_keys < 0) return "negative number of keys";
  if (!(call.scale > 0.f) || !(call.scale <= 1e30f)) return "the scale must be positive, and 1e30 at most";
  if (call.M == 0) return nullptr;
  if (!call.q || !call.out || !aligned(call.q, 16) || !aligned(call.out, 16)) return "queries and result must be 16-byte aligned";
  if (call.q_stride < (int64_t)call.n_heads * c->head_dim || call.q_stride % (int64_t)(16 / dtype_bytes(call.dtype)))
    return "queries must be a multiple of 16 bytes apart, and not overlap";
  return nullptr;
}

extern "C" int ad_cache_attention(const ad_kv_cache* c, const void* q, int32_t dtype, int64_t q_stride, int32_t n_heads, const int32_t* off,
                                  const int32_t* len, int32_t B, int32_t M, int32_t max_new, int32_t max_keys, int32_t causal, float scale, void* out,
                                  void* scratch, size_t scratch_bytes, int32_t* status, void* stream) {
  const char* entry = "ad_cache_attention";
  const AttentionCall call = {q, dtype, q_stride, n_heads, off, len, B, M, max_new, max_keys, causal != 0, scale, out, status, nullptr, nullptr, nullptr, nullptr};
  if (const char* why = cache_attention_fault(c, call)) return arg_fault(entry, why);
  if (M == 0) return AD_OK;
  const size_t need = cache_attention_scratch(c, n_heads, B, max_new, max_keys, false);
  if (scratch_bytes < need) return op_fail(AD_ERR_CAPACITY, entry, "scratch too small");
  if (need && (!scratch || !aligned(scratch, 256))) return arg_fault(entry, "scratch must be 256-byte aligned");
  return launched(entry, cache_attention(c, call, scratch, static_cast<cudaStream_t>(stream)));
}

namespace {
// Parts a row's scores are split into: four CTAs an SM where there are few rows, as long as every thread has a vector; at least so many that no
// thread adds up more than 32 vectors.  64 parts at most: the accept kernel's bound on the sums' errors counts on it.
constexpr int kMaxVocab = 1 << 20;
int score_parts(int32_t rows, int32_t vocab) {
  const int vecs = (vocab + 3) / 4;                                  // (FP32's; BF16 has half as many)
  const int least = (vecs + 32 * sampled::STAT_THREADS - 1) / (32 * sampled::STAT_THREADS);
  const int most = std::max(1, vecs / (2 * sampled::STAT_THREADS));
  const int fill = (4 * op_num_sms() - 1) / std::max(rows, 1) + 1;
  return std::max(least, std::min({most, fill, 64}));
}
}  // namespace

namespace {
// Weights stay in shared memory while there is room for them: up to 106496 ids with a drafter and 212992 without in clusters of eight CTAs, half of that in clusters of four.
constexpr size_t kKeptMax = 208 * 1024;
template <typename T, bool KEPT>
cudaError_t launch_accept_kept(const sampled::Params& p, int cluster, size_t smem, cudaStream_t st) {
  static std::atomic<uint64_t> raised{0};
  auto kernel = sampled::accept_sampled_kernel<T, KEPT>;
  const uint64_t bit = 1ull << op_device();
  if (KEPT && !(raised.load(std::memory_order_relaxed) & bit)) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kKeptMax);
    if (e != cudaSuccess) return e;
    raised.fetch_or(bit, std::memory_order_relaxed);
  }
  return launch_op(kernel, dim3(p.B * cluster), dim3(sampled::ACCEPT_THREADS), dim3(cluster), KEPT ? smem : 0, st, p);
}
template <typename T>
cudaError_t launch_accept(const sampled::Params& p, cudaStream_t st) {
  // (a CTA an SM: more rows share fewer CTAs each rather than wait for one another)
  const int cluster = p.vocab <= 2048 ? 1 : p.B * sampled::MAX_CLUSTER <= op_num_sms() ? sampled::MAX_CLUSTER : 4;
  const size_t each = (p.vocab + cluster * sampled::ACCEPT_THREADS - 1) / (cluster * sampled::ACCEPT_THREADS);
  const size_t smem = each * sampled::ACCEPT_THREADS * (p.score[1] ? 2 : 1) * sizeof(double);
  return smem <= kKeptMax ? launch_accept_kept<T, true>(p, cluster, smem, st) : launch_accept_kept<T, false>(p, cluster, smem, st);
}
}  // namespace

extern "C" size_t ad_accept_sampled_scratch_bytes(int32_t M, int32_t vocab, int32_t with_draft) {
  if (M < 0 || M > INT_MAX / 2 || vocab < 1 || vocab > kMaxVocab) return 0;
  const int z = with_draft ? 2 : 1;
  return (size_t)std::max(M, 1) * z * score_parts(M * z, vocab) * sizeof(sampled::Stat);
}

extern "C" int ad_accept_sampled(const void* target, int64_t target_stride, const void* draft, int64_t draft_stride, int32_t dtype, float temperature,
                                 int32_t vocab, const int32_t* off, const int32_t* drafts, int32_t kmax, int32_t B, int32_t M, const float* u,
                                 const float* r, int32_t eos, int32_t* tokens, int32_t* n_accepted, void* scratch, size_t scratch_bytes,
                                 int32_t* status, void* stream) {
  const char* entry = "ad_accept_sampled";
  if (!off || !drafts || !u || !r || !tokens || !n_accepted) return arg_fault(entry, "null argument");
  if (!known_dtype(dtype)) return arg_fault(entry, "unknown dtype");
  if (B < 1 || B > kMaxRows || kmax < 1 || kmax > kMaxNew || M < 0 || M > INT_MAX / 2 || vocab < 1 || vocab > kMaxVocab) return arg_fault(entry, "size out of range");
  if (!(temperature >= 1e-30f) || !(temperature < INFINITY)) return arg_fault(entry, "the temperature must be positive (1e-30 at least) and finite");
  if (M > 0 && !target) return arg_fault(entry, "null scores");
  if (!aligned(target, dtype_bytes(dtype)) || !aligned(draft, dtype_bytes(dtype))) return arg_fault(entry, "misaligned scores");
  if (target_stride < vocab || (draft && draft_stride < vocab)) return arg_fault(entry, "rows of scores overlap");
  if (scratch_bytes < ad_accept_sampled_scratch_bytes(M, vocab, draft != nullptr)) return op_fail(AD_ERR_CAPACITY, entry, "scratch too small");
  if (!scratch || !aligned(scratch, 256)) return arg_fault(entry, "scratch must be 256-byte aligned");
  sampled::Params p;
  p.score[0] = target; p.score[1] = M > 0 ? draft : nullptr; p.stride[0] = (size_t)target_stride; p.stride[1] = draft ? (size_t)draft_stride : 0;
  const int z = p.score[1] ? 2 : 1;
  p.vocab = vocab; p.parts = score_parts(M * z, vocab); p.M = M; p.B = B; p.kmax = kmax; p.eos = eos;
  p.inv_t = 1.0 / (double)temperature; p.c = (float)(M_LOG2E * p.inv_t);
  p.off = off; p.drafts = drafts; p.u = u; p.r = r; p.stats = static_cast<sampled::Stat*>(scratch); p.tokens = tokens; p.n_acc = n_accepted; p.status = status;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e = cudaSuccess;
  if (M > 0)
    e = launch_op(dtype == AD_DTYPE_BF16 ? sampled::score_stats_kernel<bf16> : sampled::score_stats_kernel<float>, dim3(M, p.parts, z),
                  dim3(sampled::STAT_THREADS), dim3(), 0, st, p);
  if (e == cudaSuccess) e = dtype == AD_DTYPE_BF16 ? launch_accept<bf16>(p, st) : launch_accept<float>(p, st);
  return launched(entry, e);
}
