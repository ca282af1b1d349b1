// Operator-level entry points of a pool of cache blocks and of filtered sampling, declared in include/aggressive_decoding.h.
#include <algorithm>
#include <atomic>

#include "block_pool.cuh"
#include "cache_checks.h"
#include "sample.cuh"

using namespace ad;

namespace {

constexpr int kPoolRows = 8192;        // (a column of the table, all rows, lies in a CTA's shared memory)
constexpr int kPoolBlocks = (1 << 30) - 512;      // (the planning kernels look up to 256 blocks beyond the last one, and keep as many holes and movers behind one another, in 32 bits)

const char* pool_fault(const ad_kv_pool* p, int32_t B) {
  if (!p || !p->table || !p->refs) return "null pool";
  if (p->block != 16 && p->block != 32 && p->block != 64 && p->block != 128) return "blocks hold 16, 32, 64 or 128 tokens";
  if (p->n_blocks < 1 || p->table_stride < 1 || p->rows < 1 || p->rows > kPoolRows) return "sizes must be positive (and at most 8192 rows)";
  if (p->n_blocks > kPoolBlocks) return "a pool has 2^30 - 512 blocks at most";
  if ((int64_t)p->table_stride * p->block > INT_MAX - kMaxNew) return "a row's capacity must stay below 2^31 - 2^19 tokens";
  if ((int64_t)p->table_stride * p->rows > INT_MAX) return "the table must have fewer than 2^31 entries";
  if (B < 1 || B > p->rows) return "a batch has 1 row to as many as the pool";
  return nullptr;
}
const char* layers_fault(const ad_kv_pool* p, const ad_kv_cache* caches, int32_t n) {
  if (n < 0 || n > pool::MAX_LAYERS) return "0 to 64 caches";
  if (n && !caches) return "null caches";
  for (int i = 0; i < n; ++i) {
    if (const char* why = cache_fault(caches + i, 1)) return why;
    if (caches[i].table != p->table || caches[i].table_stride != p->table_stride || caches[i].n_blocks != p->n_blocks || caches[i].block != p->block)
      return "caches must have the pool's table, blocks and block size";
    for (int j = 0; j < i; ++j)
      if (caches[j].k_codes == caches[i].k_codes || caches[j].v_codes == caches[i].v_codes) return "a cache is given twice";
  }
  return nullptr;
}

pool::Pool device_pool(const ad_kv_pool* p) { return pool::Pool{p->table, p->refs, p->rows, p->table_stride, p->n_blocks, p->block}; }

// CTAs of a planning kernel's cluster: one while its 32 warps have a row and a few loads of counts each at most, as every barrier of a cluster costs more.
int plan_cluster(int32_t n_blocks, int32_t B) { return n_blocks <= 8192 && B <= 32 ? 1 : pool::MAX_CLUSTER; }

// Threads of a planning kernel's CTA: a few warps where that leaves them a row and a load of counts each, as more of them take longer to start and to meet (8 rows, fork and
// reserve: 17.1 us with 1024 threads, 16.3 with 256; with a compaction between them 28.3 and 26.8).
int plan_threads(int32_t n_blocks, int32_t B) { return n_blocks <= 2048 && B <= 8 ? 256 : pool::PLAN_THREADS; }

size_t rounded(size_t bytes) { return (bytes + 255) / 256 * 256; }

pool::Contents contents_of(const ad_kv_pool* p, const ad_kv_cache* caches, int32_t n, const pool::Move* moves, const int* n_moves, int count) {
  pool::Contents c = {};
  for (int i = 0; i < n; ++i) {
    c.layer[i].codes[0] = static_cast<uint8_t*>(caches[i].k_codes); c.layer[i].codes[1] = static_cast<uint8_t*>(caches[i].v_codes);
    c.layer[i].scale[0] = caches[i].k_scale; c.layer[i].scale[1] = caches[i].v_scale;
    c.layer[i].heads = caches[i].n_kv_heads; c.layer[i].dim = caches[i].head_dim;
  }
  c.n_layers = n; c.moves = moves; c.n_moves = n_moves; c.n = count; c.block = p->block; c.n_blocks = p->n_blocks;
  return c;
}
// CTAs a layer that do at most `moves` moves: as many as there are heads' keys and values for their warps, in all layers together eight an SM at most.
int move_ctas(const ad_kv_cache* caches, int32_t n, int64_t moves) {
  int heads = 1;
  for (int i = 0; i < n; ++i) heads = std::max(heads, (int)caches[i].n_kv_heads);
  const int64_t warps = pool::COPY_THREADS / 32, ctas = (moves * 2 * heads + warps - 1) / warps;
  return (int)std::max<int64_t>(1, std::min<int64_t>(ctas, (8 * op_num_sms() + n - 1) / std::max(n, 1)));
}

}  // namespace

extern "C" int ad_cache_fork(const ad_kv_pool* p, const int32_t* parent, const int32_t* len, int32_t B, int32_t* status, void* stream) {
  const char* entry = "ad_cache_fork";
  if (const char* why = pool_fault(p, B)) return arg_fault(entry, why);
  if (!parent || !len) return arg_fault(entry, "null parents or lengths");
  // Columns a CTA: 32 (a sector and more of every row) while they fit in 48 KB and there are CTAs for all SMs, down to 8, a sector.
  int shift = 5;
  while (shift > 0 && ((int64_t)B << shift) * (int64_t)sizeof(int) > 48 * 1024) --shift;
  while (shift > 3 && (p->table_stride + (1 << shift) - 1) >> shift < op_num_sms()) --shift;
  return launched(entry, launch_op(pool::cache_fork_kernel, dim3((p->table_stride + (1 << shift) - 1) >> shift), dim3(pool::FORK_THREADS), dim3(),
                                   ((size_t)B << shift) * sizeof(int), static_cast<cudaStream_t>(stream), device_pool(p), parent, len, (int)B, shift, status));
}

extern "C" size_t ad_cache_reserve_scratch_bytes(const ad_kv_pool* p, int32_t B) {
  if (pool_fault(p, B)) return 0;
  return rounded((size_t)p->n_blocks * sizeof(int2)) + rounded((size_t)p->n_blocks * sizeof(int)) + rounded((size_t)B * sizeof(pool::Move));
}

extern "C" int ad_cache_reserve(const ad_kv_pool* p, const ad_kv_cache* caches, int32_t n_caches, const int32_t* off, const int32_t* len, int32_t B,
                                void* scratch, size_t scratch_bytes, int32_t* status, void* stream) {
  const char* entry = "ad_cache_reserve";
  if (const char* why = pool_fault(p, B)) return arg_fault(entry, why);
  if (const char* why = layers_fault(p, caches, n_caches)) return arg_fault(entry, why);
  if (!off || !len) return arg_fault(entry, "null offsets or lengths");
  if (scratch_bytes < ad_cache_reserve_scratch_bytes(p, B)) return op_fail(AD_ERR_CAPACITY, entry, "scratch too small");
  if (!scratch || !aligned(scratch, 256)) return arg_fault(entry, "scratch must be 256-byte aligned");
  char* at = static_cast<char*>(scratch);
  pool::Plan plan = {};
  plan.p = device_pool(p);
  plan.claim = reinterpret_cast<int2*>(at);
  at += rounded((size_t)p->n_blocks * sizeof(int2));
  plan.list = reinterpret_cast<int*>(at);
  at += rounded((size_t)p->n_blocks * sizeof(int));
  plan.moves = reinterpret_cast<pool::Move*>(at);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const int cluster = plan_cluster(p->n_blocks, B);
  cudaError_t e = launch_op(pool::cache_reserve_kernel, dim3(cluster), dim3(plan_threads(p->n_blocks, B)), dim3(cluster), 0, st, plan, off, len, (int)B, status);
  if (e == cudaSuccess && n_caches > 0)
    e = launch_op(pool::cache_move_kernel, dim3(move_ctas(caches, n_caches, B), n_caches), dim3(pool::COPY_THREADS), dim3(), 0, st,
                  contents_of(p, caches, n_caches, plan.moves, nullptr, B));
  return launched(entry, e);
}

extern "C" int ad_cache_append_pooled(const ad_kv_pool* p, const ad_kv_cache* c, const void* k, const void* v, int32_t dtype, int64_t token_stride,
                                      const int32_t* off, const int32_t* len, int32_t B, int32_t M, int32_t max_new, int32_t* status, void* stream) {
  const char* entry = "ad_cache_append_pooled";
  if (const char* why = pool_fault(p, B)) return arg_fault(entry, why);
  if (const char* why = layers_fault(p, c, 1)) return arg_fault(entry, why);
  return cache_append(entry, c, p->refs, k, v, dtype, token_stride, off, len, B, M, max_new, status, stream);
}

extern "C" size_t ad_cache_compact_scratch_bytes(const ad_kv_pool* p) {
  if (pool_fault(p, 1)) return 0;
  return rounded(2 * (size_t)p->n_blocks * sizeof(int)) + rounded((size_t)p->n_blocks * sizeof(int)) + rounded(sizeof(int)) +
         rounded((size_t)(p->n_blocks / 2 + 1) * sizeof(pool::Move));
}

extern "C" int ad_cache_compact(const ad_kv_pool* p, const ad_kv_cache* caches, int32_t n_caches, int32_t* n_used, void* scratch, size_t scratch_bytes,
                                void* stream) {
  const char* entry = "ad_cache_compact";
  if (const char* why = pool_fault(p, 1)) return arg_fault(entry, why);
  if (const char* why = layers_fault(p, caches, n_caches)) return arg_fault(entry, why);
  if (!n_used) return arg_fault(entry, "nowhere to put the number of blocks in use");
  if (scratch_bytes < ad_cache_compact_scratch_bytes(p)) return op_fail(AD_ERR_CAPACITY, entry, "scratch too small");
  if (!scratch || !aligned(scratch, 256)) return arg_fault(entry, "scratch must be 256-byte aligned");
  char* at = static_cast<char*>(scratch);
  pool::Plan plan = {};
  plan.p = device_pool(p);
  plan.list = reinterpret_cast<int*>(at);
  at += rounded(2 * (size_t)p->n_blocks * sizeof(int));
  plan.map = reinterpret_cast<int*>(at);
  at += rounded((size_t)p->n_blocks * sizeof(int));
  plan.n_moves = reinterpret_cast<int*>(at);
  at += rounded(sizeof(int));
  plan.moves = reinterpret_cast<pool::Move*>(at);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const int cluster = plan_cluster(p->n_blocks, 1);
  cudaError_t e = launch_op(pool::cache_compact_kernel, dim3(cluster), dim3(plan_threads(p->n_blocks, 1)), dim3(cluster), 0, st, plan, n_used);
  if (e == cudaSuccess) {
    pool::Contents c = contents_of(p, caches, n_caches, plan.moves, plan.n_moves, 0);
    c.table = p->table; c.entries = (long long)p->rows * p->table_stride; c.map = plan.map; c.n_used = n_used;
    e = launch_op(pool::cache_move_kernel, dim3(move_ctas(caches, n_caches, p->n_blocks / 2), n_caches + 1), dim3(pool::COPY_THREADS), dim3(), 0, st, c);
  }
  return launched(entry, e);
}

namespace {
constexpr int kSampleVocab = 1 << 20;
constexpr size_t kScoresKept = 188 * 1024;       // (beside the histogram and the list)
// Scores of a warp: vectors for all of its lanes, and room for one that begins in front of the row.
int scores_each(int32_t vocab, int cluster, size_t element) {
  const int64_t round = 32 * 16 / (int64_t)element, warps = (int64_t)cluster * sample::WARPS;
  return (int)((vocab + 16 / (int64_t)element + warps * round - 1) / (warps * round) * round);
}
// CTAs that share a row.  One up to 12 KB of scores, which eight take no sooner (a turn of a CTA costs as much as 40 KB of scores, of a cluster more).  Eight, or four, while all rows are under way at once
// with them.  Beyond that as few as keep a row in half an SM, one or two, so that there are two CTAs an SM and few turns; four where two cannot.  Measured with 1 / 2 / 4 / 8, us, scores from memory
// where they are 8 MB and more:
//   few rows, top-p: 1 x 3000 FP32 13.4 / 14.5 / 14.0 / 14.4; 1 x 32000 48 / 35 / 24 / 20; 64 x 32000 54 / 43 / 32 / 47; 1 x 128000 BF16 106 / 50 / 37 / 26; 64 x 128000 143 / 62 / 55 / 71
//   many: 512 x 3000 FP32, top-p 31 / 61 / 113 / 232; 256 x 16384 50 / 67 / 94 / 162; 256 x 32000 113 / 94 / 117 / 177; BF16 256 x 32000 53 / 68 / 98 / 211, 256 x 50265 100 / 92 / 130 / 196;
//   256 x 128000, filters row by row and what is left, 193 / 185 / 158 / 218
// Over 1352 such, of 500 to 160000 ids and 1 to 512 rows, the choice takes 4 % longer than the best of the four in the mean (eight or four from 2048 ids on: 24 %), and at the most twice as long: 512 x
// 80000 FP32, top-k and top-p, 188 / 254 / 368 / 331.  A row's result is the same for all.
int sample_cluster(int32_t M, int32_t vocab, size_t element) {
  if ((size_t)vocab * element <= 12 * 1024) return 1;
  const int64_t slots = 2 * (int64_t)op_num_sms();
  for (int c = sample::MAX_CLUSTER; c >= 4; c /= 2)
    if ((int64_t)M * c <= slots) return c;
  for (int c = 1; c <= 2; ++c)
    if ((size_t)scores_each(vocab, c, element) * sample::WARPS * element <= 76 * 1024) return c;
  return 4;
}
template <typename T, bool KEPT>
cudaError_t launch_sample_kept(const sample::Params& p, int cluster, size_t smem, cudaStream_t st) {
  static std::atomic<uint64_t> raised{0};
  auto kernel = sample::sample_kernel<T, KEPT>;
  const uint64_t bit = 1ull << op_device();
  if (KEPT && !(raised.load(std::memory_order_relaxed) & bit)) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kScoresKept);
    if (e != cudaSuccess) return e;
    raised.fetch_or(bit, std::memory_order_relaxed);
  }
  return launch_op(kernel, dim3(p.M * cluster), dim3(sample::THREADS), dim3(cluster), KEPT ? smem : 0, st, p);
}
template <typename T>
cudaError_t launch_sample(sample::Params p, cudaStream_t st) {
  const int cluster = sample_cluster(p.M, p.vocab, sizeof(T));
  p.each = scores_each(p.vocab, cluster, sizeof(T));
  const size_t smem = (size_t)p.each * sample::WARPS * sizeof(T);
  return smem <= kScoresKept ? launch_sample_kept<T, true>(p, cluster, smem, st) : launch_sample_kept<T, false>(p, cluster, smem, st);
}
}  // namespace

extern "C" int ad_sample(const void* scores, int64_t stride, int32_t dtype, int32_t vocab, int32_t M, const float* temperature, const int32_t* top_k,
                         const float* top_p, const float* min_p, const float* r, int32_t* tokens, float* logp, void* filtered, int64_t filtered_stride,
                         int32_t* status, void* stream) {
  const char* entry = "ad_sample";
  if (!known_dtype(dtype)) return arg_fault(entry, "unknown dtype");
  if (M < 0 || M > INT_MAX / sample::MAX_CLUSTER || vocab < 1 || vocab > kSampleVocab) return arg_fault(entry, "size out of range");
  if (M == 0) return AD_OK;
  if (!scores || !r || !tokens) return arg_fault(entry, "null argument");
  const size_t element = dtype_bytes(dtype);
  if (!aligned(scores, element) || !aligned(filtered, element)) return arg_fault(entry, "misaligned scores");
  if (stride < vocab || (filtered && filtered_stride < vocab)) return arg_fault(entry, "rows of scores overlap");
  if (filtered && rows_overlap(reinterpret_cast<uintptr_t>(scores), (size_t)stride, reinterpret_cast<uintptr_t>(filtered), (size_t)filtered_stride, (size_t)vocab, (size_t)M, element))
    return arg_fault(entry, "scores and what is left of them overlap");
  sample::Params p = {};
  p.scores = scores; p.stride = (size_t)stride; p.vocab = vocab; p.M = M; p.temperature = temperature; p.top_k = top_k; p.top_p = top_p; p.min_p = min_p; p.r = r;
  p.tokens = tokens; p.logp = logp; p.out = filtered; p.out_stride = (size_t)filtered_stride; p.status = status;
  p.scale_bits = 51;                               // (a weight in the bits of a double, and sums below 2^62)
  while ((1ll << (62 - p.scale_bits)) < vocab) --p.scale_bits;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return launched(entry, dtype == AD_DTYPE_BF16 ? launch_sample<bf16>(p, st) : launch_sample<float>(p, st));
}
