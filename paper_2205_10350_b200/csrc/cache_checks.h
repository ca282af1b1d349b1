// Checks that the entry points around the 8-bit cache share: sizes, alignment, and how a refusal is told.
#pragma once

#include <limits.h>
#include <stdint.h>

#include "ad_common.cuh"
#include "kv_cache.cuh"
#include "op_launch.h"

namespace ad {

constexpr int kMaxNew = 1 << 19;       // tokens of a row in one call (grid dimensions)
constexpr int kMaxRows = 65535;

inline bool aligned(const void* p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }
inline bool known_dtype(int32_t t) { return t == AD_DTYPE_FP32 || t == AD_DTYPE_BF16; }
inline size_t dtype_bytes(int32_t t) { return t == AD_DTYPE_FP32 ? 4 : 2; }

// Why a cache cannot be worked on, or null.
inline const char* cache_fault(const ad_kv_cache* c, int32_t B) {
  if (!c || !c->k_codes || !c->v_codes || !c->k_scale || !c->v_scale) return "null cache";
  if (!aligned(c->k_codes, 16) || !aligned(c->v_codes, 16)) return "codes must be 16-byte aligned";
  if (c->format != AD_CACHE_E4M3 && c->format != AD_CACHE_INT8) return "unknown format";
  if (c->block != 16 && c->block != 32 && c->block != 64 && c->block != 128) return "blocks hold 16, 32, 64 or 128 tokens";
  if (c->head_dim != 32 && c->head_dim != 64 && c->head_dim != 128) return "heads are 32, 64 or 128 wide";
  if (c->n_blocks < 1 || c->n_kv_heads < 1 || c->n_kv_heads > 4096 || c->table_stride < 1) return "sizes must be positive (and at most 4096 heads)";
  if ((int64_t)c->table_stride * c->block > INT_MAX - kMaxNew) return "a row's capacity must stay below 2^31 - 2^19 tokens";
  if (!c->table && (int64_t)B * c->table_stride > c->n_blocks) return "without a table there must be B * table_stride blocks";
  return nullptr;
}

inline const char* batch_fault(const int32_t* off, const int32_t* len, int32_t B, int32_t M, int32_t max_new) {
  if (!off || !len) return "null offsets or lengths";
  if (B < 1 || B > kMaxRows) return "1 to 65535 rows";
  if (M < 0) return "negative number of tokens";
  if (max_new < 1 || max_new > kMaxNew) return "1 to 2^19 tokens of a row";
  return nullptr;
}

inline kv::Cache device_cache(const ad_kv_cache* c) {
  kv::Cache d;
  d.codes[0] = static_cast<uint8_t*>(c->k_codes); d.codes[1] = static_cast<uint8_t*>(c->v_codes);
  d.scale[0] = c->k_scale; d.scale[1] = c->v_scale;
  d.table = c->table; d.table_stride = c->table_stride; d.n_blocks = c->n_blocks; d.heads = c->n_kv_heads; d.block = c->block;
  return d;
}

// Whether what is left would be written over other scores than its own: M rows of `vocab` elements at a and at b.  It may take the place of the scores themselves, lie apart from them, or, with
// the same stride, between them: then b lies the same distance behind some row of a's in all rows, and overlaps neither that row nor the next.
inline bool rows_overlap(uintptr_t a, size_t stride_a, uintptr_t b, size_t stride_b, size_t vocab, size_t M, size_t element) {
  if (a >= b + ((M - 1) * stride_b + vocab) * element || b >= a + ((M - 1) * stride_a + vocab) * element) return false;
  if (M == 1 || stride_a != stride_b) return a != b || (M > 1 && stride_a != stride_b);
  if (a == b) return false;
  const size_t stride = stride_a * element, behind = b > a ? (b - a) % stride : (stride - (a - b) % stride) % stride;
  return behind < vocab * element || behind > stride - vocab * element;
}

inline int arg_fault(const char* entry, const char* why) { return op_fail(AD_ERR_ARG, entry, why); }
inline int launched(const char* entry, cudaError_t e) { return e == cudaSuccess ? AD_OK : op_fail(AD_ERR_CUDA, entry, cudaGetErrorString(e)); }

// The attention over a cache, as its entry point gets it, and as a part of others'.  first (null: none): blocks in front of what each row looks at.  mean and weight
// (null: results go to out): means of values [M, n_heads, head_dim], and maxima of the scores (times log2 e) and sums of exponentials [M, n_heads], of items that one CTA worked on; the
// others' parts are where cache_attention_parts says.  whole (null: no such word): not zero on the device, rows are not split, although max_keys would have it.
struct AttentionCall {
  const void* q;
  int32_t dtype;
  int64_t q_stride;
  int32_t n_heads;
  const int32_t *off, *len;
  int32_t B, M, max_new, max_keys;
  bool causal;
  float scale;
  void* out;
  int32_t* status;
  const int32_t* first;
  float* mean;
  float2* weight;
  const int32_t* whole;
};
// ad_cache_append for `entry`; refs: null, or counts by which rows that do not own what they would write are left out.
int cache_append(const char* entry, const ad_kv_cache* c, const int32_t* refs, const void* k, const void* v, int32_t dtype, int64_t token_stride, const int32_t* off,
                 const int32_t* len, int32_t B, int32_t M, int32_t max_new, int32_t* status, void* stream);
const char* cache_attention_fault(const ad_kv_cache* c, const AttentionCall& call);      // why it cannot be done, or null
size_t cache_attention_scratch(const ad_kv_cache* c, int n_heads, int B, int max_new, int max_keys, bool own);      // own: with call.mean
kv::Parts cache_attention_parts(const ad_kv_cache* c, const AttentionCall& call, void* scratch);
cudaError_t cache_attention(const ad_kv_cache* c, const AttentionCall& call, void* scratch, cudaStream_t st);

}  // namespace ad
