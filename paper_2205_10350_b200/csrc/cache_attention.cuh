// Attention of the tokens of a block over the 8-bit key/value cache (kv_cache.cuh).
#pragma once

#include "kv_cache.cuh"

namespace ad {
namespace kv {

struct AttendParams {
  Cache c;
  const void* q;           // [M, n_heads, dim], rows q_stride elements apart
  size_t q_stride;
  void* out;               // [M, n_heads, dim]
  int n_heads, M, max_new;
  const int* off;          // [B + 1]
  const int* len;          // [B]
  int causal;
  float scale;             // softmax scale times log2(e)
  int* status;
};

// One warp per query and head: lanes share the head's numbers, keys one after the other, running maximum and sum of the softmax in FP32.
// grid = (n_heads, max_new, B), block = 32.
template <typename T, typename F, int DIM>
__global__ void __launch_bounds__(32)
cache_attention_kernel(AttendParams a) {
  constexpr int PER = DIM / 32;
  pdl_launch();
  pdl_wait();
  const int b = blockIdx.z, i = blockIdx.y, head = blockIdx.x, lane = threadIdx.x;
  int o, n, p;
  if (!row_tokens(a.c, a.off, a.len, b, a.M, a.max_new, !a.causal, a.status, o, n, p) || i >= n) return;
  const int keys = a.causal ? p + i + 1 : p, kvh = head / (a.n_heads / a.c.heads);
  const T* q = static_cast<const T*>(a.q) + (size_t)(o + i) * a.q_stride + (size_t)head * DIM + lane * PER;
  T* out = static_cast<T*>(a.out) + ((size_t)(o + i) * a.n_heads + head) * DIM + lane * PER;
  float qv[PER], acc[PER], m = -INFINITY, sum = 0.f;
#pragma unroll
  for (int j = 0; j < PER; ++j) { qv[j] = to_f32(q[j]); acc[j] = 0.f; }
  for (int j0 = 0; j0 < keys; j0 += a.c.block) {
    const int id = a.c.find(b, j0 / a.c.block);
    if (id < 0) { latch_error(a.status, AD_ERR_ARG); continue; }
    const size_t tile = (size_t)id * a.c.heads + kvh;
    const float ks = a.c.scale[0][tile], vs = a.c.scale[1][tile];
    for (int t = 0; t < a.c.block && j0 + t < keys; ++t) {
      const uint8_t* kc = a.c.codes[0] + (tile * a.c.block + t) * DIM + lane * PER;
      const uint8_t* vc = a.c.codes[1] + (tile * a.c.block + t) * DIM + lane * PER;
      float kx[4], vx[4], s = 0.f;
      uint32_t kw = 0, vw = 0;
#pragma unroll
      for (int j = 0; j < PER; ++j) { kw |= (uint32_t)kc[j] << (8 * j); vw |= (uint32_t)vc[j] << (8 * j); }
      F::decode4(kw, kx);
      F::decode4(vw, vx);
#pragma unroll
      for (int j = 0; j < PER; ++j) s += qv[j] * kx[j];
#pragma unroll
      for (int w = 16; w; w >>= 1) s += __shfl_xor_sync(0xffffffffu, s, w);
      s *= ks * a.scale;
      const float top = fmaxf(m, s);
      const float keep = m == top ? 1.f : exp2f(m - top), e = exp2f(s - top);
      m = top;
      sum = sum * keep + e;
#pragma unroll
      for (int j = 0; j < PER; ++j) acc[j] = acc[j] * keep + e * (vs * vx[j]);
    }
  }
  const float inv = keys ? 1.f / sum : 0.f;
#pragma unroll
  for (int j = 0; j < PER; ++j) out[j] = from_f32<T>(acc[j] * inv);
}

}  // namespace kv
}  // namespace ad
