// Key/value cache in 8 bits with one scale per block of tokens and head: writing the tokens of a block into it and reading tokens back.
#pragma once

#include <cuda_fp16.h>
#include <float.h>
#include <limits.h>

#include "ad_common.cuh"

namespace ad {
namespace kv {

// Codes, four at a time: `encode4` rounds to nearest, ties to even, and saturates; `decode4` is exact.
struct E4m3 {
  static constexpr float TOP = 448.f;
  static __device__ __forceinline__ uint32_t encode4(const float* x) {
    uint32_t w;
    asm("{ .reg .b16 l, h; cvt.rn.satfinite.e4m3x2.f32 l, %2, %1; cvt.rn.satfinite.e4m3x2.f32 h, %4, %3; mov.b32 %0, {l, h}; }"
        : "=r"(w) : "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]));
    return w;
  }
  static __device__ __forceinline__ void decode4(uint32_t w, float* x) {
    uint32_t a, b;
    asm("{ .reg .b16 l, h; mov.b32 {l, h}, %2; cvt.rn.f16x2.e4m3x2 %0, l; cvt.rn.f16x2.e4m3x2 %1, h; }" : "=r"(a), "=r"(b) : "r"(w));
    const float2 p = __half22float2(*reinterpret_cast<__half2*>(&a)), q = __half22float2(*reinterpret_cast<__half2*>(&b));
    x[0] = p.x; x[1] = p.y; x[2] = q.x; x[3] = q.y;
  }
};
struct Int8 {
  static constexpr float TOP = 127.f;
  static __device__ __forceinline__ uint32_t encode4(const float* x) {
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) w |= (uint32_t)(uint8_t)(int8_t)__float2int_rn(fminf(fmaxf(x[i], -TOP), TOP)) << (8 * i);
    return w;
  }
  static __device__ __forceinline__ void decode4(uint32_t w, float* x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = (float)(int8_t)(w >> (8 * i));
  }
};

// The smallest power of two s with amax / s <= TOP (2^-126 at least; 1 where there is nothing but zeros).  TOP = 1.75 * 2^8 or 1.984375 * 2^6:
// with amax = f * 2^e, 1 <= f < 2, s is 2^(e - 8) or 2^(e - 6) while f is within TOP's mantissa and twice that beyond it.
template <typename F>
__device__ __forceinline__ float block_scale(float amax) {
  if (amax == 0.f) return 1.f;
  const uint32_t top = __float_as_uint(F::TOP), a = __float_as_uint(amax);
  const int e = (int)(a >> 23) - (int)(top >> 23) + ((a & 0x7fffffu) > (top & 0x7fffffu) ? 1 : 0);
  return __uint_as_float((uint32_t)max(e + 127, 1) << 23);             // (a subnormal amax has a >> 23 == 0: the smallest scale)
}

struct Cache {
  uint8_t* codes[2];             // keys, values: [n_blocks, heads, block, dim]
  float* scale[2];               // [n_blocks, heads]
  const int* table;              // [B, table_stride] or null
  int table_stride, n_blocks, heads, block;
  const int* first = nullptr;    // [B] blocks of the row in front of its block 0, or null
  // block i of row b; negative when the table names none that exists
  __host__ __device__ __forceinline__ int find(int b, int i) const {
    if (first) i += first[b];
    const int id = table ? table[(size_t)b * table_stride + i] : b * table_stride + i;
    return (unsigned)id < (unsigned)n_blocks ? id : -1;
  }
};

// Where the attention leaves parts of items that more than one CTA worked on.
struct Parts {
  const float* part;             // [2 grid][tile rows][dim] means of values, then [2 grid][tile rows] maxima and sums of exponentials
  const long long* prefix;       // [B + 1] granules in front of each row of the batch
  int grid, tile_rows, fixed, granule;
};

// Whether a row's n tokens o .. o + n - 1 of M can go to positions p .. of it (in_row = n), or look at its first p (in_row = 0): AD_OK or what is wrong.
__host__ __device__ __forceinline__ int row_fault(const Cache& c, int o, int n, int p, int M, int max_new, int in_row) {
  if (o < 0 || n < 0 || n > max_new || o > M - n || p < 0) return AD_ERR_ARG;
  return p > c.table_stride * c.block - in_row ? AD_ERR_CAPACITY : AD_OK;
}
// The tokens off[b] .. off[b + 1] of row b, in the row from position len[b] on or (outside) only looking at it.  False: nothing to do; what cannot be
// done is latched.
__device__ __forceinline__ bool row_tokens(const Cache& c, const int* off, const int* len, int b, int M, int max_new, bool outside, int* status, int& o,
                                           int& n, int& p) {
  o = __ldcg(off + b);
  const long long d = (long long)__ldcg(off + b + 1) - o;
  n = d < -1 || d > INT_MAX ? -1 : (int)d;
  p = __ldcg(len + b);
  if (n == 0) return false;
  const int fault = row_fault(c, o, n, p, M, max_new, outside ? 0 : n);
  if (fault != AD_OK) latch_error(status, fault);
  return fault == AD_OK;
}

// 2^x to 2^-22 of itself; 0 for -inf.
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// Two FP32 operations in one instruction.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{ .reg .b64 a, b, c, d; mov.b64 a, {%2, %3}; mov.b64 b, {%4, %5}; mov.b64 c, {%6, %7}; fma.rn.f32x2 d, a, b, c; mov.b64 {%0, %1}, d; }"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 d;
  asm("{ .reg .b64 a, b, d; mov.b64 a, {%2, %3}; mov.b64 b, {%4, %5}; add.rn.f32x2 d, a, b; mov.b64 {%0, %1}, d; }"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 d;
  asm("{ .reg .b64 a, b, d; mov.b64 a, {%2, %3}; mov.b64 b, {%4, %5}; mul.rn.f32x2 d, a, b; mov.b64 {%0, %1}, d; }"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}

// Eight consecutive numbers of FP32 or BF16.
__device__ __forceinline__ void load8(const float* p, float* x) {
  const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
  x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
__device__ __forceinline__ void load8(const bf16* p, float* x) {
  const uint4 v = *reinterpret_cast<const uint4*>(p);
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
}
__device__ __forceinline__ void store8(float* p, const float* x) {
  *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
  *reinterpret_cast<float4*>(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
}
__device__ __forceinline__ void store8(bf16* p, const float* x) {
  __nv_bfloat162 w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
  *reinterpret_cast<uint4*>(p) = *reinterpret_cast<const uint4*>(w);
}

// Writes row b's new tokens into the blocks they fall in.  A block's scale comes from what it holds afterwards: the tokens in front (what their
// codes stand for) and the new ones, so that tokens which were written and then given up leave no trace in it.  Scales are powers of two: a live
// code that gets another scale is only moved by whole binary places, exact in E4M3 above the subnormals of the new scale, and in INT8 off by half a
// step of the new scale; steps at least double from one rounding to the next, so all of a value's roundings together stay below one step of the
// largest scale that its block ever had.
// A CTA takes a block of tokens' keys or values of one head at a time, `tiles` of them one after the other, with the next one's loads under way; numbers
// stay in registers between the maximum and the codes, so that everything is read and written once.  Bound by bytes: 8 prompts of 2500 to 8190
// tokens, 8 heads of 128, BF16 to E4M3, 59 us, 4.5 TB/s (a tile a CTA 100 us, two 76, four 64, eight 64 in a build before); a third of the time the
// issue slots are idle, in the barrier of each tile and its round trips.
// POOLED: refs counts the entries of the table that name a block, and a row that lacks a block or would write one that others hold too is left out by all of its CTAs (one more
// round trip: 32 rows of a token 6.6 -> 7.7 us, 32 of 32 7.3 -> 8.0, 8 of 4000 in blocks of 64 40 -> 42 and of 16 38 -> 45).
// grid = (ceil(2 * heads / tiles), blocks a row's new tokens may touch, B), block = max(32, block * dim / 32) threads.
constexpr int VECS = 4;                // vectors of eight numbers a thread holds
__device__ __forceinline__ uint32_t max_bits(uint32_t m, uint4 v, float) {      // largest |x| as an integer: FP32 ...
  return max(max(max(m, v.x & 0x7fffffffu), max(v.y & 0x7fffffffu, v.z & 0x7fffffffu)), v.w & 0x7fffffffu);
}
__device__ __forceinline__ uint32_t max_bits(uint32_t m, uint4 v, bf16) {       // ... or of two BF16 side by side
  m = __vmaxu2(m, v.x & 0x7fff7fffu);
  m = __vmaxu2(m, v.y & 0x7fff7fffu);
  m = __vmaxu2(m, v.z & 0x7fff7fffu);
  return __vmaxu2(m, v.w & 0x7fff7fffu);
}
template <typename T, typename F, bool POOLED>
__global__ void __launch_bounds__(512)
cache_append_kernel(Cache c, const int* __restrict__ refs, const T* __restrict__ k, const T* __restrict__ v, size_t stride, int dim, const int* __restrict__ off,
                    const int* __restrict__ len, int M, int max_new, int tiles, int* status) {
  constexpr int WORDS = sizeof(T) / 2;                    // 16-byte words of a vector
  __shared__ uint32_t s_max[2][16];
  pdl_launch();
  pdl_wait();
  const int b = blockIdx.z, first = blockIdx.x * tiles, last = min(first + tiles, 2 * c.heads), warps = blockDim.x >> 5;
  int o, n, p;
  if (!row_tokens(c, off, len, b, M, max_new, false, status, o, n, p)) return;
  const int i = p / c.block + blockIdx.y, base = i * c.block;
  if (base >= p + n) return;
  const int live = max(p - base, 0), end = min(p + n - base, c.block);          // tokens in front, end of the new ones
  const int shift = __ffs(dim) - 4, vecs = c.block << shift;                    // (dim / 8 vectors a token)
  auto token = [&](int u) { return (int)(threadIdx.x + u * blockDim.x) >> shift; };
  auto place = [&](int u) { return (int)(threadIdx.x + u * blockDim.x) * 8; };  // in the block's codes
  auto inside = [&](int u) { return (int)(threadIdx.x + u * blockDim.x) < vecs; };
  auto load_new = [&](int tile, uint4 (*raw)[WORDS]) {
    const T* src = (tile & 1 ? v : k) + (size_t)(tile >> 1) * dim + (size_t)(o + base - p) * stride;
#pragma unroll
    for (int u = 0; u < VECS; ++u) {
      const int t = token(u);
      const bool in = inside(u) && t >= live && t < end;
#pragma unroll
      for (int j = 0; j < WORDS; ++j)
        raw[u][j] = in ? __ldcs(reinterpret_cast<const uint4*>(src + (size_t)t * stride + (place(u) & (dim - 1))) + j) : make_uint4(0u, 0u, 0u, 0u);
    }
  };
  constexpr bool AHEAD = sizeof(T) == 2;                  // (FP32's would take too many registers)
  uint4 raw[VECS][WORDS], next[AHEAD ? VECS : 1][WORDS];
  load_new(first, AHEAD ? next : raw);                    // the new tokens do not wait for the table
  const int id = c.find(b, i);
  if constexpr (POOLED) {
    bool own = true;
    for (int j = p / c.block + (int)threadIdx.x; j <= (p + n - 1) / c.block; j += blockDim.x) {
      const int e = c.find(b, j);
      own = own && e >= 0 && __ldcg(refs + e) <= 1;
    }
    if (!__syncthreads_and(own)) { latch_error(status, AD_ERR_ARG); return; }
  }
  if (id < 0) { latch_error(status, AD_ERR_ARG); return; }
  for (int tile = first; tile < last; ++tile) {
    const int which = tile & 1, head = tile >> 1, turn = (tile - first) & 1;
    if constexpr (AHEAD) {
#pragma unroll
      for (int u = 0; u < VECS; ++u) raw[u][0] = next[u][0];
      if (tile + 1 < last) load_new(tile + 1, next);
    } else {
      if (tile > first) load_new(tile, raw);
    }
    uint8_t* codes = (which ? c.codes[1] : c.codes[0]) + ((size_t)id * c.heads + head) * c.block * dim;
    float* scale = (which ? c.scale[1] : c.scale[0]) + (size_t)id * c.heads + head;
    const float old = live ? __ldcg(scale) : 1.f;
    uint32_t top = 0;
#pragma unroll
    for (int u = 0; u < VECS; ++u)
#pragma unroll
      for (int j = 0; j < WORDS; ++j) top = max_bits(top, raw[u][j], T());
    if (sizeof(T) == 2) top = max(top << 16, top & 0xffff0000u);
    auto numbers = [&](int u, float* x) {
      if (token(u) < live) {
        F::decode4(raw[u][0].x, x);
        F::decode4(raw[u][0].y, x + 4);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          x[j] *= old;
          if (isinf(x[j])) x[j] = copysignf(FLT_MAX, x[j]);      // (FP32's largest had been rounded up to 2^128: FLT_MAX has the same code)
        }
      } else {
        load8(reinterpret_cast<const T*>(raw[u]), x);
      }
    };
    if (live) {                                           // those in front, as they are
#pragma unroll
      for (int u = 0; u < VECS; ++u) {
        if (!inside(u) || token(u) >= live) continue;
        const uint2 w = __ldcg(reinterpret_cast<const uint2*>(codes + place(u)));
        raw[u][0].x = w.x;
        raw[u][0].y = w.y;
        float x[8];
        numbers(u, x);
#pragma unroll
        for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(x[j]) & 0x7fffffffu);
      }
    }
    auto block_max = [&](uint32_t m) {
      m = __reduce_max_sync(0xffffffffu, m);
      if ((threadIdx.x & 31) == 0) s_max[turn][threadIdx.x >> 5] = m;
      __syncthreads();
      for (int w = 0; w < warps; ++w) m = max(m, s_max[turn][w]);
      return m;
    };
    top = block_max(top);
    if (top >= 0x7f800000u) {                             // infinities saturate, whatever the scale; a NaN becomes 0
      uint32_t finite = 0;
      bool nan = false;
#pragma unroll
      for (int u = 0; u < VECS; ++u) {
        float x[8];
        numbers(u, x);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const uint32_t m = __float_as_uint(x[j]) & 0x7fffffffu;
          if (m < 0x7f800000u) finite = max(finite, m);
          else if (m > 0x7f800000u && token(u) >= live) { nan = true; reinterpret_cast<T*>(raw[u])[j] = from_f32<T>(0.f); }
        }
      }
      if (nan) latch_error(status, AD_ERR_ARG);
      __syncthreads();
      top = block_max(finite);
    }
    const float s = block_scale<F>(__uint_as_float(top)), inv = 1.f / s;        // (both powers of two)
#pragma unroll
    for (int u = 0; u < VECS; ++u) {
      const int t = token(u);
      if (!inside(u) || t >= end || (t < live && s == old)) continue;
      float x[8];
      numbers(u, x);
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] *= inv;
      *reinterpret_cast<uint2*>(codes + place(u)) = make_uint2(F::encode4(x), F::encode4(x + 4));
    }
    if (threadIdx.x == 0) *scale = s;
  }
}

// Reads tokens start[b] .. of row b back into k, v [M, heads, dim], tile after tile as above.  Bound by bytes, two thirds of them written: the prompts
// above, E4M3 to BF16, 53 us, 5.0 TB/s (a tile a CTA 72 us).
// grid as above, block = max(32, block * dim / 64).
constexpr int READ_VECS = 4;           // vectors of sixteen codes a thread holds
template <typename T, typename F>
__global__ void __launch_bounds__(256)
cache_read_kernel(Cache c, T* __restrict__ k, T* __restrict__ v, int dim, const int* __restrict__ off, const int* __restrict__ start, int M, int max_tokens,
                  int tiles, int* status) {
  pdl_launch();
  pdl_wait();
  const int b = blockIdx.z, first = blockIdx.x * tiles, last = min(first + tiles, 2 * c.heads);
  int o, n, p;
  if (!row_tokens(c, off, start, b, M, max_tokens, false, status, o, n, p)) return;
  const int i = p / c.block + blockIdx.y, base = i * c.block;
  if (base >= p + n) return;
  const int id = c.find(b, i);
  if (id < 0) { latch_error(status, AD_ERR_ARG); return; }
  const int from = max(p - base, 0), end = min(p + n - base, c.block);
  const int shift = __ffs(dim) - 5, vecs = c.block << shift;
  auto load = [&](int tile, uint4* w, float& s) {
    const size_t at = (size_t)id * c.heads + (tile >> 1);
    const uint8_t* codes = (tile & 1 ? c.codes[1] : c.codes[0]) + at * c.block * dim;
    s = __ldcg((tile & 1 ? c.scale[1] : c.scale[0]) + at);
#pragma unroll
    for (int u = 0; u < READ_VECS; ++u) {
      const int e = threadIdx.x + u * blockDim.x, t = e >> shift;
      if (e < vecs && t >= from && t < end) w[u] = __ldcs(reinterpret_cast<const uint4*>(codes + e * 16));
    }
  };
  uint4 next[READ_VECS];
  float next_scale;
  load(first, next, next_scale);
  for (int tile = first; tile < last; ++tile) {
    uint4 w[READ_VECS];
#pragma unroll
    for (int u = 0; u < READ_VECS; ++u) w[u] = next[u];
    const float s = next_scale;
    if (tile + 1 < last) load(tile + 1, next, next_scale);
    T* dst = (tile & 1 ? v : k) + (size_t)(tile >> 1) * dim + (size_t)(o + base - p) * c.heads * dim;
#pragma unroll
    for (int u = 0; u < READ_VECS; ++u) {
      const int e = threadIdx.x + u * blockDim.x, t = e >> shift;
      if (e >= vecs || t < from || t >= end) continue;
      const uint32_t words[4] = {w[u].x, w[u].y, w[u].z, w[u].w};
      T* to = dst + (size_t)t * c.heads * dim + (e * 16 & (dim - 1));
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float x[8];
        F::decode4(words[2 * h], x);
        F::decode4(words[2 * h + 1], x + 4);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] *= s;
        store8(to + 8 * h, x);
      }
    }
  }
}

}  // namespace kv
}  // namespace ad
