// Attention of the tokens of a block over the 8-bit key/value cache (kv_cache.cuh).
#pragma once

#include <float.h>

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
  int row_tiles, splits;   // tiles of rows that queries may need; parts that keys may be split into
  int chunk;               // units of a part
  float* part;             // splits > 1: [tile rows][splits][dim] sums, then [tile rows][splits] maxima and sums of exponentials
  // units of a part of a row with that many units
  __host__ __device__ __forceinline__ int part_units(int units) const { const int least = (units + splits - 1) / splits; return least > chunk ? least : chunk; }
};

constexpr int UNIT = 32;               // keys that a warp works on at a time
constexpr int ATT_WARPS = 4;
constexpr int MAX_SPLITS = 256, FEW_SPLITS = 8;      // parts at most; parts that one thread joins
__host__ __device__ constexpr int att_stages(int dim, int nq) { return dim == 128 ? (nq == 4 ? 3 : 2) : dim == 64 ? 3 : 4; }
// CTAs an SM: what registers and shared memory allow.
__host__ __device__ constexpr int att_resident(int dim, int nq) {
  return dim == 128 ? (nq == 4 ? 2 : 3) : dim == 64 ? (nq == 1 ? 4 : 3) : (nq == 1 ? 5 : nq == 2 ? 4 : 3);
}
__host__ __device__ constexpr int att_stage_bytes(int dim) { return 2 * UNIT * dim + 16; }
__host__ __device__ constexpr int att_q_bytes(int dim, int nq, bool fp32) { return (nq + 1) / 2 * (dim / 16) * 512 * (fp32 ? 2 : 1); }
__host__ __device__ constexpr int att_smem(int dim, int nq, bool fp32) {
  return att_q_bytes(dim, nq, fp32) + ATT_WARPS * att_stages(dim, nq) * att_stage_bytes(dim);
}

// 2^x to 2^-22 of itself; 0 for -inf.
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// log2 x: the exponent as it is, which is all there is to a power of two, and the mantissa's to 2^-22.
__device__ __forceinline__ float lg2(float x) {
  const uint32_t w = __float_as_uint(x);
  float y;
  asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(__uint_as_float((w & 0x7fffffu) | 0x3f800000u)));
  return (float)((int)(w >> 23) - 127) + y;
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
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t w;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(hi), "f"(lo));
  return w;
}
__device__ __forceinline__ float2 unpack_f16(uint32_t w) { return __half22float2(*reinterpret_cast<__half2*>(&w)); }
// What rounding a pair to FP16 leaves over, in FP16.
__device__ __forceinline__ uint32_t rest_f16(float lo, float hi, uint32_t w) {
  const float2 f = unpack_f16(w);
  return pack_f16(lo - f.x, hi - f.y);
}
__device__ __forceinline__ void mma_f16(float* d, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// Four codes to FP16, exactly: lo holds the first two, hi the others.
__device__ __forceinline__ void codes_f16(E4m3, uint32_t w, uint32_t& lo, uint32_t& hi) {
  asm("{ .reg .b16 l, h; mov.b32 {l, h}, %2; cvt.rn.f16x2.e4m3x2 %0, l; cvt.rn.f16x2.e4m3x2 %1, h; }" : "=r"(lo), "=r"(hi) : "r"(w));
}
__device__ __forceinline__ void codes_f16(Int8, uint32_t w, uint32_t& lo, uint32_t& hi) {
  // c + 128 as the low byte of 0x6400 is 1152 + c
  w ^= 0x80808080u;
  const uint32_t a = __byte_perm(w, 0x64646464u, 0x4140), b = __byte_perm(w, 0x64646464u, 0x4342);
  const __half2 bias = __float2half2_rn(1152.f);
  const __half2 x = __hsub2(*reinterpret_cast<const __half2*>(&a), bias), y = __hsub2(*reinterpret_cast<const __half2*>(&b), bias);
  lo = *reinterpret_cast<const uint32_t*>(&x);
  hi = *reinterpret_cast<const uint32_t*>(&y);
}
// The same for the first product, which takes multiples of them plus a bias: (code + BIAS) / FACTOR, with BIAS times the sum of a row's query (and
// its sign) where the product starts from.  INT8's c + 128 alone in FP16's low byte is that many times 2^-24.
template <typename F> struct KeyCodes { static constexpr float BIAS = 0.f, FACTOR = 1.f; };
template <> struct KeyCodes<Int8> { static constexpr float BIAS = 128.f, FACTOR = 16777216.f; };
__device__ __forceinline__ void key_codes_f16(E4m3 f, uint32_t w, uint32_t& lo, uint32_t& hi) { codes_f16(f, w, lo, hi); }
__device__ __forceinline__ void key_codes_f16(Int8, uint32_t w, uint32_t& lo, uint32_t& hi) {
  w ^= 0x80808080u;
  lo = __byte_perm(w, 0u, 0x4140);
  hi = __byte_perm(w, 0u, 0x4342);
}
__device__ __forceinline__ void cp4(void* smem_dst, const void* gmem_src) {
  const uint32_t s = static_cast<uint32_t>(__cvta_generic_to_shared(smem_dst));
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(s), "l"(gmem_src) : "memory");
}

// Key (of a unit) that column n of score tile nt stands for.  The scores of a thread's columns 2c, 2c + 1 in tiles 2j, 2j + 1 are, as they lie, its
// part of the probabilities' operand of the second product; this order makes them keys 16 j + c + {0, 4, 8, 12}, which reads values without bank conflicts.
__device__ __forceinline__ int unit_key(int nt, int n) { return 16 * (nt >> 1) + (n >> 1) + 4 * ((nt & 1) * 2 + (n & 1)); }

// Attention of 8 NQ rows (queries of one row of the batch times the query heads that share a key/value head) over a part of the row's keys.
//
// What a number goes through.  Codes are exact in FP16, and so are queries once a power of two has brought the row's largest to 2^13 (BF16 has 8 bits;
// FP32 goes in as two FP16 numbers, 22 bits, and so do its probabilities).  Scores are FP32: the keys' scale, the softmax scale and the query's power
// of two come in one factor per block and row.  Probabilities meet the values' scale before they are rounded: p * vs, as a multiple of its largest
// value so far in the row (2^d times what the softmax's own maximum m stands for), times 2^14: nothing that matters comes near FP16's subnormals,
// however far the blocks' scales are apart.  Sums, maxima and results are FP32.
//
// Why this shape.  What has to be read is 2 * dim bytes a key; 16 rows make 64 operations a byte of it, which mma.sync delivers several times over, so the kernel
// is a stream of the cache with as little as possible per byte: each warp copies its own units of 32 keys through its own ring in shared memory
// (16-byte asynchronous copies, zeros where no key is), nothing but __syncwarp between them, and keeps maximum, sum and result in registers until its
// keys are through; the four warps' results are joined at the end.  The 16-byte pieces lie in shared memory so that both products' operands come out
// of it whole, in the registers where mma wants them, without a transposition: dims and keys may be summed in any order.
// TWO: blocks of 16 tokens, two in a unit.
// grid = (row_tiles * splits, heads, B), block = 32 * ATT_WARPS.
template <typename T, typename F, int DIM, int NQ, bool TWO>
__global__ void __launch_bounds__(32 * ATT_WARPS, att_resident(DIM, NQ))
cache_attention_kernel(AttendParams a) {
  constexpr bool WIDE = sizeof(T) == 4;               // two FP16 numbers for each query and probability
  constexpr int HL = WIDE ? 2 : 1;
  constexpr int KSTEPS = DIM / 16, ND = DIM / 16, MT = (NQ + 1) / 2, ROWS = 8 * NQ;
  constexpr int STAGES = att_stages(DIM, NQ), STAGE = att_stage_bytes(DIM), COPIES = DIM / 16;
  constexpr int P_BITS = 14;
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ float s_rf[ROWS], s_start[ROWS];
  uint4* sq = reinterpret_cast<uint4*>(smem);          // [HL][MT][KSTEPS][lane]: operands as mma wants them
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, c = lane & 3;
  unsigned char* ring = smem + att_q_bytes(DIM, NQ, WIDE) + warp * STAGES * STAGE;
  pdl_launch();
  pdl_wait();
  const int b = blockIdx.z, kvh = blockIdx.y, rt = blockIdx.x % a.row_tiles, split = blockIdx.x / a.row_tiles;
  int o, n, p;
  if (!row_tokens(a.c, a.off, a.len, b, a.M, a.max_new, !a.causal, a.status, o, n, p)) return;
  const int group = a.n_heads / a.c.heads, rows = n * group, r0 = rt * ROWS;
  if (r0 >= rows) return;
  const int r_last = min(r0 + ROWS, rows) - 1;
  auto visible = [&](int r) { return a.causal ? p + min(r, r_last) / group + 1 : p; };
  const int vis_min = visible(r0), vis_max = visible(r_last);
  const int units = (vis_max + UNIT - 1) / UNIT, per_part = a.part_units(units);
  const int first_unit = split * per_part, part_units = min(units - first_unit, per_part);
  if (part_units <= 0 && split > 0) return;
  const int u0 = first_unit + part_units * warp / ATT_WARPS, u1 = first_unit + part_units * (warp + 1) / ATT_WARPS;

  // ---- the ring ----
  const int block = a.c.block;
  int ids[2] = {0, 0}, id_base = u0;                             // lane i: block(s) of unit id_base + i
  auto look_up = [&](int base) {
    id_base = base;
    const int u = base + lane;
#pragma unroll
    for (int z = 0; z < (TWO ? 2 : 1); ++z) {
      const int pos = u * UNIT + 16 * z;
      ids[z] = u < u1 && pos < vis_max ? a.c.find(b, pos / block) : 0;
      if (ids[z] < 0) latch_error(a.status, AD_ERR_ARG);
    }
  };
  // Piece i of a thread's copies: byte 512 i + 16 lane of a unit's keys or values.  In shared memory keys lie in the order of score columns, values in
  // their own, both with their 16-byte pieces exchanged so that eight threads that read at once meet all banks.  What depends on the thread is the same for
  // every piece (for every other one, at DIM = 128), the rest is a constant.
  const int my_key = lane * 16 / DIM, my_x = lane * 16 % DIM / 16;
  const int my_col = ((my_key >> 3) & 1) * 8 + ((my_key & 3) << 1) + ((my_key >> 2) & 1);
  const uint32_t ring_s = static_cast<uint32_t>(__cvta_generic_to_shared(ring));
  const uint32_t k_dst = ring_s + my_col * DIM + my_x * 16, k_odd = ring_s + my_col * DIM + (DIM == 128 ? my_x ^ 4 : my_x) * 16;
  const uint32_t v_dst = ring_s + UNIT * DIM + my_key * DIM + (DIM == 128 ? my_x ^ ((my_key & 3) << 1) : DIM == 64 ? my_x ^ (((my_key >> 1) & 1) << 1) : my_x) * 16;
  auto issue = [&](int u, int stage) {
    if (u >= u1) return;
    if (u - id_base >= 32) look_up(u);
    const int first = u * UNIT;
    const uint32_t so = stage * STAGE;
    size_t tile[2];
    bool there[2];
#pragma unroll
    for (int z = 0; z < 2; ++z) {
      const int id = z == 0 || TWO ? __shfl_sync(0xffffffffu, ids[z], u - id_base) : 0;
      there[z] = id >= 0;
      tile[z] = (size_t)max(id, 0) * a.c.heads + kvh;
    }
    const size_t src = (tile[0] * block + (TWO ? 0 : first & (block - 1))) * DIM + lane * 16;
    const uint8_t* ks = a.c.codes[0] + src;
    const uint8_t* vs = a.c.codes[1] + src;
    const ptrdiff_t second = TWO ? (ptrdiff_t)(tile[1] - tile[0]) * 16 * DIM - 16 * DIM : 0;     // from where the second half would lie to where it does
    const bool whole = first + UNIT <= vis_max && there[0] && (!TWO || there[1]);
#pragma unroll
    for (int i = 0; i < COPIES; ++i) {
      const uint32_t kd = (DIM == 128 && (i & 1) ? k_odd : k_dst) + so + (DIM == 128 ? (16 * (i >> 2) + 8 * ((i >> 1) & 1) + (i & 1)) * DIM : i * 512);
      const uint32_t vd = v_dst + so + i * 512;
      const ptrdiff_t at = i * 512 + (TWO && i >= COPIES / 2 ? second : 0);
      const int z = TWO && i >= COPIES / 2 ? 1 : 0;
      const int n = whole || (there[z] && first + my_key + i * (512 / DIM) < vis_max) ? 16 : 0;   // zeros where there is no key
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(kd), "l"(ks + at), "r"(n) : "memory");
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(vd), "l"(vs + at), "r"(n) : "memory");
    }
    if (lane < 4) {                                               // ks0, ks1, vs0, vs1; negative: no such block
      const int z = lane & 1;
      float* dst = reinterpret_cast<float*>(ring + stage * STAGE + 2 * UNIT * DIM) + lane;
      const bool need = (z == 0 || TWO) && first + 16 * z < vis_max;
      if (need && (z ? there[1] : there[0])) cp4(dst, (lane < 2 ? a.c.scale[0] : a.c.scale[1]) + (z ? tile[1] : tile[0]));
      else *dst = need && lane < 2 ? -1.f : 1.f;
    }
  };
  look_up(u0);
#pragma unroll
  for (int s = 0; s < STAGES - 1; ++s) {
    issue(u0 + s, s);
    asm volatile("cp.async.commit_group;" ::: "memory");
  }

  // ---- queries: the row's power of two, FP16, into operand order ----
  // Thread's dims in step j: 64 (j / 4) + 16 c + 4 (j % 4) + 0 .. 3 (DIM = 32: 8 c + 4 j + 0 .. 3)
  for (int r = warp; r < 16 * MT; r += ATT_WARPS) {
    constexpr int PER = DIM / 32;
    const int row = r0 + r;
    float x[PER], top = 0.f;
#pragma unroll
    for (int i = 0; i < PER; ++i) x[i] = 0.f;
    if (r < ROWS && row <= r_last) {
      const T* q = static_cast<const T*>(a.q) + (size_t)(o + row / group) * a.q_stride + ((size_t)kvh * group + row % group) * DIM + lane * PER;
#pragma unroll
      for (int i = 0; i < PER; ++i) { x[i] = to_f32(q[i]); top = fmaxf(top, fabsf(x[i])); }
    }
    const uint32_t e = min(max(__reduce_max_sync(0xffffffffu, __float_as_uint(top)) >> 23, 27u), 253u);     // exponent, 2^-100 .. 2^126
    const float up = __uint_as_float((267u - e) << 23);            // 2^(13 - exponent)
    float total = 0.f;
#pragma unroll
    for (int i = 0; i < PER; i += (PER > 1 ? 2 : 1)) {
      // one number (DIM = 32) or pairs
      const int d = lane * PER + i;
      const int j = DIM == 32 ? (d >> 2) & 1 : (d >> 6) * 4 + ((d >> 2) & 3), cc = DIM == 32 ? d >> 3 : (d >> 4) & 3, half = (d >> 1) & 1;
      const int mt = r >> 4, word = half * 2 + ((r >> 3) & 1), ln = (r & 7) * 4 + cc;
      const float y0 = x[i] * up, y1 = PER > 1 ? x[PER > 1 ? i + 1 : 0] * up : 0.f;
      const uint32_t hi = pack_f16(y0, y1), lo = rest_f16(y0, y1, hi);
      if constexpr (KeyCodes<F>::BIAS != 0.f) {
        const float2 h2 = unpack_f16(hi), l2 = unpack_f16(lo);
        total += h2.x + h2.y + (WIDE ? l2.x + l2.y : 0.f);
      }
#pragma unroll
      for (int h = 0; h < HL; ++h) {
        unsigned char* dst = reinterpret_cast<unsigned char*>(sq + ((h * MT + mt) * KSTEPS + j) * 32 + ln) + word * 4;
        if (PER > 1) *reinterpret_cast<uint32_t*>(dst) = h ? lo : hi;
        else reinterpret_cast<uint16_t*>(dst)[d & 1] = (uint16_t)(h ? lo : hi);
      }
    }
#pragma unroll
    for (int w = 16; w; w >>= 1) total += __shfl_xor_sync(0xffffffffu, total, w);
    if (lane == 0 && r < ROWS) {
      s_rf[r] = a.scale * (1.f / up) * KeyCodes<F>::FACTOR;
      s_start[r] = -KeyCodes<F>::BIAS / KeyCodes<F>::FACTOR * total;
    }
  }
  __syncthreads();
  // Scores: thread's row g of each eight, columns as above.  Results: dims DIM / 8 * g .. of rows 2 c and 2 c + 1 of each eight.
  float rf[NQ], start[NQ], m[NQ], d[NQ], l[NQ], acc[NQ][ND][4];
  bool large = false;                                 // scores whose steps in FP32 are a quarter and more
  int vis[NQ];
#pragma unroll
  for (int q = 0; q < NQ; ++q) {
    rf[q] = s_rf[q * 8 + g];
    start[q] = s_start[q * 8 + g];
    vis[q] = visible(r0 + q * 8 + g);
    m[q] = d[q] = -INFINITY;
    l[q] = 0.f;
#pragma unroll
    for (int i = 0; i < ND; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[q][i][j] = 0.f;
  }
  // queries of few steps stay in registers
  constexpr bool Q_REGS = HL * MT * KSTEPS <= 4;
  uint4 qr[Q_REGS ? HL : 1][Q_REGS ? MT : 1][Q_REGS ? KSTEPS : 1];
  if constexpr (Q_REGS) {
#pragma unroll
    for (int h = 0; h < HL; ++h)
#pragma unroll
      for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int j = 0; j < KSTEPS; ++j) qr[h][t][j] = sq[((h * MT + t) * KSTEPS + j) * 32 + lane];
  }

  int stage = 0;
  for (int u = u0; u < u1; ++u) {
    asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 2) : "memory");
    __syncwarp();
    issue(u + STAGES - 1, stage == 0 ? STAGES - 1 : stage - 1);
    asm volatile("cp.async.commit_group;" ::: "memory");
    const unsigned char* st = ring + stage * STAGE;
    stage = stage == STAGES - 1 ? 0 : stage + 1;
    const float4 sc = *reinterpret_cast<const float4*>(st + 2 * UNIT * DIM);
    // ---- scores ----
    float s[MT][4][4];
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
      for (int nt = 0; nt < 4; ++nt)
#pragma unroll
        for (int j = 0; j < 4; ++j) s[t][nt][j] = KeyCodes<F>::BIAS != 0.f && 2 * t + (j >> 1) < NQ ? start[2 * t + (j >> 1) < NQ ? 2 * t + (j >> 1) : 0] : 0.f;
    constexpr int RAW = KSTEPS < 4 ? KSTEPS : 4;       // words of codes of one load
#pragma unroll
    for (int hh = 0; hh < KSTEPS / RAW; ++hh) {
      uint32_t raw[4][RAW];
#pragma unroll
      for (int nt = 0; nt < 4; ++nt) {
        const unsigned char* row = st + (nt * 8 + g) * DIM;
        if constexpr (DIM == 32) {
          const uint2 v = *reinterpret_cast<const uint2*>(row + c * 8);
          raw[nt][0] = v.x; raw[nt][1] = v.y;
        } else {
          const int x = hh * 4 + c;
          const uint4 v = *reinterpret_cast<const uint4*>(row + (DIM == 128 ? x ^ ((g & 1) << 2) : x) * 16);
          raw[nt][0] = v.x; raw[nt][1] = v.y; raw[nt][RAW - 2] = v.z; raw[nt][RAW - 1] = v.w;
        }
      }
#pragma unroll
      for (int j = 0; j < RAW; ++j) {
        uint4 qf[HL][MT];
#pragma unroll
        for (int h = 0; h < HL; ++h)
#pragma unroll
          for (int t = 0; t < MT; ++t) {
            if constexpr (Q_REGS) qf[h][t] = qr[h][t][hh * RAW + j];
            else qf[h][t] = sq[((h * MT + t) * KSTEPS + hh * RAW + j) * 32 + lane];
          }
#pragma unroll
        for (int nt = 0; nt < 4; ++nt) {
          uint32_t b0, b1;
          key_codes_f16(F(), raw[nt][j], b0, b1);
#pragma unroll
          for (int h = HL - 1; h >= 0; --h)
#pragma unroll
            for (int t = 0; t < MT; ++t) mma_f16(s[t][nt], reinterpret_cast<const uint32_t*>(&qf[h][t]), b0, b1);
        }
      }
    }
    if (u * UNIT + UNIT > vis_min || sc.x < 0.f || sc.y < 0.f) {
#pragma unroll
      for (int q = 0; q < NQ; ++q)
#pragma unroll
        for (int nt = 0; nt < 4; ++nt)
#pragma unroll
          for (int j = 0; j < 2; ++j)
            if (u * UNIT + unit_key(nt, 2 * c + j) >= vis[q] || (TWO && nt >= 2 ? sc.y : sc.x) < 0.f) s[q / 2][nt][2 * (q & 1) + j] = -INFINITY;
    }
    // ---- probabilities ----
    float ks[2] = {fabsf(sc.x), TWO ? fabsf(sc.y) : fabsf(sc.x)};
    const float ve[2] = {lg2(sc.z), TWO ? lg2(sc.w) : lg2(sc.z)};
    float ref[NQ], top[NQ], tod[NQ], tk[NQ][2];
    bool moved = false;
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      const float(*sq4)[4] = s[q / 2];
      const int h = 2 * (q & 1);
      float x0 = fmaxf(max3(sq4[0][h], sq4[0][h + 1], sq4[1][h]), sq4[1][h + 1]), x1 = max3(sq4[2][h], sq4[2][h + 1], sq4[3][h]);
      if (!TWO) x0 = max3(x0, x1, sq4[3][h + 1]);
      else x1 = fmaxf(x1, sq4[3][h + 1]);
      x0 = fmaxf(x0, __shfl_xor_sync(0xffffffffu, x0, 1));
      x0 = fmaxf(x0, __shfl_xor_sync(0xffffffffu, x0, 2));
      if (TWO) {
        x1 = fmaxf(x1, __shfl_xor_sync(0xffffffffu, x1, 1));
        x1 = fmaxf(x1, __shfl_xor_sync(0xffffffffu, x1, 2));
      } else {
        x1 = x0;
      }
      tk[q][0] = fmaxf(rf[q] * ks[0], FLT_MIN);
      tk[q][1] = fmaxf(rf[q] * ks[1], FLT_MIN);
      x0 = ceilf(x0 * tk[q][0]);                       // references are whole numbers: what goes from one to another is an exact power of two
      x1 = TWO ? ceilf(x1 * tk[q][1]) : x0;
      top[q] = fmaxf(m[q], fmaxf(x0, x1));
      ref[q] = top[q] == -INFINITY ? 0.f : top[q];
      tod[q] = fmaxf(d[q] + (m[q] - ref[q]), x0 - ref[q] + ve[0]);
      if (TWO) tod[q] = fmaxf(tod[q], x1 - ref[q] + ve[1]);
      moved |= top[q] != m[q] || tod[q] != d[q];
    }
    if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
      for (int q = 0; q < NQ; ++q) {
        const float less = m[q] - ref[q], keep_o = tod[q] == -INFINITY ? 0.f : ex2(less + (d[q] - tod[q]));
        m[q] = top[q];
        d[q] = tod[q];
        l[q] *= ex2(less);
        const float k0 = __shfl_sync(0xffffffffu, keep_o, 8 * c), k1 = __shfl_sync(0xffffffffu, keep_o, 8 * c + 4);
#pragma unroll
        for (int i = 0; i < ND; ++i) {
          const float2 y0 = mul2(make_float2(acc[q][i][0], acc[q][i][1]), make_float2(k0, k1)), y1 = mul2(make_float2(acc[q][i][2], acc[q][i][3]), make_float2(k0, k1));
          acc[q][i][0] = y0.x; acc[q][i][1] = y0.y; acc[q][i][2] = y1.x; acc[q][i][3] = y1.y;
        }
        large |= fabsf(ref[q]) > 4194304.f;
      }
      large = __any_sync(0xffffffffu, large);
    }
    if (large) {                                       // the exponent below then is a difference of rounded scores, as the maximum is one of them
#pragma unroll
      for (int q = 0; q < NQ; ++q) {
#pragma unroll
        for (int nt = 0; nt < 4; ++nt)
#pragma unroll
          for (int j = 0; j < 2; ++j) s[q / 2][nt][2 * (q & 1) + j] = __fsub_rn(__fmul_rn(s[q / 2][nt][2 * (q & 1) + j], tk[q][nt >> 1]), ref[q]);
        tk[q][0] = tk[q][1] = 1.f;
        ref[q] = 0.f;
      }
    }
    uint32_t pf[HL][NQ][4];                            // [score tile]: two keys' probabilities of row g, as the second product's operand
#pragma unroll
    for (int q = 0; q < NQ; ++q)
#pragma unroll
      for (int z = 0; z < 2; ++z) {
        // p, as a share of the softmax's maximum, times 2^(14 + e), e = log2(values' scale) - d: what goes into the second product.  Its sum is taken
        // as it is and brought back afterwards, which the bounds on e keep inside FP32 (beyond them the values do not count, or the probability).
        const float e = (float)P_BITS + fminf(fmaxf(ve[z] - d[q], -100.f), 100.f), less = e - ref[q];
        const float2 t2 = make_float2(tk[q][z], tk[q][z]), r2 = make_float2(less, less);
        float2 sum;
#pragma unroll
        for (int nt = 2 * z; nt < 2 * z + 2; ++nt) {
          float2 y = fma2(make_float2(s[q / 2][nt][2 * (q & 1)], s[q / 2][nt][2 * (q & 1) + 1]), t2, r2);
          y.x = ex2(y.x);
          y.y = ex2(y.y);
          sum = nt == 2 * z ? y : add2(sum, y);
          pf[0][q][nt] = pack_f16(y.x, y.y);
          if constexpr (WIDE) pf[HL - 1][q][nt] = rest_f16(y.x, y.y, pf[0][q][nt]);
        }
        l[q] = fmaf(sum.x + sum.y, ex2(-e), l[q]);
      }
    // ---- times values ----
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      constexpr int WORDS = DIM / 32;                  // words of a key's codes that the thread reads
      uint32_t v[4][WORDS];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int key = 16 * j + c + 4 * i;
        const unsigned char* row = st + UNIT * DIM + key * DIM;
        if constexpr (DIM == 128) {
          const uint4 x = *reinterpret_cast<const uint4*>(row + ((g ^ ((key & 3) << 1)) * 16));
          v[i][0] = x.x; v[i][1] = x.y; v[i][WORDS - 2] = x.z; v[i][WORDS - 1] = x.w;
        } else if constexpr (DIM == 64) {
          const uint2 x = *reinterpret_cast<const uint2*>(row + ((g >> 1) ^ (((key >> 1) & 1) << 1)) * 16 + (g & 1) * 8);
          v[i][0] = x.x; v[i][WORDS - 1] = x.y;
        } else {
          v[i][0] = *reinterpret_cast<const uint32_t*>(row + g * 4);
        }
      }
#pragma unroll
      for (int x = 0; x < WORDS; ++x)
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const uint32_t w0 = __byte_perm(v[0][x], v[1][x], y ? 0x7362 : 0x5140), w1 = __byte_perm(v[2][x], v[3][x], y ? 0x7362 : 0x5140);
          uint32_t av[4];                              // dims DIM / 8 * g + 4 x + 2 y and the next one, four keys
          codes_f16(F(), w0, av[0], av[1]);
          codes_f16(F(), w1, av[2], av[3]);
#pragma unroll
          for (int h = HL - 1; h >= 0; --h)
#pragma unroll
            for (int q = 0; q < NQ; ++q) mma_f16(acc[q][2 * x + y], av, pf[h][q][2 * j], pf[h][q][2 * j + 1]);
        }
    }
  }
  asm volatile("cp.async.wait_group 0;" ::: "memory");
  __syncthreads();

  // ---- the warps' results together ----
  constexpr int PITCH = DIM + 4;
  float* so = reinterpret_cast<float*>(smem);                     // [warps][ROWS][PITCH]
  float* sm = so + ATT_WARPS * ROWS * PITCH;                      // [warps][ROWS] maxima, sums, exponents of the results
  float* sl = sm + ATT_WARPS * ROWS;
  float* sd = sl + ATT_WARPS * ROWS;
  static_assert((ATT_WARPS * ROWS * (PITCH + 3)) * 4 <= att_smem(DIM, NQ, WIDE), "results fit where the ring was");
#pragma unroll
  for (int q = 0; q < NQ; ++q) {
    float* dst = so + (warp * ROWS + q * 8 + 2 * c) * PITCH + g * (DIM / 8);
#pragma unroll
    for (int i = 0; i < ND; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) *reinterpret_cast<float2*>(dst + j * PITCH + 2 * i) = make_float2(acc[q][i][j], acc[q][i][2 + j]);
    float sum = l[q];
    sum += __shfl_xor_sync(0xffffffffu, sum, 1);
    sum += __shfl_xor_sync(0xffffffffu, sum, 2);
    if (c == 0) {
      const int r = warp * ROWS + q * 8 + g;
      sm[r] = m[q]; sl[r] = sum; sd[r] = d[q] - (float)P_BITS;
    }
  }
  __syncthreads();
  constexpr int LANES = DIM / 8, AT_ONCE = 32 * ATT_WARPS / LANES;      // threads a row, each eight dims
  const int d0 = tid % LANES * 8;
  const size_t tile_row = (((size_t)b * a.c.heads + kvh) * a.row_tiles + rt) * ROWS, all_rows = (size_t)gridDim.z * gridDim.y * a.row_tiles * ROWS;
  for (int r = tid / LANES; r < ROWS && r0 + r <= r_last; r += AT_ONCE) {
    float top = -INFINITY, sum = 0.f, x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = 0.f;
#pragma unroll
    for (int v = 0; v < ATT_WARPS; ++v) top = fmaxf(top, sm[v * ROWS + r]);
#pragma unroll
    for (int v = 0; v < ATT_WARPS; ++v) {
      const float mv = sm[v * ROWS + r], lv = sl[v * ROWS + r], f = mv == top ? 1.f : ex2(mv - top), fo = ex2(sd[v * ROWS + r]) * f;
      if (lv == 0.f) continue;                          // (no key)
      sum += lv * f;
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] += so[(v * ROWS + r) * PITCH + d0 + i] * fo;
    }
    if (per_part < units) {
      const size_t slot = (tile_row + r) * a.splits + split;
      store8(a.part + slot * DIM + d0, x);
      if (d0 == 0) reinterpret_cast<float2*>(a.part + all_rows * a.splits * DIM)[slot] = make_float2(top, sum);
    } else {
      const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] *= inv;
      const int row = r0 + r;
      store8(static_cast<T*>(a.out) + ((size_t)(o + row / group) * a.n_heads + kvh * group + row % group) * DIM + d0, x);
    }
  }
}

// Joins the parts of a row's keys, where there is more than one.  Four dims a thread, so that 128 threads are 128 / (DIM / 4) groups: SHARED, they take
// a row's parts in turn and add up in their order, else each has a row of its own.  Bound by latency: maxima and sums of all parts are loaded at once
// (each lane of a warp one part), results eight parts ahead.
// grid = (rows, or rows / groups, heads, B), block = 128.
template <typename T, int DIM, int NQ, bool SHARED>
__global__ void __launch_bounds__(128)
cache_attention_join_kernel(AttendParams a) {
  constexpr int ROWS = 8 * NQ, LANES = DIM / 4, GROUPS = 128 / LANES;
  __shared__ float4 s_x[SHARED ? GROUPS - 1 : 1][LANES];
  __shared__ float s_w[SHARED ? MAX_SPLITS : 1];
  pdl_launch();
  pdl_wait();
  const int tid = threadIdx.x, grp = tid / LANES, d0 = tid % LANES * 4;
  const int b = blockIdx.z, kvh = blockIdx.y, r = SHARED ? blockIdx.x : blockIdx.x * GROUPS + grp;
  int o, n, p;
  if (!row_tokens(a.c, a.off, a.len, b, a.M, a.max_new, !a.causal, a.status, o, n, p)) return;
  const int group = a.n_heads / a.c.heads;
  if (r >= n * group) return;
  // as many parts as the row's tile has been split into
  const int r_last = min(r / ROWS * ROWS + ROWS, n * group) - 1, units = ((a.causal ? p + r_last / group + 1 : p) + UNIT - 1) / UNIT;
  const int per_part = a.part_units(units), parts = (units + per_part - 1) / per_part;
  if (parts <= 1) return;
  const size_t all_rows = (size_t)gridDim.z * gridDim.y * a.row_tiles * ROWS;
  const size_t slot = (((size_t)b * a.c.heads + kvh) * a.row_tiles * ROWS + r) * a.splits;
  const float2* ml = reinterpret_cast<const float2*>(a.part + all_rows * a.splits * DIM) + slot;
  const float* part = a.part + slot * DIM + d0;
  float sum = 0.f;
  float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
  auto add = [&](float4 y, float f) { x.x = fmaf(y.x, f, x.x); x.y = fmaf(y.y, f, x.y); x.z = fmaf(y.z, f, x.z); x.w = fmaf(y.w, f, x.w); };
  if constexpr (SHARED) {
    // every warp for itself: maxima, weights, and their sum
    const int lane = tid & 31;
    float top = -INFINITY;
    float2 v[MAX_SPLITS / 32];
#pragma unroll
    for (int i = 0; i < MAX_SPLITS / 32; ++i) {
      v[i] = i * 32 + lane < parts ? __ldcg(ml + i * 32 + lane) : make_float2(-INFINITY, 0.f);
      top = fmaxf(top, v[i].x);
    }
#pragma unroll
    for (int w = 16; w; w >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
#pragma unroll
    for (int i = 0; i < MAX_SPLITS / 32; ++i) {
      const float f = v[i].y == 0.f ? 0.f : v[i].x == top ? 1.f : ex2(v[i].x - top);      // (no key: nothing, whatever the maxima)
      sum += v[i].y * f;
      if (tid < 32 && i * 32 + lane < parts) s_w[i * 32 + lane] = f;
    }
#pragma unroll
    for (int w = 16; w; w >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, w);
    __syncthreads();
    for (int s0 = grp; s0 < parts; s0 += 8 * GROUPS) {
      float4 y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (s0 + i * GROUPS < parts) y[i] = __ldcg(reinterpret_cast<const float4*>(part + (size_t)(s0 + i * GROUPS) * DIM));
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (s0 + i * GROUPS < parts) add(y[i], s_w[s0 + i * GROUPS]);
    }
    if (grp > 0) s_x[grp - 1][tid % LANES] = x;
    __syncthreads();
    if (grp > 0) return;
#pragma unroll
    for (int i = 0; i < GROUPS - 1; ++i) add(s_x[i][tid], 1.f);
  } else {
    float top = -INFINITY;
    float2 v[FEW_SPLITS];
    float4 y[FEW_SPLITS];
#pragma unroll
    for (int i = 0; i < FEW_SPLITS; ++i) {
      v[i] = i < parts ? __ldcg(ml + i) : make_float2(-INFINITY, 0.f);
      if (i < parts) y[i] = __ldcg(reinterpret_cast<const float4*>(part + (size_t)i * DIM));
      top = fmaxf(top, v[i].x);
    }
#pragma unroll
    for (int i = 0; i < FEW_SPLITS; ++i) {
      if (i >= parts || v[i].y == 0.f) continue;
      const float f = v[i].x == top ? 1.f : ex2(v[i].x - top);
      sum = fmaf(v[i].y, f, sum);
      add(y[i], f);
    }
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  T* out = static_cast<T*>(a.out) + ((size_t)(o + r / group) * a.n_heads + kvh * group + r % group) * DIM + d0;
  if constexpr (sizeof(T) == 4) {
    *reinterpret_cast<float4*>(out) = make_float4(x.x * inv, x.y * inv, x.z * inv, x.w * inv);
  } else {
    __nv_bfloat162 w[2] = {__floats2bfloat162_rn(x.x * inv, x.y * inv), __floats2bfloat162_rn(x.z * inv, x.w * inv)};
    *reinterpret_cast<uint2*>(out) = *reinterpret_cast<const uint2*>(w);
  }
}

}  // namespace kv
}  // namespace ad
