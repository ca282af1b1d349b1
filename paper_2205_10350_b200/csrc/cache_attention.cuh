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
  int B;
  int stream_once;         // more keys and values than L2 could hold for the next call
  int grid;                // CTAs
  int fixed;               // what an item takes besides its units, in units
  int granule;             // units that one CTA works on at the least where a row's keys are split; 0: they are not
  float* part;             // [2 grid][tile rows][dim] means of values, then [2 grid][tile rows] maxima and sums of exponentials
  long long* prefix;       // [B + 1] granules in front of each row of the batch
};

constexpr int UNIT = 32;               // keys that a warp works on at a time
constexpr int ATT_WARPS = 4;
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

// Work.  A row of the batch has `heads` times `tiles` (of its queries) items, each over all of the keys that the tile sees; an item is cut into `pieces`
// granules of about the same number of units, and the CTAs share all granules evenly, in their order.  So a CTA works on a part of an item, or on
// several, of which only the first and the last may be parts; lengths live on the device, and no batch is too ragged.
struct RowWork {
  int o, n, p, tiles, units, pieces;
  long long granules;
};
__device__ __forceinline__ RowWork row_work(const AttendParams& a, int b, int tile_rows) {
  RowWork w;
  w.granules = 0;
  if (!row_tokens(a.c, a.off, a.len, b, a.M, a.max_new, !a.causal, a.status, w.o, w.n, w.p)) return w;
  w.tiles = (w.n * (a.n_heads / a.c.heads) + tile_rows - 1) / tile_rows;
  w.units = (w.p + (a.causal ? w.n : 0) + UNIT - 1) / UNIT;
  w.pieces = a.granule ? (w.units + a.fixed + a.granule / 2) / a.granule : 1;
  w.granules = (long long)a.c.heads * w.tiles * w.pieces;
  return w;
}
__host__ __device__ __forceinline__ long long cta_start(long long total, long long cta, long long ctas) { return total * cta / ctas; }
// The CTA that granule g falls to.
__host__ __device__ __forceinline__ int cta_of(long long total, long long g, long long ctas) { return (int)(((g + 1) * ctas - 1) / total); }

// A CTA's place in its share of the work, kept in shared memory: the loop over keys has no use for it, and every use for its registers.
struct Segment {
  RowWork work;
  long long at, cur;                   // granule of the row of the batch, and of all
  int b, piece, piece_end, kvh, r0, r_last;
  long long scan[ATT_WARPS], base;
  int row;
};
// Granules g0 .. g1 - 1 are this CTA's; the first of them is where seg starts.  False: none.  CTA 0 leaves the granules in front of each row for the join.
__device__ __forceinline__ bool find_share(const AttendParams& a, int rows, Segment& seg, long long& g0, long long& g1) {
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  long long total = 0, mine = 0, front = 0;
  for (int b0 = 0; b0 < a.B; b0 += 32 * ATT_WARPS) {
    mine = b0 + tid < a.B ? row_work(a, b0 + tid, rows).granules : 0;
    long long run = mine;
#pragma unroll
    for (int w = 1; w < 32; w <<= 1) {
      const long long y = __shfl_up_sync(0xffffffffu, run, w);
      if (lane >= w) run += y;
    }
    if (lane == 31) seg.scan[warp] = run;
    __syncthreads();
    front = total + run - mine;
#pragma unroll
    for (int w = 0; w < ATT_WARPS; ++w) {
      if (w < warp) front += seg.scan[w];
      total += seg.scan[w];
    }
    if (blockIdx.x == 0 && a.granule && b0 + tid < a.B) a.prefix[b0 + tid] = front;
    __syncthreads();
  }
  if (blockIdx.x == 0 && a.granule && tid == 0) a.prefix[a.B] = total;
  const long long ctas = min((long long)gridDim.x, total);
  if (blockIdx.x >= ctas) return false;
  g0 = cta_start(total, blockIdx.x, ctas);
  g1 = cta_start(total, blockIdx.x + 1, ctas);
  if (a.B <= 32 * ATT_WARPS) {
    if (front <= g0 && g0 < front + mine) { seg.row = tid; seg.base = front; }
  } else if (warp == 0) {                     // (the same scan again, by one warp)
    long long base = 0;
    for (int b0 = 0; b0 < a.B; b0 += 32) {
      const long long x = b0 + lane < a.B ? row_work(a, b0 + lane, rows).granules : 0;
      long long run = x;
#pragma unroll
      for (int w = 1; w < 32; w <<= 1) {
        const long long y = __shfl_up_sync(0xffffffffu, run, w);
        if (lane >= w) run += y;
      }
      const long long f = base + run - x;
      if (f <= g0 && g0 < f + x) { seg.row = b0 + lane; seg.base = f; }
      base += __shfl_sync(0xffffffffu, run, 31);
      if (base > g0) break;
    }
  }
  __syncthreads();
  if (tid == 0) {
    seg.b = seg.row;
    seg.at = g0 - seg.base;
    seg.cur = g0;
    seg.work = row_work(a, seg.row, rows);
  }
  return true;
}
struct SegmentKeys { int kvh, r0, r_last, vis_min, vis_max, u0, u1; };      // positions that the first and the last row see; units (the tile may see fewer than the row has)
// Opens the segment that seg has come to; s_vis: positions that each row of the tile sees.
__device__ __forceinline__ SegmentKeys open_segment(const AttendParams& a, int rows, Segment& seg, int* s_vis, long long g1) {
  const RowWork& work = seg.work;
  const int tid = threadIdx.x, group = a.n_heads / a.c.heads;
  const int item = (int)(seg.at / work.pieces), piece = (int)(seg.at % work.pieces), piece_end = (int)min((long long)work.pieces, piece + (g1 - seg.cur));
  SegmentKeys v;
  v.kvh = item / work.tiles;
  v.r0 = item % work.tiles * rows;
  v.r_last = min(v.r0 + rows, work.n * group) - 1;
  v.vis_min = a.causal ? work.p + v.r0 / group + 1 : work.p;
  v.vis_max = a.causal ? work.p + v.r_last / group + 1 : work.p;
  const int units = (v.vis_max + UNIT - 1) / UNIT;
  v.u0 = min((int)((long long)work.units * piece / work.pieces), units);
  v.u1 = min((int)((long long)work.units * piece_end / work.pieces), units);
  if (tid < rows) s_vis[tid] = a.causal ? work.p + min(v.r0 + tid, v.r_last) / group + 1 : work.p;
  if (tid == 0) { seg.piece = piece; seg.piece_end = piece_end; seg.kvh = v.kvh; seg.r0 = v.r0; seg.r_last = v.r_last; }
  return v;
}
// On to the next segment (all threads, behind the last use of shared memory's segment); false: that was all.
__device__ __forceinline__ bool next_segment(const AttendParams& a, int rows, Segment& seg, long long g1) {
  const int done = seg.piece_end - seg.piece;
  if (seg.cur + done >= g1) return false;
  __syncthreads();                             // shared memory is the next item's
  if (threadIdx.x == 0) {
    seg.cur += done;
    seg.at += done;
    while (seg.at == seg.work.granules) { seg.at = 0; seg.work = row_work(a, ++seg.b, rows); }   // (rows without work have no granules)
  }
  return true;
}
constexpr int P_BITS = 15;                     // results lie this many binary places above p * scale's reference
constexpr float P_ONE = 1.f / (1 << P_BITS);
// Joins what PARTS warps found for the same rows over their keys (so [PARTS][ROWS][PITCH] results, sm, sl, sd [PARTS][ROWS] references, sums, exponents of
// the results) and writes it out, or as this CTA's part of the item.
template <typename T, int DIM, int ROWS, int PARTS, int PITCH>
__device__ __forceinline__ void store_results(const AttendParams& a, const Segment& seg, long long g0, const float* so, const float* sm, const float* sl,
                                              const float* sd) {
  constexpr int LANES = DIM / 8, AT_ONCE = 32 * ATT_WARPS / LANES;      // threads a row, each eight dims
  const int tid = threadIdx.x, d0 = tid % LANES * 8, group = a.n_heads / a.c.heads;
  const bool whole_item = seg.piece == 0 && seg.piece_end == seg.work.pieces;
  const size_t slot = 2 * (size_t)blockIdx.x + (seg.cur == g0 ? 0 : 1);
  const int r0 = seg.r0, r_last = seg.r_last, kvh = seg.kvh;
  for (int r = tid / LANES; r < ROWS && r0 + r <= r_last; r += AT_ONCE) {
    float top = -INFINITY, sum = 0.f, f[PARTS], x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = 0.f;
#pragma unroll
    for (int v = 0; v < PARTS; ++v) top = fmaxf(top, sm[v * ROWS + r]);
#pragma unroll
    for (int v = 0; v < PARTS; ++v) {
      const float mv = sm[v * ROWS + r], lv = sl[v * ROWS + r];
      f[v] = mv == top ? 1.f : ex2(mv - top);
      if (lv != 0.f) sum += lv * f[v];                  // (else: no key)
    }
    // Means, not sums, which FP32 may have no room for; factor after factor, as they may have none together.
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
    for (int v = 0; v < PARTS; ++v) {
      if (sl[v * ROWS + r] == 0.f) continue;
      const float share = f[v] * inv * P_ONE, unit = ex2(sd[v * ROWS + r]);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] += so[(v * ROWS + r) * PITCH + d0 + i] * share * unit;
    }
    if (!whole_item) {
      store8(a.part + (slot * ROWS + r) * DIM + d0, x);
      if (d0 == 0) reinterpret_cast<float2*>(a.part + 2 * (size_t)a.grid * ROWS * DIM)[slot * ROWS + r] = make_float2(top, sum);
    } else {
      const int row = r0 + r;
      store8(static_cast<T*>(a.out) + ((size_t)(seg.work.o + row / group) * a.n_heads + kvh * group + row % group) * DIM + d0, x);
    }
  }
}

// log2 x of a positive normal number, rounded up to a whole one; and its own value, which is the same for a power of two, else to 2^-22.
__device__ __forceinline__ float whole_lg2(float x) { return __int_as_float(0x4b400000 + (int)((__float_as_uint(x) + 0x7fffffu) >> 23) - 127) - 12582912.f; }
__device__ __forceinline__ float lg2(float x, float whole) {
  const uint32_t m = __float_as_uint(x) & 0x7fffffu;
  if (m) {
    float y;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(__uint_as_float(m | 0x3f800000u)));
    whole += y - 1.f;
  }
  return whole;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t w;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(hi), "f"(lo));
  return w;
}
__device__ __forceinline__ float2 unpack_f16(uint32_t w) { return __half22float2(*reinterpret_cast<__half2*>(&w)); }
// What rounding a pair to FP16 leaves over, in FP16, 2^UP times as much.
template <int UP = 0>
__device__ __forceinline__ uint32_t rest_f16(float lo, float hi, uint32_t w) {
  const float2 f = unpack_f16(w);
  return pack_f16((lo - f.x) * (float)(1 << UP), (hi - f.y) * (float)(1 << UP));
}
__device__ __forceinline__ uint32_t times_f16(uint32_t w, float f) {
  const __half2 x = __hmul2(*reinterpret_cast<const __half2*>(&w), __float2half2_rn(f));
  return *reinterpret_cast<const uint32_t*>(&x);
}
__device__ __forceinline__ void mma_f16(float* d, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// The same from c0 in its first row and c1 in its second.
__device__ __forceinline__ void mma_f16_from(float* d, const uint32_t* a, uint32_t b0, uint32_t b1, float c0, float c1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %11, %11};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(c0), "f"(c1));
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
// The same for the first product, which takes multiples of them plus a bias: (code + BIAS) / 2^FACTOR_BITS, with BIAS times the sum of a row's query (and
// its sign) where the product starts from.  INT8's c + 128 alone in FP16's low byte is that many times 2^-24, which saves a subtraction per pair and
// costs a bit of the sum; FP32 queries take the codes as they are (their error would double: 5e-7 to 1.2e-6).
template <typename F, bool WIDE> struct KeyCodes {
  static constexpr float BIAS = 0.f;
  static constexpr int FACTOR_BITS = 0;
  static __device__ __forceinline__ void f16(uint32_t w, uint32_t& lo, uint32_t& hi) { codes_f16(F(), w, lo, hi); }
};
template <> struct KeyCodes<Int8, false> {
  static constexpr float BIAS = 128.f;
  static constexpr int FACTOR_BITS = 24;
  static __device__ __forceinline__ void f16(uint32_t w, uint32_t& lo, uint32_t& hi) {
    w ^= 0x80808080u;
    lo = __byte_perm(w, 0u, 0x4140);
    hi = __byte_perm(w, 0u, 0x4342);
  }
};
__device__ __forceinline__ void cp4(void* smem_dst, const void* gmem_src) {
  const uint32_t s = static_cast<uint32_t>(__cvta_generic_to_shared(smem_dst));
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(s), "l"(gmem_src) : "memory");
}

// Key (of a unit) that column n of score tile nt stands for.  The scores of a thread's columns 2c, 2c + 1 in tiles 2j, 2j + 1 are, as they lie, its
// part of the probabilities' operand of the second product; this order makes them keys 16 j + c + {0, 4, 8, 12}, which reads values without bank conflicts.
__device__ __forceinline__ int unit_key(int nt, int n) { return 16 * (nt >> 1) + (n >> 1) + 4 * ((nt & 1) * 2 + (n & 1)); }

// What a warp keeps of its rows (thread's row g of each eight) between units.
template <int NQ>
struct Softmax {
  float m[NQ], d[NQ], l[NQ];           // reference of the scores, exponent of probability * scale beyond it, sum of probabilities
  float up[NQ][2], down[NQ][2];        // what goes on a score, and the power of two that a sum of what comes out is multiplied by
  float ve[2], vs_of[2];               // log2 of the values' scales of the last unit, rounded up, and these
  bool large;                          // scores whose steps in FP32 are a quarter and more
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      m[q] = d[q] = -INFINITY;
      l[q] = up[q][0] = up[q][1] = down[q][0] = down[q][1] = 0.f;
    }
    ve[0] = ve[1] = 0.f;
    vs_of[0] = vs_of[1] = -1.f;
    large = false;
  }
};
constexpr float SPAN = 100.f;           // exponents that values' scales may be apart from p * scale's reference: 2^(15 + SPAN) and its inverse are FP32 numbers
constexpr int REST_UP = 11;             // FP32's second operands are taken this many binary places up, and meet values that far down: steps of 2^-35
// How far above a new largest score references are put, so that fewer units move them: each place is one that small probabilities lose at FP16's lower end.
// BF16: 2, which keeps keys that another one leads by 20 nats to BF16's half step (32 x 64 queries: none 137 us, 2 or 3 134, 8 130); FP32: none (161 us, 8 157).
__host__ __device__ constexpr float att_slack(bool fp32) { return fp32 ? 0.f : 2.f; }
// A unit's probabilities from its scores s (times tk: exponents), masked ones -inf: pf [score tile] holds two keys' of row g, times their values' scale
// vs0 (TWO: the second half's vs1) as described below, ready to be the second product's operand.  Results acc move along when a reference does.
template <int NQ, int ND, bool TWO, bool WIDE>
__device__ __forceinline__ void probabilities(Softmax<NQ>& st, float (&s)[(NQ + 1) / 2][4][4], float (&tk)[NQ][2], float vs0, float vs1, float (&acc)[NQ][ND][4],
                                              uint32_t (&pf)[WIDE ? 2 : 1][NQ][4], int c) {
  constexpr float SLACK = att_slack(WIDE);
  // has any row a new maximum, or its values' scale another exponent?
  const bool other_scale = vs0 != st.vs_of[0] || (TWO && vs1 != st.vs_of[1]);
  bool moved = false;
  if (other_scale) {
    st.vs_of[0] = vs0;
    st.ve[0] = whole_lg2(vs0);
    if (TWO) { st.vs_of[1] = vs1; st.ve[1] = whole_lg2(vs1); }
    const float least = (TWO ? fmaxf(st.ve[0], st.ve[1]) : st.ve[0]) - SPAN;
#pragma unroll
    for (int q = 0; q < NQ; ++q) moved |= least > st.d[q];
  }
  float x[NQ][2];
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
    }
    x[q][0] = ceilf(x0 * tk[q][0]);                  // references are whole numbers: what goes from one to another is an exact power of two
    x[q][1] = TWO ? ceilf(x1 * tk[q][1]) : x[q][0];
    moved |= x[q][0] > st.m[q] || x[q][0] - st.m[q] + st.ve[0] > st.d[q];
    if (TWO) moved |= x[q][1] > st.m[q] || x[q][1] - st.m[q] + st.ve[1] > st.d[q];
  }
  moved = __any_sync(0xffffffffu, moved);
  if (moved) {
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      // reference st.m of the row's scores, and exponent st.d of p * scale beyond st.m's own
      const float most = TWO ? fmaxf(x[q][0], x[q][1]) : x[q][0];
      const float top = most > st.m[q] ? most + SLACK : st.m[q], ref = top == -INFINITY ? 0.f : top, less = st.m[q] - ref;
      const float with = TWO ? fmaxf(x[q][0] - ref + st.ve[0], x[q][1] - ref + st.ve[1]) : x[q][0] - ref + st.ve[0];
      const float tod = fmaxf(with > st.d[q] + less ? with + SLACK : st.d[q] + less, (TWO ? fmaxf(st.ve[0], st.ve[1]) : st.ve[0]) - SPAN);
      const float keep_o = tod == -INFINITY ? 0.f : ex2(less + (st.d[q] - tod));
      st.m[q] = top;
      st.d[q] = tod;
      st.l[q] *= ex2(less);
      const float k0 = __shfl_sync(0xffffffffu, keep_o, 8 * c), k1 = __shfl_sync(0xffffffffu, keep_o, 8 * c + 4);
#pragma unroll
      for (int i = 0; i < ND; ++i) {
        const float2 y0 = mul2(make_float2(acc[q][i][0], acc[q][i][1]), make_float2(k0, k1)), y1 = mul2(make_float2(acc[q][i][2], acc[q][i][3]), make_float2(k0, k1));
        acc[q][i][0] = y0.x; acc[q][i][1] = y0.y; acc[q][i][2] = y1.x; acc[q][i][3] = y1.y;
      }
      st.large |= fabsf(ref) > 4194304.f;
    }
    st.large = __any_sync(0xffffffffu, st.large);
  }
  if (moved || other_scale) {
    // p, as a share of the softmax's maximum, goes into the second product times 2^(15 + e), e = log2(values' scale) - st.d.  Its sum is taken as it is
    // and brought back afterwards, which the bounds on e keep inside FP32: at -SPAN values do not count, and SPAN is as far as the reference lets them go.
#pragma unroll
    for (int z = 0; z < (TWO ? 2 : 1); ++z) {
      const float ve = lg2(st.vs_of[z], st.ve[z]);
#pragma unroll
      for (int q = 0; q < NQ; ++q) {
        const float e = (float)P_BITS + fminf(fmaxf(ve - st.d[q], -SPAN), SPAN);
        st.up[q][z] = st.m[q] == -INFINITY ? e : e - st.m[q];
        st.down[q][z] = ex2(-e);
      }
    }
  }
  float from[NQ][TWO ? 2 : 1];
#pragma unroll
  for (int q = 0; q < NQ; ++q)
#pragma unroll
    for (int z = 0; z < (TWO ? 2 : 1); ++z) from[q][z] = st.up[q][z];
  if (st.large) {                                       // scores in steps of a quarter and more: a difference of rounded ones, as the maximum is one of them
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      const float ref = st.m[q] == -INFINITY ? 0.f : st.m[q];
#pragma unroll
      for (int nt = 0; nt < 4; ++nt)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          float& v = s[q / 2][nt][2 * (q & 1) + j];
          v = __fsub_rn(__fmul_rn(v, tk[q][nt >> 1]), ref);
        }
      tk[q][0] = tk[q][1] = 1.f;
#pragma unroll
      for (int z = 0; z < (TWO ? 2 : 1); ++z) from[q][z] = -log2f(st.down[q][z]);
    }
  }
#pragma unroll
  for (int q = 0; q < NQ; ++q)
#pragma unroll
    for (int z = 0; z < 2; ++z) {
      const int zz = TWO ? z : 0;
      const float2 t2 = make_float2(tk[q][zz], tk[q][zz]), r2 = make_float2(from[q][zz], from[q][zz]);
      float2 sum;
#pragma unroll
      for (int nt = 2 * z; nt < 2 * z + 2; ++nt) {
        float2 y = fma2(make_float2(s[q / 2][nt][2 * (q & 1)], s[q / 2][nt][2 * (q & 1) + 1]), t2, r2);
        y.x = ex2(y.x);
        y.y = ex2(y.y);
        sum = nt == 2 * z ? y : add2(sum, y);
        pf[0][q][nt] = pack_f16(y.x, y.y);
        if constexpr (WIDE) pf[WIDE ? 1 : 0][q][nt] = rest_f16<REST_UP>(y.x, y.y, pf[0][q][nt]);
      }
      st.l[q] = fmaf(sum.x + sum.y, st.down[q][zz], st.l[q]);
    }
}

// Attention of 8 NQ rows (queries of one row of the batch times the query heads that share a key/value head) over a part of the row's keys.
//
// What a number goes through.  Codes are exact in FP16.  Queries are brought to 2^13 by a power of two of their row: BF16 is exact then, and FP32 goes in as two
// FP16 numbers, 22 bits, both down to 2^-38 of the row's largest number.  Scores are FP32: the keys' scale, the softmax scale and the query's power
// of two come in one factor per block and row.  Probabilities meet the values' scale before they are rounded: p * vs, as a multiple of its largest
// value so far in the row (2^d times what the softmax's own reference m stands for), times 2^15, so that blocks' scales may be far apart.  FP16's steps
// end at 2^-24, and with them what is left of small ones: BF16's have 11 bits down to 2^-26 of the largest in their row and steps of 2^-36 of it below, FP32's, whose second
// number is taken 2^11 times and meets values of 2^-11 for it, 22 bits down to 2^-27 and steps of 2^-49.  References are whole exponents, so that results
// go from one to another by exact powers of two.  Sums and results are FP32.
//
// Why this shape.  What has to be read is 2 * dim bytes a key; 16 rows make 64 operations a byte of it, which mma.sync delivers several times over, so the kernel
// is a stream of the cache with as little as possible per byte: each warp copies its own units of 32 keys through its own ring in shared memory
// (16-byte asynchronous copies, zeros where no key is), nothing but __syncwarp between them, and keeps maximum, sum and result in registers until its
// keys are through; the four warps' results are joined at the end.  The 16-byte pieces lie in shared memory so that both products' operands come out
// of it whole, in the registers where mma wants them, without a transposition: dims and keys may be summed in any order.
// What it measured (BF16 queries, whole calls one after the other): one query on 200001 keys, 32 query heads on 8 of 128, INT8, 84 to 100 us by GPU, 4.1 to
// 4.9 TB/s, 81 of them this kernel at 5.1 TB/s, bound by DRAM and the ends; 16 rows of 3 to 8 queries on 6000 to 32000 keys, the same heads, E4M3, 166 to 176 us, 3.7 TB/s
// at 49 % of mma.sync's rate: 32 rows take 255 registers, two warps a scheduler that wait for their own instructions more than for anything else, so that neither pipe is
// full; 32 rows of 17 to 64 queries on 200 to 4000 keys, 16 heads of 64, INT8, 138 us (120 with another kernel between the calls), of which 115 here, two tiles of rows
// reading the keys.  FP32 queries: 161, 246 and 93 us.
// Tried and slower: codes turned into FP16 in shared memory once for 64 rows by the whole CTA (ldmatrix, a barrier every 64 keys), 117 -> 147 us;
// 16 rows a CTA at three CTAs an SM, 127 -> 136 and 178 -> 200; 32 rows at two CTAs an SM without spills (64 wide), 127 -> 137.
// TWO: blocks of 16 tokens, two in a unit.
// grid = as many as are resident at once, or as there are granules; block = 32 * ATT_WARPS.
template <typename T, typename F, int DIM, int NQ, bool TWO>
__global__ void __launch_bounds__(32 * ATT_WARPS, att_resident(DIM, NQ))
cache_attention_kernel(AttendParams a) {
  constexpr bool WIDE = sizeof(T) == 4;               // two FP16 numbers for each query and probability
  constexpr int HL = WIDE ? 2 : 1;
  typedef KeyCodes<F, WIDE> Keys;
  constexpr int KSTEPS = DIM / 16, ND = DIM / 16, MT = (NQ + 1) / 2, ROWS = 8 * NQ;
  constexpr int STAGES = att_stages(DIM, NQ), STAGE = att_stage_bytes(DIM), COPIES = DIM / 16;
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ float2 s_rf[ROWS];                       // factor of a row's scores, and what its first product starts from
  __shared__ float s_rest[ROWS];                      // power of two that the factor has no room for; one in all but the oddest of rows
  uint4* sq = reinterpret_cast<uint4*>(smem);          // [HL][MT][KSTEPS][lane]: operands as mma wants them
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, c = lane & 3;
  unsigned char* ring = smem + att_q_bytes(DIM, NQ, WIDE) + warp * STAGES * STAGE;
  __shared__ int s_vis[ROWS];
  __shared__ Segment s_seg;
  pdl_launch();
  pdl_wait();
  long long g0, g1;
  if (!find_share(a, ROWS, s_seg, g0, g1)) return;
  const int group = a.n_heads / a.c.heads;
  // What the loop over keys has no use for stays in shared memory meanwhile, for the sake of its registers.
  for (;;) {
    __syncthreads();
    const SegmentKeys view = open_segment(a, ROWS, s_seg, s_vis, g1);
    const int kvh = view.kvh, r0 = view.r0, r_last = view.r_last, vis_min = view.vis_min, vis_max = view.vis_max, n_units = view.u1 - view.u0;
    const int u0 = view.u0 + (int)((long long)n_units * warp / ATT_WARPS), u1 = view.u0 + (int)((long long)n_units * (warp + 1) / ATT_WARPS);      // this warp's
    const int b = s_seg.b;

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
    uint64_t policy;
    if (a.stream_once) asm("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));
    else asm("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(policy));
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
      auto k_to = [&](int i) { return (DIM == 128 && (i & 1) ? k_odd : k_dst) + so + (DIM == 128 ? (16 * (i >> 2) + 8 * ((i >> 1) & 1) + (i & 1)) * DIM : i * 512); };
      auto from = [&](int i) { return i * 512 + (TWO && i >= COPIES / 2 ? second : 0); };
      constexpr int SCALES = TWO ? 4 : 2;                           // ks0, ks1, vs0, vs1 (without a second block, the first of each)
      const int slot = TWO ? lane : 2 * lane, z = TWO ? lane & 1 : 0;
      float* scale_dst = reinterpret_cast<float*>(ring + stage * STAGE + 2 * UNIT * DIM) + slot;
      const float* scale_src = (slot < 2 ? a.c.scale[0] : a.c.scale[1]) + (z ? tile[1] : tile[0]);
      if (first + UNIT <= vis_max && there[0] && (!TWO || there[1])) {
#pragma unroll
        for (int i = 0; i < COPIES; ++i) {
          asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2;" ::"r"(k_to(i)), "l"(ks + from(i)), "l"(policy) : "memory");
          asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2;" ::"r"(v_dst + so + i * 512), "l"(vs + from(i)), "l"(policy) : "memory");
        }
        if (lane < SCALES) cp4(scale_dst, scale_src);
      } else {                                                      // zeros where there is no key; a block that is not there: a negative scale
#pragma unroll
        for (int i = 0; i < COPIES; ++i) {
          const int n = there[TWO && i >= COPIES / 2 ? 1 : 0] && first + my_key + i * (512 / DIM) < vis_max ? 16 : 0;
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(k_to(i)), "l"(ks + from(i)), "r"(n) : "memory");
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(v_dst + so + i * 512), "l"(vs + from(i)), "r"(n) : "memory");
        }
        if (lane < SCALES) {
          const bool need = first + 16 * z < vis_max;
          if (need && (z ? there[1] : there[0])) cp4(scale_dst, scale_src);
          else *scale_dst = need && slot < 2 ? -1.f : 1.f;
        }
      }
    };
    // ---- queries, a few rows a warp: under way first ----
    constexpr int PER = DIM / 32, Q_ROWS = 16 * MT / ATT_WARPS;
    T qx[Q_ROWS][PER];
#pragma unroll
    for (int k = 0; k < Q_ROWS; ++k) {
      const int r = warp + k * ATT_WARPS, row = r0 + r;
#pragma unroll
      for (int i = 0; i < PER; ++i) qx[k][i] = from_f32<T>(0.f);
      if (r < ROWS && row <= r_last) {
        const T* q = static_cast<const T*>(a.q) + (size_t)(s_seg.work.o + row / group) * a.q_stride + ((size_t)kvh * group + row % group) * DIM + lane * PER;
#pragma unroll
        for (int i = 0; i < PER; ++i) qx[k][i] = q[i];
      }
    }
    look_up(u0);
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s) {
      issue(u0 + s, s);
      asm volatile("cp.async.commit_group;" ::: "memory");
    }

    // The row's power of two, FP16, into operand order.
    // Thread's dims in step j: 64 (j / 4) + 16 c + 4 (j % 4) + 0 .. 3 (DIM = 32: 8 c + 4 j + 0 .. 3)
#pragma unroll
    for (int k = 0; k < Q_ROWS; ++k) {
      const int r = warp + k * ATT_WARPS;
      float x[PER], top = 0.f;
#pragma unroll
      for (int i = 0; i < PER; ++i) { x[i] = to_f32(qx[k][i]); top = fmaxf(top, fabsf(x[i])); }
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
        if constexpr (Keys::BIAS != 0.f) {
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
      if (lane == 0 && r < ROWS) s_rf[r] = make_float2(__int_as_float((int)e), total);
    }
    __syncthreads();
    int odd = 0;                                        // whether any row of the tile has a rest
    if (tid < ROWS) {
      // scale / up * 2^FACTOR_BITS: the part within 2^-120 .. 2^121 meets the keys' scale first, what is left of the powers of two their product
      const float2 v = s_rf[tid];
      const int power = __float_as_int(v.x) - 140 + Keys::FACTOR_BITS, room = 247 - (int)(__float_as_uint(a.scale) >> 23), first = min(max(power, room - 240), room);
      s_rf[tid] = make_float2(ldexpf(a.scale, first), -Keys::BIAS / (float)(1 << Keys::FACTOR_BITS) * v.y);
      s_rest[tid] = ldexpf(1.f, power - first);
      odd = power != first;
    }
    // The loop's branch for units that some row does not see whole is the one for tiles with a rest, too.
    const int whole_until = __syncthreads_or(odd) ? 0 : vis_min;
    // Scores: thread's row g of each eight, columns as above.  Results: dims DIM / 8 * g .. of rows 2 c and 2 c + 1 of each eight.
    constexpr bool ROW_REGS = NQ < 4;                   // (with 32 rows registers are short: read again for every unit)
    float2 row_rf[NQ];
    float acc[NQ][ND][4];
    Softmax<NQ> soft;
    soft.clear();
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      if (ROW_REGS) row_rf[q] = s_rf[q * 8 + g];
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
      float rf[NQ], start[NQ];
#pragma unroll
      for (int q = 0; q < NQ; ++q) {
        const float2 v = ROW_REGS ? row_rf[q] : s_rf[q * 8 + g];
        rf[q] = v.x;
        start[q] = Keys::BIAS != 0.f ? v.y : 0.f;
      }
      float s[MT][4][4];
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
            Keys::f16(raw[nt][j], b0, b1);
#pragma unroll
            for (int h = HL - 1; h >= 0; --h)
#pragma unroll
              for (int t = 0; t < MT; ++t) {
                const uint32_t* qa = reinterpret_cast<const uint32_t*>(&qf[h][t]);
                if (hh == 0 && j == 0 && h == HL - 1) mma_f16_from(s[t][nt], qa, b0, b1, start[2 * t], start[2 * t + 1 < NQ ? 2 * t + 1 : 2 * t]);
                else mma_f16(s[t][nt], qa, b0, b1);
              }
          }
        }
      }
      float tk[NQ][2];
#pragma unroll
      for (int q = 0; q < NQ; ++q) {
        tk[q][0] = rf[q] * fabsf(sc.x);
        tk[q][1] = TWO ? rf[q] * fabsf(sc.y) : tk[q][0];
      }
      if (u * UNIT + UNIT > whole_until || sc.x < 0.f || (TWO && sc.y < 0.f)) {
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
#pragma unroll
          for (int nt = 0; nt < 4; ++nt)
#pragma unroll
            for (int j = 0; j < 2; ++j)
              if (u * UNIT + unit_key(nt, 2 * c + j) >= s_vis[q * 8 + g] || (TWO && nt >= 2 ? sc.y : sc.x) < 0.f) s[q / 2][nt][2 * (q & 1) + j] = -INFINITY;
          const float rest = s_rest[q * 8 + g];
          tk[q][0] = fmaxf(tk[q][0] * rest, FLT_MIN);    // (not 0 times -inf)
          tk[q][1] = TWO ? fmaxf(tk[q][1] * rest, FLT_MIN) : tk[q][0];
        }
      }
      // ---- probabilities ----
      uint32_t pf[HL][NQ][4];
      probabilities<NQ, ND, TWO, WIDE>(soft, s, tk, sc.z, sc.w, acc, pf, c);
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
            if constexpr (WIDE) {
              uint32_t down[4];                          // (E4M3's smallest is 2^-9, so that these are exact)
#pragma unroll
              for (int i = 0; i < 4; ++i) down[i] = times_f16(av[i], 1.f / (1 << REST_UP));
#pragma unroll
              for (int q = 0; q < NQ; ++q) mma_f16(acc[q][2 * x + y], down, pf[HL - 1][q][2 * j], pf[HL - 1][q][2 * j + 1]);
            }
#pragma unroll
            for (int q = 0; q < NQ; ++q) mma_f16(acc[q][2 * x + y], av, pf[0][q][2 * j], pf[0][q][2 * j + 1]);
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
      float sum = soft.l[q];
      sum += __shfl_xor_sync(0xffffffffu, sum, 1);
      sum += __shfl_xor_sync(0xffffffffu, sum, 2);
      if (c == 0) {
        const int r = warp * ROWS + q * 8 + g;
        sm[r] = soft.m[q]; sl[r] = sum; sd[r] = soft.d[q];
      }
    }
    __syncthreads();
    store_results<T, DIM, ROWS, ATT_WARPS, PITCH>(a, s_seg, g0, so, sm, sl, sd);
    if (!next_segment(a, ROWS, s_seg, g1)) break;
  }
}

// Joins the parts of items that more than one CTA worked on.  Four dims a thread, so that 128 threads are 128 / (DIM / 4) groups: SHARED, they take a
// row's parts in turn, else each has a row of its own; parts are added up in their order.  Bound by latency: SHARED, maxima and sums of all parts are
// loaded at once and results eight parts ahead.
// grid = (rows, or rows / groups, heads, B), block = 128; dynamic shared memory (SHARED): a float per CTA of the attention.
template <typename T, int DIM, int NQ, bool SHARED>
__global__ void __launch_bounds__(128)
cache_attention_join_kernel(AttendParams a) {
  constexpr int ROWS = 8 * NQ, LANES = DIM / 4, GROUPS = 128 / LANES;
  extern __shared__ float s_w[];
  __shared__ float4 s_x[SHARED ? GROUPS - 1 : 1][LANES];
  __shared__ float s_red[2][4];
  pdl_launch();
  pdl_wait();
  const int tid = threadIdx.x, lane = tid & 31, grp = tid / LANES, d0 = tid % LANES * 4;
  const int b = blockIdx.z, kvh = blockIdx.y, r = SHARED ? blockIdx.x : blockIdx.x * GROUPS + grp;
  const long long total = __ldcg(a.prefix + a.B), in_front = __ldcg(a.prefix + b);
  const RowWork work = row_work(a, b, ROWS);
  const int group = a.n_heads / a.c.heads;
  if (work.granules == 0 || r >= work.n * group || work.pieces == 1) return;
  const long long ctas = min((long long)a.grid, total);
  const long long first = in_front + ((long long)kvh * work.tiles + r / ROWS) * work.pieces;
  const int c0 = cta_of(total, first, ctas), parts = cta_of(total, first + work.pieces - 1, ctas) - c0 + 1;
  if (parts == 1) return;
  // the first CTA's part is its last segment unless it starts there; the others' are their first
  const int slot0 = 2 * c0 + (cta_start(total, c0, ctas) < first ? 1 : 0);
  const int rr = r % ROWS;
  auto row_of = [&](int i) { return (size_t)(i == 0 ? slot0 : 2 * (c0 + i)) * ROWS + rr; };
  const float2* ml = reinterpret_cast<const float2*>(a.part + 2 * (size_t)a.grid * ROWS * DIM);
  float sum = 0.f;
  float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
  auto add = [&](float4 y, float f) { x.x = fmaf(y.x, f, x.x); x.y = fmaf(y.y, f, x.y); x.z = fmaf(y.z, f, x.z); x.w = fmaf(y.w, f, x.w); };
  if constexpr (SHARED) {
    constexpr int AHEAD = 8;
    auto load_parts = [&](float4* y, int s0) {
#pragma unroll
      for (int i = 0; i < AHEAD; ++i)
        if (s0 + i * GROUPS < parts) y[i] = __ldcg(reinterpret_cast<const float4*>(a.part + row_of(s0 + i * GROUPS) * DIM + d0));
    };
    float4 y[AHEAD];
    load_parts(y, grp);                          // (on their way while the weights are worked out)
    float2 v = tid < parts ? __ldcg(ml + row_of(tid)) : make_float2(-INFINITY, 0.f);
    float top = v.x;
    for (int i = tid + 128; i < parts; i += 128) top = fmaxf(top, __ldcg(ml + row_of(i)).x);
#pragma unroll
    for (int w = 16; w; w >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
    if (lane == 0) s_red[0][tid >> 5] = top;
    __syncthreads();
    top = fmaxf(fmaxf(s_red[0][0], s_red[0][1]), fmaxf(s_red[0][2], s_red[0][3]));
    for (int i = tid; i < parts; i += 128) {
      if (i > tid) v = __ldcg(ml + row_of(i));
      const float f = v.y == 0.f ? 0.f : v.x == top ? v.y : v.y * ex2(v.x - top);      // (no key: nothing, whatever the maxima)
      s_w[i] = f;
      sum += f;
    }
#pragma unroll
    for (int w = 16; w; w >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, w);
    if (lane == 0) s_red[1][tid >> 5] = sum;
    __syncthreads();
    sum = (s_red[1][0] + s_red[1][1]) + (s_red[1][2] + s_red[1][3]);
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    for (int s0 = grp; s0 < parts; s0 += AHEAD * GROUPS) {
#pragma unroll
      for (int i = 0; i < AHEAD; ++i)
        if (s0 + i * GROUPS < parts) add(y[i], s_w[s0 + i * GROUPS] * inv);
      load_parts(y, s0 + AHEAD * GROUPS);
    }
    if (grp > 0) s_x[grp - 1][tid % LANES] = x;
    __syncthreads();
    if (grp > 0) return;
#pragma unroll
    for (int i = 0; i < GROUPS - 1; ++i) add(s_x[i][tid], 1.f);
  } else {
    float top = -INFINITY;
    for (int i = 0; i < parts; ++i) {
      const float2 v = __ldcg(ml + row_of(i));
      if (v.y == 0.f) continue;                  // (no key: nothing, whatever the maxima)
      const float most = fmaxf(top, v.x);
      sum = v.x == top ? sum + v.y : fmaf(sum, ex2(top - most), v.x == most ? v.y : v.y * ex2(v.x - most));
      top = most;
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll 4
    for (int i = 0; i < parts; ++i) {
      const float2 v = __ldcg(ml + row_of(i));
      const float4 y = __ldcg(reinterpret_cast<const float4*>(a.part + row_of(i) * DIM + d0));
      if (v.y == 0.f) continue;
      add(y, (v.x == top ? v.y : v.y * ex2(v.x - top)) * inv);
    }
  }
  T* out = static_cast<T*>(a.out) + ((size_t)(work.o + r / group) * a.n_heads + kvh * group + r % group) * DIM + d0;
  if constexpr (sizeof(T) == 4) {
    *reinterpret_cast<float4*>(out) = x;
  } else {
    __nv_bfloat162 w[2] = {__floats2bfloat162_rn(x.x, x.y), __floats2bfloat162_rn(x.z, x.w)};
    *reinterpret_cast<uint2*>(out) = *reinterpret_cast<const uint2*>(w);
  }
}

}  // namespace kv
}  // namespace ad
