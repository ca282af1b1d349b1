// Sampling of tokens with temperature, top-k, top-p and min-p from given random numbers.
#pragma once

#include <cooperative_groups.h>
#include <math.h>

#include "kv_cache.cuh"

namespace ad {
namespace sample {

namespace cg = cooperative_groups;

constexpr int THREADS = 512, WARPS = THREADS / 32, MAX_CLUSTER = 8;
constexpr int DIGIT = 11, BINS = 1 << DIGIT, PER = BINS / THREADS;      // bins of a histogram, and of a thread
constexpr int HALF = 2048, VALUES = 2 * HALF;      // BF16 numbers of either sign that have a bin of their own
constexpr int LIST = 4096;             // scores of one bin that are put in order
typedef unsigned long long u64;

struct Params {
  const void* scores;            // [M, vocab], rows `stride` scores apart
  size_t stride;
  int vocab, M;
  const float* temperature;      // [M] or null (one); the same for the others (no such filter)
  const int* top_k;
  const float* top_p;
  const float* min_p;
  const float* r;                // [M]
  int* tokens;                   // [M]
  float* logp;                   // [M] or null
  void* out;                     // [M, vocab] or null
  size_t out_stride;
  int scale_bits;                // weights are counted in units of 2^-scale_bits
  int each;                      // scores of a warp, a multiple of 32 vectors
  int* status;
};

// Scores as integers in the same order, 0.0 and -0.0 alike.  BF16's are 16 bits wide.
template <typename T> struct Key;
template <> struct Key<float> {
  static constexpr int BITS = 32;
  static __device__ __forceinline__ uint32_t of(float x) {
    const uint32_t u = __float_as_uint(x + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
  }
};
template <> struct Key<bf16> {
  static constexpr int BITS = 16;
  static __device__ __forceinline__ uint32_t of(float x) { return Key<float>::of(x) >> 16; }
};
template <typename T> __device__ __forceinline__ T clean(T x) { return to_f32(x) == to_f32(x) ? x : from_f32<T>(-INFINITY); }     // a NaN counts as -inf
// Vectors of 16 bytes: as FP32 numbers, their largest, and whether a NaN is among them.
__device__ __forceinline__ void unpack(uint4 v, float (&x)[4]) { x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y); x[2] = __uint_as_float(v.z); x[3] = __uint_as_float(v.w); }
__device__ __forceinline__ void unpack(uint4 v, float (&x)[8]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
}
__device__ __forceinline__ float largest(uint4 v, float) {
  return fmaxf(kv::max3(__uint_as_float(v.x), __uint_as_float(v.y), __uint_as_float(v.z)), __uint_as_float(v.w));
}
__device__ __forceinline__ float largest(uint4 v, bf16) {
  const __nv_bfloat162* p = reinterpret_cast<const __nv_bfloat162*>(&v);
  const __nv_bfloat162 m = __hmax2(__hmax2(p[0], p[1]), __hmax2(p[2], p[3]));
  return fmaxf(__low2float(m), __high2float(m));
}
// Which of a vector's are x, a bit each.
__device__ __forceinline__ uint32_t equal(uint4 v, float x, float) {
  return (__uint_as_float(v.x) == x ? 1u : 0u) | (__uint_as_float(v.y) == x ? 2u : 0u) | (__uint_as_float(v.z) == x ? 4u : 0u) | (__uint_as_float(v.w) == x ? 8u : 0u);
}
__device__ __forceinline__ uint32_t equal(uint4 v, float x, bf16) {
  const __nv_bfloat162* p = reinterpret_cast<const __nv_bfloat162*>(&v);
  const __nv_bfloat162 y = __float2bfloat162_rn(x);
  const uint32_t m = (__heq2_mask(p[0], y) & 0x00020001u) | (__heq2_mask(p[1], y) & 0x00080004u) | (__heq2_mask(p[2], y) & 0x00200010u) | (__heq2_mask(p[3], y) & 0x00800040u);
  return (m | m >> 16) & 0xffu;
}
__device__ __forceinline__ bool has_nan(uint4 v, float) {
  return max(max(v.x & 0x7fffffffu, v.y & 0x7fffffffu), max(v.z & 0x7fffffffu, v.w & 0x7fffffffu)) > 0x7f800000u;
}
__device__ __forceinline__ bool has_nan(uint4 v, bf16) {
  const uint32_t m = __vmaxu2(__vmaxu2(v.x & 0x7fff7fffu, v.y & 0x7fff7fffu), __vmaxu2(v.z & 0x7fff7fffu, v.w & 0x7fff7fffu));
  return max(m & 0xffffu, m >> 16) > 0x7f80u;
}
// A key's score.
template <typename T> __device__ __forceinline__ float score_of(uint32_t key) {
  const uint32_t wide = Key<T>::BITS == 16 ? key << 16 | (key & 0x8000u ? 0u : 0xffffu) : key;
  return __uint_as_float(wide & 0x80000000u ? wide & 0x7fffffffu : ~wide);
}

// What has been counted: scores, or their weights in two halves.
struct Histogram { uint32_t lo[BINS], hi[BINS]; };
struct Found { int bin; u64 in_front, amount; };       // of scores, or of weight
// BF16 numbers from the largest on, one to a bin: the 16 octaves up to the largest magnitude that has any weight, 128 numbers each, of either sign.  The first bin of either
// sign holds all smaller magnitudes instead.  In shared memory a number that has a bin lies at its bits' distance from `first`, those of either sign in a half of their own; the last
// place of either half belongs to the first number without weight.
struct Values {
  int first;                     // bits of the smallest magnitude that has a bin
  __device__ __forceinline__ int distance(uint32_t bits) const { return (int)bits - first; }                   // of a score's 16 bits
  static __device__ __forceinline__ bool outside(int distance) { return (distance & 0x7800) != 0; }            // (of several at once, too: their bits together)
  static __device__ __forceinline__ int at(int distance) { return (distance & 0x7ff) | (distance >> 4 & 0x800); }
  __device__ __forceinline__ float value(int at) const { return __uint_as_float((uint32_t)((at & (HALF - 1)) + first + (at >= HALF ? 0x8000 : 0)) << 16); }
  // bins, and where they lie
  __device__ __forceinline__ int bin(float x) const {
    const int place = min(max((int)(__float_as_uint(x) >> 16 & 0x7fffu) - first + 1, 0), HALF - 1);
    return x < 0.f ? HALF + place : HALF - 1 - place;
  }
  static __device__ __forceinline__ bool small(int bin) { return bin == HALF || bin == HALF - 1; }
  static __device__ __forceinline__ int at_bin(int bin) { return bin < HALF ? HALF - 2 - bin : bin - 1; }
};
__device__ __forceinline__ uint32_t score_bits(uint4 v, int j) {      // BF16's
  const uint32_t w = j < 2 ? v.x : j < 4 ? v.y : j < 6 ? v.z : v.w;
  return j & 1 ? w >> 16 : w & 0xffffu;
}
struct Counts { static constexpr bool MASS = false; };      // what a search goes by
struct Mass { static constexpr bool MASS = true; };
struct Border { uint32_t key, kept, ties; };      // scores above this key stay, and of those that have it, `ties`, the first `kept`

// 64-bit sums from 32-bit atomic additions: exact, so that their order does not matter.  (Additions of 64 bits in shared memory are loops: 256 rows of 128000, top-p 384 -> 505 us.)
__device__ __forceinline__ void add_to(Histogram& h, uint32_t bin, u64 w) {
  const uint32_t l = (uint32_t)w, old = atomicAdd(&h.lo[bin], l), carry = old + l < old;
  const uint32_t up = (uint32_t)(w >> 32) + carry;
  if (up) atomicAdd(&h.hi[bin], up);
}
// Bin of a score x: by how far it lies below the largest, 128 to the octave, from 2^-7 to 2^9.  (Two infinities are no distance apart.)
__device__ __forceinline__ int bin_of(float top, float x) { return min(max((int)(__float_as_uint(fmaxf(top - x, 0.f)) >> 16) - (120 << 7), 0), BINS - 1); }

// Weights in units of 2^-bits, bits <= 51, to the last bits of FP64: w = 2^(k / 256) exp(f), k / 256 and f the whole 256ths and the rest of the exponent to the base of 2,
// the first from a table of 2^(j / 256) and the exponent, the second from its Taylor series up to f^4 (f^5 / 120 < 5e-17); the table-driven scheme of Tang (1989).
constexpr int EXP_TABLE = 256;
struct Weights {
  const double* table;
  double top, scale;             // largest score; 256 log2(e) / T
  float topf, half_top, far;     // largest score, half of it; half a distance that leaves no weight to speak of
  int bits;
  bool infinite;
  // Whether x has any weight to speak of: 2^-54 and less is none in these units.
  __device__ __forceinline__ bool any(float x) const { return fmaf(-0.5f, x, half_top) < far; }
  // Without branches, so that a vector's are worked out side by side.  (An infinite largest score takes all of it.)
  __device__ __forceinline__ u64 operator()(float x) const {
    const double ROUND = 6755399441055744.0;                                  // 1.5 * 2^52: the sum's low word is k
    const double z = ((double)x - top) * scale, kd = z + ROUND;
    const int k = __double2loint(kd);
    const double f = (z - (kd - ROUND)) * (0.693147180559945309417 / 256.0), t = table[k & (EXP_TABLE - 1)];
    double e = fma(f, 1.0 / 24.0, 1.0 / 6.0);
    e = fma(f, e, 0.5);
    e = fma(f, e, 1.0);
    e = fma(t * f, e, t);
    const double w = __hiloint2double(__double2hiint(e) + (((k >> 8) + bits) << 20), __double2loint(e)) + 4503599627370496.0;      // (2^52: the sum's low bits are w, rounded)
    const u64 u = (u64)__double_as_longlong(w) & 0xfffffffffffffull;
    return infinite ? (x == topf ? 1ull << bits : 0ull) : any(x) ? u : 0ull;
  }
  // w(x) >= least, in FP64; one is reached by the largest score alone, however close to it others' weights come
  __device__ __forceinline__ bool reaches(float x, double least) const {
    if (x == topf) return 1.0 >= least;
    if (infinite || x == -INFINITY) return 0.0 >= least;
    return least < 1.0 && exp(((double)x - top) * (scale * (0.693147180559945309417 / 256.0))) >= least;
  }
};

// One row by a cluster of CTAs that share the vocabulary, every warp a run of ids.
//   w(v) = exp((score(v) - largest) / T); tokens are ordered by score, ties by id.  Top-k keeps the first k; top-p, of these, the ones in front of
//   which less than top_p of their weight lies (and the first); min-p, of those, the ones with w >= min_p.  All three keep a beginning of the order, so that what
//   is kept is told by one score and the number of ids that are kept of those that have just this score.  The token is the lowest kept id at which
//   the running sum of weights, over kept ids in order, exceeds r times their total.
// The k-th largest score, and the one at which the weight in front reaches top_p of the whole: a histogram over the distance from the largest (in shared memory, summed
// over the cluster), the bin in which the border lies, and that bin's scores put in order by one CTA; where these are too many (ties, as a rule), digit
// by digit of their keys.  Weights are worked out in FP64 and summed as integers in units of 2^-scale_bits (vocab * 2^scale_bits <= 2^62): the largest is 1, so a
// sum is off by vocab * 2^-(scale_bits + 1) of itself at most, 2^-42 with 1000 ids and 2^-23 with 2^20 (roundings of either sign: their root, a 2^-10th
// of that, in fact), and comes out the same in any order.
// A row of FP32, or a short one, has every score's weight worked out, about 45 instructions; a long one of BF16 the weights of the 4096 numbers that lie within 16 octaves of the
// largest magnitude with any weight, once a CTA: top-p's histogram counts numbers then, its border is one of them, and what is kept is looked up.
// Bound by instructions and the cluster's barriers, about 0.7 us each: 256 rows of 128000 in BF16 (1024 CTAs, two an SM, four turns) take 90 us without a filter, 54 with min-p 0.05, 111 with
// top-k 50, 190 with top-p 0.9, 104 with both (one search; two: 140); reading them takes 10.  One row of 32000 in FP32: 14, 14, 15, 20 and 16 us.
// Scores are taken 16 bytes at a time: places g = id + shift, shift such that a place that is a multiple of a vector's lies on a vector's boundary.
// grid = M clusters, block = THREADS.  Dynamic shared memory: KEPT, the CTA's scores.
template <typename T, bool KEPT>
__global__ void __launch_bounds__(THREADS, 2)
sample_kernel(Params p) {
  constexpr int VEC = 16 / sizeof(T);
  extern __shared__ __align__(16) unsigned char s_raw[];
  __shared__ __align__(16) union { Histogram h; uint32_t count[VALUES]; u64 list[LIST], value[VALUES]; } s_u;
  __shared__ uint32_t s_small[2][2];                         // weight of small magnitudes of either sign, in halves
  __shared__ double s_table[EXP_TABLE];
  __shared__ float s_top[MAX_CLUSTER];
  __shared__ u64 s_warp[WARPS], s_scan[WARPS], s_sum[2][MAX_CLUSTER];
  __shared__ Found s_found, s_best[MAX_CLUSTER];
  __shared__ u64 s_chunk[MAX_CLUSTER];
  __shared__ Border s_border;
  __shared__ int s_n;
  Histogram& s_h = s_u.h;
  T* s_x = reinterpret_cast<T*>(s_raw);
  cg::cluster_group cluster = cg::this_cluster();
  const int rank = cluster.block_rank(), size = cluster.num_blocks(), m = blockIdx.x / size, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");      // (waited for before any other CTA's shared memory is written)
  pdl_launch();
  if (tid < EXP_TABLE) s_table[tid] = exp2(tid / (double)EXP_TABLE);
  pdl_wait();
  const T* row = static_cast<const T*>(p.scores) + (size_t)m * p.stride;
  T* out = p.out ? static_cast<T*>(p.out) + (size_t)m * p.out_stride : nullptr;
  const float temperature = p.temperature ? __ldg(p.temperature + m) : 1.f, top_p = p.top_p ? __ldg(p.top_p + m) : 1.f, min_p = p.min_p ? __ldg(p.min_p + m) : 0.f,
              r = __ldg(p.r + m);
  int top_k = p.top_k ? __ldg(p.top_k + m) : 0;
  const bool bad = !(temperature >= 0.f) || isinf(temperature) || top_p != top_p || min_p != min_p || r != r;
  const bool greedy = temperature == 0.f;
  if (greedy) top_k = 1;
  const double inv_t = greedy ? 1.0 : 1.0 / (double)temperature;

  // ---- places: the warp's g0 .. g1 - 1, of the CTA's c0 ..; scores at shift .. end - 1 ----
  const int shift = (int)(reinterpret_cast<uintptr_t>(row) / sizeof(T) % VEC), end = p.vocab + shift;
  const int each = p.each, c0 = rank * WARPS * each, g0 = c0 + warp * each, g1 = min(g0 + each, (end + VEC - 1) / VEC * VEC);
  const uint32_t nothing = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;      // -inf
  auto fetch = [&](int g) {                                    // VEC scores from memory, -inf where there are none
    uint4 v;
    const bool inside = g >= shift && g + VEC <= end;
    if (inside) v = *reinterpret_cast<const uint4*>(row + (g - shift));
    if (!inside || has_nan(v, T())) {
      T x[VEC];
#pragma unroll
      for (int j = 0; j < VEC; ++j) x[j] = g + j >= shift && g + j < end ? clean(row[g + j - shift]) : from_f32<T>(-INFINITY);
      v = *reinterpret_cast<const uint4*>(x);
    }
    return v;
  };
  // calls f(place of the first, VEC scores) by all lanes of the warp alike: lanes beyond the end get -inf
  auto sweep = [&](auto f) {
    for (int i0 = g0; i0 < g1; i0 += 32 * VEC) {
      const int g = i0 + lane * VEC;
      f(g, g >= g1 ? make_uint4(nothing, nothing, nothing, nothing) : KEPT ? *reinterpret_cast<const uint4*>(s_x + (g - c0)) : fetch(g));
    }
  };
  float top = -INFINITY;
#pragma unroll 4
  for (int g = g0 + lane * VEC; g < g1; g += 32 * VEC) {
    const uint4 v = fetch(g);
    if (KEPT) *reinterpret_cast<uint4*>(s_x + (g - c0)) = v;
    top = fmaxf(top, largest(v, T()));
  }
  const float my_top = top;                                    // the thread's own
#pragma unroll
  for (int w = 16; w; w >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
  if (lane == 0) s_warp[warp] = __float_as_uint(top);
  __syncthreads();
  top = lane < WARPS ? __uint_as_float((uint32_t)s_warp[lane]) : -INFINITY;
#pragma unroll
  for (int w = WARPS / 2; w; w >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
  top = __shfl_sync(0xffffffffu, top, 0);
  asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
  if (size > 1) {
    if (tid < size) cluster.map_shared_rank(s_top, tid)[rank] = top;
    cluster.sync();
    for (int j = 0; j < size; ++j) top = fmaxf(top, s_top[j]);
  }

  if (bad || top == -INFINITY) {                              // (all CTAs alike)
    if (out)
      for (int g = max(c0, shift) + tid; g < min(c0 + WARPS * each, end); g += THREADS) out[g - shift] = from_f32<T>(-INFINITY);
    if (rank == 0 && tid == 0) {
      if (bad) latch_error(p.status, AD_ERR_ARG);
      p.tokens[m] = bad ? -1 : 0;
      if (p.logp) p.logp[m] = -INFINITY;
    }
    return;
  }
  const Weights weight = {s_table, (double)top, inv_t * (256.0 / 0.693147180559945309417), top, 0.5f * top, (float)(19.0 / inv_t), p.scale_bits, isinf(top) != 0};
  const double unit = ldexp(1.0, p.scale_bits);

  // ---- sums over the cluster in the order of its warps: of x (alike in all lanes of a warp), in front of this warp, and all ----
  auto cluster_sum = [&](u64 x, u64& before, int which) {
    __syncthreads();
    if (lane == 0) s_warp[warp] = x;
    __syncthreads();
    u64 sum = lane < WARPS ? s_warp[lane] : 0, all = 0;
#pragma unroll
    for (int w = 1; w < WARPS; w <<= 1) {
      const u64 y = __shfl_up_sync(0xffffffffu, sum, w);
      if (lane >= w) sum += y;
    }
    const u64 mine = __shfl_sync(0xffffffffu, sum, WARPS - 1);
    before = __shfl_sync(0xffffffffu, sum, (warp + 31) & 31);
    if (warp == 0) before = 0;
    if (size == 1) return mine;
    if (tid < size) *cluster.map_shared_rank(&s_sum[which][rank], tid) = mine;
    cluster.sync();
    for (int j = 0; j < size; ++j) {
      const u64 y = s_sum[which][j];
      if (j < rank) before += y;
      all += y;
    }
    return all;
  };
  auto warp_sum = [&](u64 x) {
#pragma unroll
    for (int w = 16; w; w >>= 1) x += __shfl_xor_sync(0xffffffffu, x, w);
    return x;
  };
  // sums over the CTA in the order of its threads, in front of this one, and all
  auto cta_scan = [&](u64 x, u64& front, u64& all) {
    u64 run = x;
#pragma unroll
    for (int w = 1; w < 32; w <<= 1) {
      const u64 y = __shfl_up_sync(0xffffffffu, run, w);
      if (lane >= w) run += y;
    }
    __syncthreads();
    if (lane == 31) s_scan[warp] = run;
    __syncthreads();
    u64 sum = lane < WARPS ? s_scan[lane] : 0;
#pragma unroll
    for (int w = 1; w < WARPS; w <<= 1) {
      const u64 y = __shfl_up_sync(0xffffffffu, sum, w);
      if (lane >= w) sum += y;
    }
    all = __shfl_sync(0xffffffffu, sum, WARPS - 1);
    front = __shfl_sync(0xffffffffu, sum, (warp + 31) & 31);
    front = (warp ? front : 0) + run - x;
  };

  // ---- borders: of the scores above `from`, and the first from_n of those that have it (0: of all), where top-k's count or top-p's share of the weight ends ----
  // (Scores of -inf have no weight and are never among those; places that there are no scores for hold -inf.)
  // BF16 rows with more scores a CTA than there are bins: weights are worked out number by number, not score by score.  (256 rows of 128000, top-p: 189 us instead of 370; without
  // a filter 89 instead of 133.)
  const bool by_values = sizeof(T) == 2 && WARPS * each > VALUES;
  Values values = {0};
  if (by_values) {
    const float bottom = fmaxf(top - 2.1f * weight.far, -FLT_MAX);
    values.first = ((max((int)(__float_as_uint(fmaxf(fabsf(top), fabsf(bottom))) >> 23), 15) - 15) << 7) + 1;
  }
  uint32_t from = Key<T>::of(-INFINITY), from_n = 0;
  float from_x = -INFINITY;
  const bool by_k = top_k > 0 && top_k < p.vocab, by_p = top_p < 1.f;
  // Of n ties of weight w, those with front + j w below the goal, the very first in any case.
  auto ties_below = [&](u64 n, u64 w, u64 front, double goal) {
    if (w == 0) return n;
    const double want = (goal - (double)front) / (double)w;
    u64 t = want < 1.0 ? 1 : want >= (double)n ? n : (u64)want;
    while (t > 1 && !((double)(front + (t - 1) * w) < goal)) --t;
    while (t < n && (double)(front + t * w) < goal) ++t;
    return t;
  };
  // Digit by digit of the key: any number of ties, and as many rounds as digits.  Counts scores, or (by_mass) their weight.
  auto search_digits = [&](bool by_mass, double share, u64 k) {
    uint32_t prefix = 0;
    int above = Key<T>::BITS;                                  // bits below which the digit lies
    u64 in_front = 0;
    double goal = 0.0;
    Found f;
    while (above > 0) {
      const int bits = min(DIGIT, above), shr = above - bits;
      for (int i = tid; i < BINS; i += THREADS) s_h.lo[i] = s_h.hi[i] = 0;
      __syncthreads();
      const bool first_level = above == Key<T>::BITS;
      sweep([&](int g, uint4 v) {
        float x[VEC];
        unpack(v, x);
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          const uint32_t key = Key<T>::of(x[j]);
          if ((first_level || key >> above == prefix) && x[j] > from_x) add_to(s_h, key >> shr & ((1u << bits) - 1u), by_mass ? weight(x[j]) : 1ull);
        }
      });
      if (from_n != 0 && rank == 0 && tid == 0 && (first_level || from >> above == prefix))      // ties at the border found before: as many as were kept
        add_to(s_h, from >> shr & ((1u << bits) - 1u), by_mass ? weight(from_x) * from_n : from_n);
      cluster.sync();
      // a thread's bins, from the last one on
      u64 amount[PER], sum = 0;
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const int bin = BINS - 1 - (tid * PER + i);
        amount[i] = 0;
        for (int j = 0; j < size; ++j) {
          const Histogram* h = cluster.map_shared_rank(&s_h, j);
          amount[i] += ((u64)h->hi[bin] << 32) + h->lo[bin];
        }
        sum += amount[i];
      }
      u64 front, all;
      cta_scan(sum, front, all);
      front += in_front;
      if (first_level) goal = by_mass ? share * (double)all : (double)k;
      // the last bin that has any, and in front of which there is less than the goal (the first one in any case)
      if (tid == 0) s_found.bin = BINS;
      __syncthreads();
      int best = BINS;
      Found mine = {};
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const int bin = BINS - 1 - (tid * PER + i);
        if (amount[i] > 0 && (front == 0 || (double)front < goal)) {
          best = bin;
          mine = Found{bin, front, amount[i]};
        }
        front += amount[i];
      }
      if (best < BINS) atomicMin(&s_found.bin, best);
      __syncthreads();
      if (best < BINS && s_found.bin == best) s_found = mine;
      __syncthreads();
      f = s_found;
      in_front = f.in_front;
      prefix = prefix << bits | (uint32_t)f.bin;
      above = shr;
      cluster.sync();                                          // (histograms have been read)
    }
    const u64 w = by_mass ? weight(score_of<T>(prefix)) : 1, n = w ? f.amount / w : f.amount;
    return Border{prefix, (uint32_t)(by_mass ? ties_below(n, w, in_front, goal) : min(n, k - in_front)), (uint32_t)n};
  };
  // few: of the threads' own largest scores instead of all, whose k-th lies no higher than the k-th of all; what is in its bin and in front of it is put in order.
  auto search = [&](auto what, double share, u64 k, bool few) {
    constexpr bool by_mass = decltype(what)::MASS;
    const bool by_value = by_mass && by_values;
    auto small = [&](float x, u64 n) {                         // n of a score whose magnitude is small
      const u64 w = weight(x) * n;
      uint32_t* h = s_small[x < 0.f];
      const uint32_t l = (uint32_t)w, old = atomicAdd(h, l), carry = old + l < old;
      atomicAdd(h + 1, (uint32_t)(w >> 32) + carry);
    };
    for (int i = tid; i < BINS; i += THREADS) s_h.lo[i] = s_h.hi[i] = 0;
    if (tid < 4) s_small[tid >> 1][tid & 1] = 0;
    __syncthreads();
    if (few) {
      if (my_top > from_x) atomicAdd(&s_h.lo[bin_of(top, my_top)], 1u);
    } else if (__any_sync(0xffffffffu, my_top > from_x)) {
      sweep([&](int g, uint4 v) {
        if (!__any_sync(0xffffffffu, largest(v, T()) > from_x)) return;
        float x[VEC];
        unpack(v, x);
        if (by_value) {
          int d[VEC], any = 0;
#pragma unroll
          for (int j = 0; j < VEC; ++j) {
            d[j] = values.distance(score_bits(v, j));
            any |= d[j];
          }
          if (!__any_sync(0xffffffffu, Values::outside(any))) {
#pragma unroll
            for (int j = 0; j < VEC; ++j)
              if (x[j] > from_x) atomicAdd(&s_u.count[Values::at(d[j])], 1u);
          } else {
#pragma unroll 1
            for (int j = 0; j < VEC; ++j)
              if (x[j] > from_x) {
                if (!Values::outside(d[j])) atomicAdd(&s_u.count[Values::at(d[j])], 1u);
                else if (weight.any(x[j])) small(x[j], 1);
              }
          }
        } else if (by_mass) {
          u64 w[VEC];
#pragma unroll
          for (int j = 0; j < VEC; ++j) w[j] = weight(x[j]);
#pragma unroll
          for (int j = 0; j < VEC; ++j)
            if (x[j] > from_x) add_to(s_h, bin_of(top, x[j]), w[j]);
        } else {
#pragma unroll
          for (int j = 0; j < VEC; ++j)
            if (x[j] > from_x) atomicAdd(&s_h.lo[bin_of(top, x[j])], 1u);
        }
      });
    }
    const u64 from_w = from_n != 0 && by_mass ? weight(from_x) : 0;
    const int from_bin = from_n == 0 ? -1 : by_value ? values.bin(from_x) : bin_of(top, from_x);
    if (from_n != 0 && rank == 0 && tid == 0) {                // ties at the border found before: as many as were kept
      if (!by_value) add_to(s_h, from_bin, by_mass ? from_w * from_n : from_n);
      else if (Values::small(from_bin)) small(from_x, from_n);
      else if (const int d = values.distance(__float_as_uint(from_x) >> 16); !Values::outside(d)) atomicAdd(&s_u.count[Values::at(d)], from_n);
    }
    cluster.sync();
    // every CTA adds up its part of the bins, a few a thread
    constexpr int MOST = by_mass && sizeof(T) == 2 ? VALUES / THREADS : PER;
    const int chunk = (by_value ? VALUES : BINS) / size, per = max(1, chunk / THREADS), b0 = rank * chunk + tid * per;
    u64 amount[MOST], sum = 0;
#pragma unroll
    for (int i = 0; i < MOST; ++i) {
      amount[i] = 0;
      if (i < per && tid * per < chunk) {
        if (by_value) {
          const bool small_ones = Values::small(b0 + i);
          for (int j = 0; j < size; ++j) {
            const uint32_t* h = cluster.map_shared_rank(&s_small[b0 + i == HALF][0], j);
            amount[i] += small_ones ? ((u64)h[1] << 32) + h[0] : cluster.map_shared_rank(s_u.count, j)[Values::at_bin(b0 + i)];
          }
          if (amount[i] && !small_ones) amount[i] *= weight(values.value(Values::at_bin(b0 + i)));
        } else {
          for (int j = 0; j < size; ++j) {
            const Histogram* h = cluster.map_shared_rank(&s_h, j);
            amount[i] += ((u64)h->hi[b0 + i] << 32) + h->lo[b0 + i];
          }
        }
      }
      sum += amount[i];
    }
    u64 front, all;
    cta_scan(sum, front, all);
    if (size > 1) {
      if (tid < size) cluster.map_shared_rank(s_chunk, tid)[rank] = all;
      cluster.sync();
      all = 0;
      for (int j = 0; j < size; ++j) {
        if (j < rank) front += s_chunk[j];
        all += s_chunk[j];
      }
    }
    if (few && all < k) {                                      // (not so many threads have scores)
      cluster.sync();
      return Border{0, 0, 0};
    }
    const double goal = by_mass ? share * (double)all : (double)k;
    // the last bin that has any, and in front of which there is less than the goal (the first one in any case)
    if (tid == 0) s_found.bin = -1;
    __syncthreads();
    int best = -1;
    Found mine = {};
    mine.bin = -1;
#pragma unroll
    for (int i = 0; i < MOST; ++i) {
      if (amount[i] > 0 && (front == 0 || (double)front < goal)) {
        best = b0 + i;
        mine = Found{best, front, amount[i]};
      }
      front += amount[i];
    }
    if (best >= 0) atomicMax(&s_found.bin, best);
    __syncthreads();
    if (best >= 0 && s_found.bin == best) s_found = mine;
    if (tid == 0) s_n = 0;
    __syncthreads();
    Found f = s_found;
    if (size > 1) {
      if (tid < size) cluster.map_shared_rank(s_best, tid)[rank] = f;
      cluster.sync();
      for (int j = 0; j < size; ++j)
        if (s_best[j].bin >= f.bin) f = s_best[j];
    }
    if (few) f.in_front = 0;
    if (by_value && !Values::small(f.bin)) {                   // ties, all of them
      if (tid == 0) {
        const float x = values.value(Values::at_bin(f.bin));
        const u64 w = weight(x), n = f.amount / w;
        s_border = Border{Key<T>::of(x), (uint32_t)ties_below(n, w, f.in_front, goal), f.bin == from_bin ? 0xffffffffu : (uint32_t)n};      // (as many as were found before)
      }
      __syncthreads();
      return s_border;
    }
    // the bin's scores, with their ids, to the first CTA: in ascending order of (keys from the largest on, ids)
    int* counter = cluster.map_shared_rank(&s_n, 0);
    u64* list = cluster.map_shared_rank(s_u.list, 0);
    auto bin_in = [&](float x) { return by_value ? values.bin(x) : bin_of(top, x); };
    if (__any_sync(0xffffffffu, my_top > from_x && bin_in(my_top) <= f.bin)) {
      sweep([&](int g, uint4 v) {
        const float most = largest(v, T());
        if (!(most > from_x) || bin_in(most) > f.bin) return;
        float x[VEC];
        unpack(v, x);
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          const int bin = bin_in(x[j]);
          if (x[j] > from_x && (few ? bin <= f.bin : bin == f.bin)) {
            const int at = atomicAdd(counter, 1);
            if (at < LIST) list[at] = (u64)~Key<T>::of(x[j]) << 32 | (uint32_t)(g + j - shift);
          }
        }
      });
    }
    cluster.sync();
    if (*counter > LIST) {
      cluster.sync();                                          // (has been read)
      return few ? Border{0, 0, 0} : search_digits(by_mass, share, k);
    }
    if (rank == 0) {
      const int have = s_n;
      int n2 = 2;
      while (n2 < have) n2 <<= 1;
      if (have <= THREADS) {                                   // a thread an entry: its place is the number of those in front of it
        const u64 x = tid < have ? s_u.list[tid] : 0;
        int place = 0;
#pragma unroll 4
        for (int i = 0; i < have; ++i) place += s_u.list[i] < x;
        __syncthreads();
        if (tid < have) s_u.list[place] = x;
        __syncthreads();
      } else {
        for (int i = have + tid; i < n2; i += THREADS) s_u.list[i] = ~0ull;
        __syncthreads();
        for (int a = 2; a <= n2; a <<= 1)
          for (int b = a >> 1; b; b >>= 1) {
            for (int i = tid; i < n2 / 2; i += THREADS) {
              const int lo = (i & (b - 1)) | (i & ~(b - 1)) << 1, hi = lo | b;
              const u64 x = s_u.list[lo], y = s_u.list[hi];
              if ((x > y) == ((lo & a) == 0)) { s_u.list[lo] = y; s_u.list[hi] = x; }
            }
            __syncthreads();
          }
      }
      auto key_at = [&](int i) { return ~(uint32_t)(s_u.list[i] >> 32); };
      // how many of them, in order, are kept
      int kept = (int)min((u64)have, k - f.in_front);
      u64 inside = 0;                                          // weight of all of them
      const int per_thread = (n2 + THREADS - 1) / THREADS, i0 = tid * per_thread;
      if (few && share < 1.0) {                                // all that top-k keeps is here: what top-p leaves of it
        u64 w = 0, below_goal = 0, run, all, unused;
        for (int i = i0; i < min(i0 + per_thread, kept); ++i) w += weight(score_of<T>(key_at(i)));
        cta_scan(w, run, all);
        for (int i = i0; i < min(i0 + per_thread, kept); ++i) {
          below_goal += i == 0 || (double)run < share * (double)all;
          run += weight(score_of<T>(key_at(i)));
        }
        cta_scan(below_goal, unused, all);
        kept = (int)all;
      } else if (by_mass) {
        u64 w = 0, before, unused;
        for (int i = i0; i < min(i0 + per_thread, have); ++i) w += weight(score_of<T>(key_at(i)));
        cta_scan(w, before, inside);
        u64 below_goal = 0, run = f.in_front + before, total;
        for (int i = i0; i < min(i0 + per_thread, have); ++i) {
          below_goal += (i == 0 && f.in_front == 0) || (double)run < goal;
          run += weight(score_of<T>(key_at(i)));
        }
        cta_scan(below_goal, unused, total);
        kept = (int)total;
      }
      if (tid == 0) {
        Border x;
        const u64 virtual_ties = f.bin == from_bin ? from_n : 0;       // (of the border before: behind all others)
        const bool into = by_mass && virtual_ties > 0 && kept == have && (have == 0 || (double)(f.in_front + inside) < goal);
        if (into || have == 0) {
          x.key = from;
          x.kept = (uint32_t)ties_below(virtual_ties, from_w, f.in_front + inside, goal);
          x.ties = 0xffffffffu;                                // (as many as were found before)
        } else {
          x.key = key_at(kept - 1);
          int lo = kept - 1, hi = kept;
          while (lo > 0 && key_at(lo - 1) == x.key) --lo;
          while (hi < have && key_at(hi) == x.key) ++hi;
          x.kept = kept - lo;
          x.ties = hi - lo;
        }
        s_border = x;
        for (int j = 1; j < size; ++j) *cluster.map_shared_rank(&s_border, j) = x;
      }
    }
    cluster.sync();
    return s_border;
  };
  Border border = {from, 0, 0};                               // (all above -inf)
  const bool few = top_k <= min(size * THREADS / 2, LIST / 4);
  // (Either form is called at one place only, so that its code is there once and in line: a third call took one row of FP32 from 21 us to 38.)
  bool both = false;                                           // top-k's search has found top-p's border
  uint32_t ties_before = 0;
#pragma unroll 1
  for (bool among_few = few; by_k; among_few = false) {
    border = search(Counts(), by_p ? (double)top_p : 1.0, (u64)top_k, among_few);
    if (border.ties == 0 && among_few) continue;               // (not enough threads, or too many scores)
    both = among_few && by_p;
    from = border.key;
    from_n = border.kept;
    from_x = score_of<T>(from);
    ties_before = border.ties;
    break;
  }
  if (by_p && !both) {
    border = search(Mass(), (double)top_p, 0, false);
    if (by_k && border.key == from) border.ties = ties_before;      // (of those at the border before, some more go)
  }

  // ---- what is kept, in the order of ids ----
  const bool some_ties = (by_k || by_p) && border.kept < border.ties;
  const float border_x = score_of<T>(border.key);
  u64 tie_rank = 0;
  if (some_ties) {
    u64 mine = 0;
    sweep([&](int, uint4 v) { mine += __popc(equal(v, border_x, T())); });
    cluster_sum(warp_sum(mine), tie_rank, 0);
  }
  const double least = min_p > 0.f ? fmin((double)min_p, 1.0) : 0.0;
  // min-p: scores above `sure` reach it, those below `never` do not (a hundred thousandth of the distance, and some steps of FP32, to either side of the border)
  float sure = INFINITY, never = -INFINITY;
  if (least > 0.0 && !isinf(top)) {
    const double away = fmax(-log(least) / inv_t, 0.0), slack = away * 1e-5 + (fabs((double)top) + away) * 1e-6;
    sure = (float)((double)top - away + slack);
    never = (float)((double)top - away - slack);
  }
  // Of the ties at the border, the first border.kept: all lanes' bits; `at` ties lie in front of the warp's, and it goes on.
  auto ties_that_stay = [&](uint32_t tie, u64& at) {
    if (!__any_sync(0xffffffffu, tie)) return 0u;
    int before = __popc(tie);
#pragma unroll
    for (int s = 1; s < 32; s <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, before, s);
      if (lane >= s) before += y;
    }
    const int all = __shfl_sync(0xffffffffu, before, 31);
    before -= __popc(tie);
    uint32_t stay = 0;
#pragma unroll
    for (int j = 0; j < VEC; ++j)
      if (tie >> j & 1u && at + before + __popc(tie & ((1u << j) - 1u)) < border.kept) stay |= 1u << j;
    at += all;
    return stay;
  };
  const float low = fmaxf(border_x, never);                    // below it nothing stays
  // BF16 rows with many scores: every number's weight where it stays, and the highest bit.  (Border ties of which some go are looked at one by one.)
  constexpr u64 STAYS = 1ull << 63;
  const bool border_stays = some_ties && (least == 0.0 || weight.reaches(border_x, least));
  const u64 border_w = border_stays ? weight(border_x) : 0;
  if (by_values) {
    for (int i = tid; i < VALUES; i += THREADS) {
      const float x = values.value(i);
      bool stays = x <= top && (x > border_x || (x == border_x && (by_k || by_p) && !some_ties));
      if (stays && least > 0.0 && !(x > sure)) stays = !(x < never) && weight.reaches(x, least);
      s_u.value[i] = stays ? STAYS | weight(x) : 0;
    }
    __syncthreads();
  }
  // Weights of VEC scores, 0 where they go, and which stay; `at`: ties in front of the warp's first.
  auto keep = [&](uint4 v, u64& at, u64 (&w)[VEC]) {
    uint32_t stay = 0;
#pragma unroll
    for (int j = 0; j < VEC; ++j) w[j] = 0;
    const float most = largest(v, T());
    if (!__any_sync(0xffffffffu, most >= low && most > -INFINITY)) return stay;
    if (by_values) {
      int d[VEC], any = 0;
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        d[j] = values.distance(score_bits(v, j));
        any |= d[j];
      }
      if (!__any_sync(0xffffffffu, Values::outside(any))) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          const u64 y = s_u.value[Values::at(d[j])];
          stay |= (uint32_t)(y >> 63) << j;
          w[j] = y & ~STAYS;
        }
        if (border_stays) {
          const uint32_t ties = ties_that_stay(equal(v, border_x, T()), at);
#pragma unroll
          for (int j = 0; j < VEC; ++j)
            if (ties >> j & 1u) w[j] = border_w;
          stay |= ties;
        }
        return stay;
      }
    }
    float x[VEC];
    unpack(v, x);
#pragma unroll
    for (int j = 0; j < VEC; ++j)
      if (x[j] > border_x) stay |= 1u << j;
    if (by_k || by_p) {                                        // (else the border is -inf)
      const uint32_t tie = equal(v, border_x, T());
      stay |= some_ties ? ties_that_stay(tie, at) : tie;
    }
    if (least > 0.0) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        // clear of the border by far, or worked out
        if ((stay >> j & 1u) && !(x[j] > sure) && (x[j] < never || !weight.reaches(x[j], least))) stay &= ~(1u << j);
      }
    }
    if (__any_sync(0xffffffffu, stay != 0)) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const u64 u = weight(x[j]);
        w[j] = stay >> j & 1u ? u : 0;
      }
    }
    return stay;
  };
  const bool aligned_out = out && reinterpret_cast<uintptr_t>(out) / sizeof(T) % VEC == (unsigned)shift;
  u64 mine = 0, before, at = tie_rank;
  if (out || __any_sync(0xffffffffu, my_top >= low))
    sweep([&](int g, uint4 v) {
      u64 w[VEC];
      const uint32_t stay = keep(v, at, w);
#pragma unroll
      for (int j = 0; j < VEC; ++j) mine += w[j];
      if (out && g < g1) {
        uint4 y = make_uint4(nothing, nothing, nothing, nothing);
        if (stay) {
          const T* x = reinterpret_cast<const T*>(&v);
          T z[VEC];
#pragma unroll
          for (int j = 0; j < VEC; ++j) z[j] = stay >> j & 1u ? x[j] : from_f32<T>(-INFINITY);
          y = *reinterpret_cast<const uint4*>(z);
        }
        if (aligned_out && g >= shift && g + VEC <= end) {
          __stcs(reinterpret_cast<uint4*>(out + (g - shift)), y);
        } else {
#pragma unroll
          for (int j = 0; j < VEC; ++j)
            if (g + j >= shift && g + j < end) out[g + j - shift] = reinterpret_cast<const T*>(&y)[j];
        }
      }
    });
  mine = warp_sum(mine);
  const u64 all = cluster_sum(mine, before, 1);
  const double goal = fmax((double)r, 0.0) * (double)all;
  // the warp in which the running sum passes the goal; beyond all of them (r not below one), the last that has any weight
  const bool past = !((double)all > goal);
  const bool hit = mine > 0 && (past ? before + mine == all : !((double)before > goal) && (double)(before + mine) > goal);
  if (hit) {
    u64 run = before;
    at = tie_rank;
    bool done = false;
    // (without KEPT, scores may have been overwritten by what is left of them: those that went are -inf, and the others, ties among them, all stay)
    sweep([&](int g, uint4 v) {
      if (done) return;
      float x[VEC];
      unpack(v, x);
      u64 w[VEC], sum = 0;
      if (!KEPT && out == row) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) w[j] = weight(x[j]);
      } else {
        keep(v, at, w);
      }
#pragma unroll
      for (int j = 0; j < VEC; ++j) sum += w[j];
      u64 upto = sum;
#pragma unroll
      for (int s = 1; s < 32; s <<= 1) {
        const u64 y = __shfl_up_sync(0xffffffffu, upto, s);
        if (lane >= s) upto += y;
      }
      auto passes = [&](u64 x) { return past ? x == all : (double)x > goal; };
      const unsigned who = __ballot_sync(0xffffffffu, sum > 0 && passes(run + upto));
      if (who) {
        done = true;
        if (lane == __ffs(who) - 1) {
          u64 y = run + upto - sum;
          int token = -1;
          float x_of = 0.f;
#pragma unroll
          for (int j = 0; j < VEC; ++j) {
            y += w[j];
            if (token < 0 && w[j] > 0 && passes(y)) { token = g + j - shift; x_of = x[j]; }
          }
          p.tokens[m] = token;
          if (p.logp) p.logp[m] = (float)((x_of == top ? 0.0 : ((double)x_of - (double)top) * inv_t) - log((double)all / unit));
        }
      }
      run += __shfl_sync(0xffffffffu, upto, 31);
    });
  }
}

}  // namespace sample
}  // namespace ad
