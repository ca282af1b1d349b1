// Sampling of tokens with temperature, top-k, top-p and min-p from given random numbers.
#pragma once

#include <cooperative_groups.h>
#include <math.h>

#include "accept_sampled.cuh"      // exp_below
#include "kv_cache.cuh"

namespace ad {
namespace sample {

namespace cg = cooperative_groups;

constexpr int THREADS = 512, WARPS = THREADS / 32, MAX_CLUSTER = 8;
constexpr int DIGIT = 11, BINS = 1 << DIGIT, PER = BINS / THREADS;      // bins of a level, and of a thread
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

// What a level of the search has counted: scores, and their weights in two halves.
struct Histogram { uint32_t n[BINS], lo[BINS], hi[BINS]; };
struct Found { uint32_t bin, n; u64 in_front_n, in_front, mass; };

// 64-bit sums from 32-bit atomic additions: exact, so that their order does not matter.
__device__ __forceinline__ void add_mass(Histogram& h, uint32_t bin, u64 w) {
  const uint32_t l = (uint32_t)w, old = atomicAdd(&h.lo[bin], l), carry = old + l < old;
  const uint32_t up = (uint32_t)(w >> 32) + carry;
  if (up) atomicAdd(&h.hi[bin], up);
}

// One row by a cluster of CTAs that share the vocabulary, every warp a run of ids.
//   w(v) = exp((score(v) - largest) / T); tokens are ordered by score, ties by id.  Top-k keeps the first k; top-p, of these, the ones in front of
//   which less than top_p of their weight lies (and the first); min-p, of those, the ones with w >= min_p.  All three keep a beginning of the order, so that what
//   is kept is told by one score and the number of ids that are kept of those that have just this score.  The token is the lowest kept id at which
//   the running sum of weights, over kept ids in order, exceeds r times their total.
// The k-th largest score, and the one at which the weight in front reaches top_p of the whole, are found digit by digit of its key: a histogram of the digit
// among the scores that share the digits so far, summed over the cluster, and the bin in which the border lies.  Weights are worked out in FP64 and
// summed as integers in units of 2^-scale_bits (vocab * 2^scale_bits <= 2^62): the largest is 1, so a sum is off by vocab * 2^-(scale_bits + 1) of itself at
// most, 2^-43 with 1000 ids and 2^-23 with 2^20 (roundings of either sign: their root, a 2^-10th of that, in fact), and comes out the same in any order.
// grid = M clusters, block = THREADS.  Dynamic shared memory: KEPT, the CTA's scores.
template <typename T, bool KEPT>
__global__ void __launch_bounds__(THREADS)
sample_kernel(Params p) {
  extern __shared__ __align__(16) unsigned char s_raw[];
  __shared__ Histogram s_h;
  __shared__ double s_table[sampled::EXP_TABLE];
  __shared__ float s_top[MAX_CLUSTER];
  __shared__ u64 s_warp[WARPS], s_cta[2];
  __shared__ uint32_t s_scan_n[WARPS];
  __shared__ u64 s_scan[WARPS];
  __shared__ Found s_found;
  T* s_x = reinterpret_cast<T*>(s_raw);
  cg::cluster_group cluster = cg::this_cluster();
  const int rank = cluster.block_rank(), size = cluster.num_blocks(), m = blockIdx.x / size, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  pdl_launch();
  if (tid < sampled::EXP_TABLE) s_table[tid] = exp2(tid / (double)sampled::EXP_TABLE);
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

  // ---- scores: warp's ids v0 .. v1 - 1, of the CTA's c0 .. ----
  const int each = ((p.vocab + size * WARPS - 1) / (size * WARPS) + 31) / 32 * 32;
  const int c0 = min(rank * WARPS * each, p.vocab), v0 = min(c0 + warp * each, p.vocab), v1 = min(v0 + each, p.vocab);
  auto score = [&](int v) { return KEPT ? s_x[v - c0] : clean(row[v]); };
  float top = -INFINITY;
  for (int v = v0 + lane; v < v1; v += 32) {
    const T x = clean(row[v]);
    if (KEPT) s_x[v - c0] = x;
    top = fmaxf(top, to_f32(x));
  }
#pragma unroll
  for (int w = 16; w; w >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
  if (lane == 0) s_warp[warp] = __float_as_uint(top);
  __syncthreads();
  for (int w = 0; w < WARPS; ++w) top = fmaxf(top, __uint_as_float((uint32_t)s_warp[w]));
  cluster.sync();                                            // (all CTAs run: their shared memory may be written)
  if (tid < size) cluster.map_shared_rank(s_top, tid)[rank] = top;
  cluster.sync();
  for (int j = 0; j < size; ++j) top = fmaxf(top, s_top[j]);

  if (bad || top == -INFINITY) {                              // (all CTAs alike)
    if (out)
      for (int v = v0 + lane; v < v1; v += 32) out[v] = from_f32<T>(-INFINITY);
    if (rank == 0 && tid == 0) {
      if (bad) latch_error(p.status, AD_ERR_ARG);
      p.tokens[m] = bad ? -1 : 0;
      if (p.logp) p.logp[m] = -INFINITY;
    }
    return;
  }
  auto exact = [&](float x) {                                 // weight; 1 at the top even where that is infinite
    return x == top ? 1.0 : isinf(top) || x == -INFINITY ? 0.0 : sampled::exp_below(((double)x - (double)top) * inv_t, s_table);
  };
  const double unit = ldexp(1.0, p.scale_bits);
  auto weight = [&](float x) { return __double2ull_rn(exact(x) * unit); };

  // ---- sums over the cluster in the order of its warps: of x (alike in all lanes of a warp), in front of this warp, and all ----
  auto cluster_sum = [&](u64 x, u64& before) {
    __syncthreads();
    if (lane == 0) s_warp[warp] = x;
    __syncthreads();
    u64 mine = 0, all = 0;
    before = 0;
    for (int w = 0; w < WARPS; ++w) {
      if (w < warp) before += s_warp[w];
      mine += s_warp[w];
    }
    if (tid == 0) s_cta[0] = mine;
    cluster.sync();
    for (int j = 0; j < size; ++j) {
      const u64 y = *cluster.map_shared_rank(&s_cta[0], j);
      if (j < rank) before += y;
      all += y;
    }
    cluster.sync();
    return all;
  };
  auto warp_sum = [&](u64 x) {
#pragma unroll
    for (int w = 16; w; w >>= 1) x += __shfl_xor_sync(0xffffffffu, x, w);
    return x;
  };

  // ---- the border: of those with keys from `from` on (of those at `from` itself only the first `from_n`), the key at which `passes` ends ----
  // BY_MASS: goal is what the weight in front has to be below; else the number in front.
  uint32_t border = 0, border_n = 0xffffffffu;                // kept: keys above border, and the first border_n that have it
  uint32_t from = 0, from_n = 0xffffffffu;
  auto search = [&](bool by_mass, double share, u64 k) {
    uint32_t prefix = 0;
    int above = Key<T>::BITS;                                  // bits below which the digit lies
    u64 in_front_n = 0, in_front = 0;
    double goal = 0.0;
    Found f;
    while (above > 0) {
      const int bits = min(DIGIT, above), shift = above - bits;
      for (int i = tid; i < BINS; i += THREADS) s_h.n[i] = s_h.lo[i] = s_h.hi[i] = 0;
      __syncthreads();
      const bool first_level = above == Key<T>::BITS;
      for (int v = v0 + lane; v < v1; v += 32) {
        const float x = to_f32(score(v));
        const uint32_t key = Key<T>::of(x);
        if ((first_level || key >> above == prefix) && (key > from || from == 0)) {
          const uint32_t bin = key >> shift & ((1u << bits) - 1u);
          atomicAdd(&s_h.n[bin], 1u);
          if (by_mass) add_mass(s_h, bin, weight(x));
        }
      }
      if (from != 0 && rank == 0 && tid == 0 && (first_level || from >> above == prefix)) {     // ties at the border found before: as many as were kept
        const uint32_t bin = from >> shift & ((1u << bits) - 1u);
        // (a key's score)
        const uint32_t wide = Key<T>::BITS == 16 ? from << 16 | (from & 0x8000u ? 0u : 0xffffu) : from;
        const float x = __uint_as_float(wide & 0x80000000u ? wide & 0x7fffffffu : ~wide);
        atomicAdd(&s_h.n[bin], from_n);
        if (by_mass) {
          const u64 w = weight(x) * from_n;
          add_mass(s_h, bin, w);
        }
      }
      cluster.sync();
      // a thread's bins, from the last one on
      uint32_t n[PER];
      u64 mass[PER], sum_n = 0, sum = 0;
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const int bin = BINS - 1 - (tid * PER + i);
        n[i] = 0;
        mass[i] = 0;
        for (int j = 0; j < size; ++j) {
          const Histogram* h = cluster.map_shared_rank(&s_h, j);
          n[i] += h->n[bin];
          if (by_mass) mass[i] += ((u64)h->hi[bin] << 32) + h->lo[bin];
        }
        sum_n += n[i];
        sum += mass[i];
      }
      // in front of them
      u64 run_n = sum_n, run = sum;
#pragma unroll
      for (int w = 1; w < 32; w <<= 1) {
        const u64 a = __shfl_up_sync(0xffffffffu, run_n, w), b = __shfl_up_sync(0xffffffffu, run, w);
        if (lane >= w) { run_n += a; run += b; }
      }
      if (lane == 31) { s_scan_n[warp] = (uint32_t)run_n; s_scan[warp] = run; }
      __syncthreads();
      u64 front_n = in_front_n + run_n - sum_n, front = in_front + run - sum, total = in_front;
      for (int w = 0; w < WARPS; ++w) {
        if (w < warp) { front_n += s_scan_n[w]; front += s_scan[w]; }
        total += s_scan[w];
      }
      if (first_level) goal = share * (double)total;
      // the last bin that has any, and in front of which there is less than the goal (the first one in any case)
      if (tid == 0) s_found.bin = BINS;
      __syncthreads();
      uint32_t best = BINS;
      Found mine = {};
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const uint32_t bin = BINS - 1 - (tid * PER + i);
        if (n[i] > 0 && (by_mass ? front_n == 0 || (double)front < goal : front_n < k)) {
          best = bin;
          mine = Found{bin, n[i], front_n, front, mass[i]};
        }
        front_n += n[i];
        front += mass[i];
      }
      if (best < BINS) atomicMin(&s_found.bin, best);
      __syncthreads();
      if (best < BINS && s_found.bin == best) s_found = mine;
      __syncthreads();
      f = s_found;
      in_front_n = f.in_front_n;
      in_front = f.in_front;
      prefix = prefix << bits | f.bin;
      above = shift;
      cluster.sync();                                          // (histograms have been read)
    }
    border = prefix;
    if (by_mass) {
      // of n ties of weight w, those with in_front + j w below the goal (the very first in any case)
      const u64 w = f.mass / f.n;
      u64 t = f.n;
      if (w > 0) {
        const double want = (goal - (double)in_front) / (double)w;
        t = want < 1.0 ? 1 : want >= (double)f.n ? f.n : (u64)want;
        while (t > 1 && !((double)(in_front + (t - 1) * w) < goal)) --t;
        while (t < f.n && (double)(in_front + t * w) < goal) ++t;
      }
      border_n = (uint32_t)t;
    } else {
      border_n = (uint32_t)min((u64)f.n, k - in_front_n);
    }
    return f.n;
  };
  uint32_t ties = 0;                                           // that have the border's key
  const bool by_k = top_k > 0 && top_k < p.vocab, by_p = top_p < 1.f;
  if (by_k) {
    ties = search(false, 0.0, (u64)top_k);
    from = border;
    from_n = border_n;
  }
  if (by_p) {
    const uint32_t all = search(true, (double)top_p, 0);
    if (border != from) ties = all;                            // (else: of those at the border before, some more go)
  }

  // ---- what is kept, in the order of ids ----
  const bool some_ties = (by_k || by_p) && border_n < ties;
  u64 tie_rank = 0;
  if (some_ties) {
    u64 mine = 0;
    for (int v = v0 + lane; v < v1; v += 32) mine += Key<T>::of(to_f32(score(v))) == border;
    cluster_sum(warp_sum(mine), tie_rank);
  }
  const double least = min_p > 0.f ? (double)min_p : 0.0;
  // f(v, score, whether it is kept, its weight) for the warp's ids, 32 at a time by all lanes
  auto over = [&](auto f) {
    u64 at = tie_rank;
    for (int i0 = v0; i0 < v1; i0 += 32) {
      const int v = i0 + lane;
      const T x = v < v1 ? score(v) : from_f32<T>(-INFINITY);
      const float xf = to_f32(x);
      const uint32_t key = Key<T>::of(xf);
      bool keep = v < v1 && key >= border;
      if (some_ties) {
        const unsigned tie = __ballot_sync(0xffffffffu, v < v1 && key == border);
        if (key == border) keep = keep && at + __popc(tie & ((1u << lane) - 1u)) < border_n;
        at += __popc(tie);
      }
      const double w = keep ? exact(xf) : 0.0;
      keep = keep && w >= least;
      f(v, x, keep, keep ? __double2ull_rn(w * unit) : 0ull);
    }
  };
  u64 mine = 0, before;
  over([&](int v, T x, bool keep, u64 w) {
    mine += w;
    if (out && v < v1) out[v] = keep ? x : from_f32<T>(-INFINITY);
  });
  mine = warp_sum(mine);
  const u64 all = cluster_sum(mine, before);
  const double goal = fmax((double)r, 0.0) * (double)all;
  // the warp in which the running sum passes the goal; beyond all of them (r not below one), the last that has any weight
  const bool past = !((double)all > goal);
  const bool hit = mine > 0 && (past ? before + mine == all : !((double)before > goal) && (double)(before + mine) > goal);
  if (hit) {
    u64 run = before;
    int token = -1;
    float x_of = 0.f;
    // (scores may have been overwritten by what is left of them: the token's is among those)
    u64 at = tie_rank;
    (void)at;
    for (int i0 = v0; i0 < v1 && token < 0; i0 += 32) {
      const int v = i0 + lane;
      const float xf = v < v1 ? to_f32(out && !KEPT ? clean(out[v]) : score(v)) : -INFINITY;
      const uint32_t key = Key<T>::of(xf);
      bool keep = v < v1 && key >= border;
      if (some_ties && !(out && !KEPT)) {
        const unsigned tie = __ballot_sync(0xffffffffu, v < v1 && key == border);
        if (key == border) keep = keep && at + __popc(tie & ((1u << lane) - 1u)) < border_n;
        at += __popc(tie);
      }
      const double w = keep ? exact(xf) : 0.0;
      const u64 x = keep && w >= least ? __double2ull_rn(w * unit) : 0ull;
      u64 sum = x;
#pragma unroll
      for (int s = 1; s < 32; s <<= 1) {
        const u64 y = __shfl_up_sync(0xffffffffu, sum, s);
        if (lane >= s) sum += y;
      }
      const bool is = x > 0 && (past ? run + sum == all : (double)(run + sum) > goal);
      const unsigned who = __ballot_sync(0xffffffffu, is);
      if (who) {
        const int l = __ffs(who) - 1;
        token = i0 + l;
        x_of = __shfl_sync(0xffffffffu, xf, l);
      }
      run += __shfl_sync(0xffffffffu, sum, 31);
    }
    if (lane == 0) {
      p.tokens[m] = token;
      if (p.logp) p.logp[m] = (float)((x_of == top ? 0.0 : ((double)x_of - (double)top) * inv_t) - log((double)all / unit));
    }
  }
}

}  // namespace sample
}  // namespace ad
