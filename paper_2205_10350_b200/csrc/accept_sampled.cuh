// Verification of drafted tokens against the verifier's probabilities, from given random numbers.
#pragma once

#include <cooperative_groups.h>
#include <math.h>

#include <type_traits>

#include "kv_cache.cuh"      // load8

namespace ad {
namespace sampled {

constexpr int STAT_THREADS = 256;
constexpr int ACCEPT_THREADS = 512;

struct Stat { float top, sum; };     // of a part of a row: its largest score, and the sum of exp2(score * c - reference(top))

struct Params {
  const void* score[2];              // verifier's and drafter's [M, vocab]; drafter's null: each draft had probability one
  size_t stride[2];
  int vocab, parts, M, B, kmax, eos;
  float c;                           // log2(e) / temperature
  double inv_t;                      // 1 / temperature
  const int* off;                    // [B + 1]
  const int* drafts;                 // [B, kmax]
  const float* u;                    // [B, kmax]
  const float* r;                    // [B]
  Stat* stats;                       // [2][M][parts]
  int* tokens;                       // [B, kmax]
  int* n_acc;                        // [B]
  int* status;
};

// What exponents are taken against: finite whatever the maximum is.
__device__ __forceinline__ float reference(float top, float c) { return isinf(top) ? 0.f : top * c; }

__device__ __forceinline__ void join(Stat& a, const Stat& b, float c) {
  const float top = fmaxf(a.top, b.top), ref = reference(top, c);
  a.sum = a.sum * exp2f(reference(a.top, c) - ref) + b.sum * exp2f(reference(b.top, c) - ref);
  a.top = top;
}

// Largest score and sum of exponentials of part blockIdx.y of row blockIdx.x, of the verifier's scores or (blockIdx.z) the drafter's.  Scores are
// read once, 16 bytes at a time behind a ragged beginning; bound by bytes.  grid = (M, parts, 1 or 2), block = STAT_THREADS.
template <typename T>
__global__ void __launch_bounds__(STAT_THREADS)
score_stats_kernel(Params p) {
  constexpr int W = 16 / sizeof(T);                       // scores in a vector
  __shared__ Stat s_part[STAT_THREADS / 32];
  pdl_launch();
  pdl_wait();
  const T* row = static_cast<const T*>(p.score[blockIdx.z]) + blockIdx.x * p.stride[blockIdx.z];
  const int head = min((int)((16 - reinterpret_cast<uintptr_t>(row) % 16) % 16 / sizeof(T)), p.vocab);
  const int vecs = (p.vocab - head) / W, tail = head + vecs * W;
  const int each = (vecs + p.parts - 1) / p.parts, v0 = min((int)blockIdx.y * each, vecs), v1 = min(v0 + each, vecs);
  Stat s = {-INFINITY, 0.f};
  auto add = [&](float* x, auto count) {
    constexpr int N = decltype(count)::value;
    float top = s.top;
#pragma unroll
    for (int j = 0; j < N; ++j) top = fmaxf(top, x[j]);
    const float ref = reference(top, p.c);
    s.sum *= exp2f(reference(s.top, p.c) - ref);
    s.top = top;
#pragma unroll
    for (int j = 0; j < N; ++j) x[j] = exp2f(fmaf(x[j], p.c, -ref));
#pragma unroll
    for (int w = N / 2; w; w >>= 1)                       // (pairs first: a thread's sum is a chain of as many additions as it has vectors)
#pragma unroll
      for (int j = 0; j < w; ++j) x[j] += x[j + w];
    s.sum += x[0];
  };
  typedef std::integral_constant<int, 1> One;
  for (int v = v0 + threadIdx.x; v < v1; v += STAT_THREADS) {
    float x[8];
    if constexpr (sizeof(T) == 2) {
      kv::load8(row + head + (size_t)v * W, x);
    } else {
      const float4 f = *reinterpret_cast<const float4*>(row + head + (size_t)v * W);
      x[0] = f.x; x[1] = f.y; x[2] = f.z; x[3] = f.w;
    }
    add(x, std::integral_constant<int, W>());
  }
  if (blockIdx.y == 0) {
    const int i = threadIdx.x;
    if (i < head) { float x = to_f32(row[i]); add(&x, One()); }
    if (tail + i < p.vocab) { float x = to_f32(row[tail + i]); add(&x, One()); }      // (fewer than W left)
  }
#pragma unroll
  for (int w = 16; w; w >>= 1) {
    Stat t = {__shfl_xor_sync(0xffffffffu, s.top, w), __shfl_xor_sync(0xffffffffu, s.sum, w)};
    join(s, t, p.c);
  }
  if ((threadIdx.x & 31) == 0) s_part[threadIdx.x >> 5] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < STAT_THREADS / 32; ++w) join(s, s_part[w], p.c);
    p.stats[((size_t)blockIdx.z * p.M + blockIdx.x) * p.parts + blockIdx.y] = s;
  }
}

enum Decision { KEEP = 0, STOP = 1, NEAR = 2, DROP = 3 };     // STOP: kept, and the end of the output.  NEAR: too close to call in 32 bits

namespace cg = cooperative_groups;

// Exchange between the CTAs of a cluster, one slot per CTA.
constexpr int MAX_CLUSTER = 8;
struct Exchange {
  double sum[2][MAX_CLUSTER];       // (two, taken in turn)
  int pick[2][MAX_CLUSTER];         // [lowest hit, highest token with weight]
};

// The decision for one row, by one cluster.
//   Position i keeps its draft d while u_i q_i(d) < p_i(d).  The first one that does not gets the token at which the running sum of
//   max(p_i - q_i, 0), in the order of ids, passes r times its total, and is the last (n = i + 1); without a draft the sum is p_i's own.
// A token that is drawn depends on sums over the vocabulary to the last bit near a border, and a decision on a comparison; both have to come out as
// the formula says and alike for every way of adding up.  So decisions are taken from the 32-bit sums of score_stats_kernel only where these leave no
// doubt, and else, like the draw, from sums in 64 bits over the one position's scores, which are still in L2.
// grid = B clusters of CTAs that share the vocabulary, block = ACCEPT_THREADS.  Every CTA of a cluster takes the same decisions from the same numbers.
template <typename T>
__global__ void __launch_bounds__(ACCEPT_THREADS)
accept_sampled_kernel(Params p) {
  __shared__ int s_first[2];
  __shared__ double s_warp[ACCEPT_THREADS / 32];
  __shared__ int s_pick[2];
  __shared__ Exchange s_ex;
  cg::cluster_group cluster = cg::this_cluster();
  const int rank = cluster.block_rank(), size = cluster.num_blocks(), b = blockIdx.x / size, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  pdl_launch();
  pdl_wait();
  const int o = __ldcg(p.off + b);
  const long long n_tokens = (long long)__ldcg(p.off + b + 1) - o;
  const int k = n_tokens < 0 || n_tokens > p.kmax ? -1 : (int)n_tokens;
  const int* drafts = p.drafts + (size_t)b * p.kmax;
  const bool bad = o < 0 || k < 0 || o > p.M - k;
  if (bad || k == 0) {                                      // (all of the cluster's CTAs alike)
    if (rank == 0) {
      if (bad && tid == 0) latch_error(p.status, AD_ERR_ARG);
      if (tid == 0) p.n_acc[b] = 0;
      for (int i = tid; i < p.kmax; i += ACCEPT_THREADS) p.tokens[(size_t)b * p.kmax + i] = -1;
    }
    return;
  }
  cluster.sync();                                           // (another CTA's shared memory may be written once that CTA runs)
  const T* prow = static_cast<const T*>(p.score[0]) + (size_t)o * p.stride[0];
  const T* qrow = static_cast<const T*>(p.score[1]) + (size_t)o * p.stride[1];
  auto draft_at = [&](int i) {
    const int d = __ldg(drafts + i);
    return d < p.vocab ? d : -1;
  };

  // ---- the scores' weights in 64 bits: exp((score - top) / temperature), 1 at the top (even where it is infinite), 0 for a NaN ----
  auto weight = [&](float x, float top) {
    if (x == top) return 1.0;
    const double e = exp(((double)x - (double)top) * p.inv_t);
    return e >= 0.0 && !isinf(top) ? e : 0.0;
  };
  auto row_stat = [&](int z, int i) {
    Stat s = {-INFINITY, 0.f};
    const Stat* part = p.stats + ((size_t)z * p.M + o + i) * p.parts;
    for (int j = 0; j < p.parts; ++j) {
      Stat t;
      t.top = __ldcg(&part[j].top); t.sum = __ldcg(&part[j].sum);
      join(s, t, p.c);
    }
    return s;
  };

  // ---- a position's decision from the 32-bit sums ----
  auto decide = [&](int i) -> int {
    const int d = draft_at(i);
    if (d < 0) return DROP;
    const Stat sp = row_stat(0, i), sq = p.score[1] ? row_stat(1, i) : Stat{0.f, 1.f};
    if (!isfinite(sp.top) || !isfinite(sp.sum) || !isfinite(sq.top) || !isfinite(sq.sum)) return NEAR;
    const float xp = to_f32(prow[(size_t)i * p.stride[0] + d]), xq = p.score[1] ? to_f32(qrow[(size_t)i * p.stride[1] + d]) : 0.f;
    if (xp != xp || xq != xq) return NEAR;
    const double qd = p.score[1] ? exp2((double)xq * p.c - reference(sq.top, p.c)) : 1.0;
    const double want = (double)__ldg(p.u + (size_t)b * p.kmax + i) * qd * (double)sp.sum;
    const double have = exp2((double)xp * p.c - reference(sp.top, p.c)) * (double)sq.sum;
    // How far off the two may be, relatively.  A sum: chains of at most 128 additions in all, 2^-24 each, an exponential within 2^-21 of what its
    // rounded exponent asks for; 1.6e-5 for both sums.  The exponents' factor c is off by 2^-24 of itself, which moves a probability by that share
    // of its distance from the top and of the mean distance (below 64 where it counts: what lies further off has no weight).
    const double away = (isinf(xp) ? 0.0 : (double)(sp.top - xp)) + (p.score[1] && !isinf(xq) ? (double)(sq.top - xq) : 0.0);
    const double doubt = 3e-5 + 1.2e-7 * away * p.c;
    if (fabs(want - have) <= doubt * fmax(fabs(want), have)) return NEAR;
    return want < have ? (d == p.eos ? STOP : KEEP) : DROP;
  };

  int first = -1, how = KEEP, from = 0;      // the first position that does not simply keep its draft
  double zp = 0.0, zq = 0.0;
  Stat sp = {0.f, 1.f}, sq = {0.f, 1.f};
  int turn = 0;
  // sum of a value over the cluster, in the order of its threads: in front of this thread's, and all of it
  auto cluster_sum = [&](double x, double& before, double& all) {
    double run = x;
#pragma unroll
    for (int w = 1; w < 32; w <<= 1) {
      const double y = __shfl_up_sync(0xffffffffu, run, w);
      if (lane >= w) run += y;
    }
    __syncthreads();
    if (lane == 31) s_warp[warp] = run;
    __syncthreads();
    double mine = 0.0, front = 0.0;
    for (int w = 0; w < ACCEPT_THREADS / 32; ++w) {
      if (w == warp) front = mine;
      mine += s_warp[w];
    }
    const int slot = turn & 1;
    if (tid < size) cluster.map_shared_rank(&s_ex, tid)->sum[slot][rank] = mine;
    cluster.sync();
    double ahead = 0.0;
    all = 0.0;
    for (int j = 0; j < size; ++j) {
      if (j == rank) ahead = all;
      all += s_ex.sum[slot][j];
    }
    before = ahead + front + (run - x);
    ++turn;
  };
  const int each = (p.vocab + size * ACCEPT_THREADS - 1) / (size * ACCEPT_THREADS);
  const int v0 = min((rank * ACCEPT_THREADS + tid) * each, p.vocab), v1 = min(v0 + each, p.vocab);
  for (;;) {
    if (tid == 0) s_first[0] = k;
    __syncthreads();
    for (int i = from + tid; i < k; i += ACCEPT_THREADS)
      if (decide(i) != KEEP) { atomicMin(&s_first[0], i); break; }              // (an integer minimum: no order in it)
    __syncthreads();
    first = s_first[0];
    if (first == k) { how = KEEP; break; }
    if (tid == 0) s_first[1] = decide(first);
    __syncthreads();
    how = s_first[1];
    if (how == STOP) break;
    // the position's sums in 64 bits
    sp = row_stat(0, first);
    sq = p.score[1] ? row_stat(1, first) : Stat{0.f, 1.f};
    const T* pr = prow + (size_t)first * p.stride[0];
    const T* qr = qrow + (size_t)first * p.stride[1];
    double a = 0.0, c = 0.0, unused;
    for (int v = v0; v < v1; ++v) {
      a += weight(to_f32(pr[v]), sp.top);
      if (p.score[1]) c += weight(to_f32(qr[v]), sq.top);
    }
    cluster_sum(a, unused, zp);
    if (p.score[1] && sq.top > -INFINITY) cluster_sum(c, unused, zq); else zq = 1.0;
    if (how == DROP) break;
    const int d = draft_at(first);
    const double pd = sp.top > -INFINITY ? weight(to_f32(pr[d]), sp.top) : 0.0;
    const double qd = !p.score[1] ? 1.0 : sq.top > -INFINITY ? weight(to_f32(qr[d]), sq.top) : 0.0;
    if ((double)__ldg(p.u + (size_t)b * p.kmax + first) * qd * zp < pd * zq) {
      if (d == p.eos) { how = STOP; break; }
      from = first + 1;
      if (from == k) { first = k; how = KEEP; break; }
    } else {
      how = DROP;
      break;
    }
  }

  // ---- the token of the first position that does not keep its draft ----
  int token = 0;
  if (how == DROP) {
    const T* pr = prow + (size_t)first * p.stride[0];
    const T* qr = qrow + (size_t)first * p.stride[1];
    const int d = draft_at(first);
    const double r = (double)__ldg(p.r + b);
    for (int form = d < 0 ? 1 : 0; form < 2; ++form) {      // 0: what the verifier gives beyond the drafter; 1: the verifier's own
      auto left = [&](int v) {
        if (sp.top == -INFINITY) return 0.0;
        const double pv = weight(to_f32(pr[v]), sp.top) / zp;
        if (form == 1) return pv;
        if (!p.score[1]) return v == d ? 0.0 : pv;
        return sq.top == -INFINITY ? pv : fmax(pv - weight(to_f32(qr[v]), sq.top) / zq, 0.0);
      };
      double mine = 0.0, before, all;
      int last = -1;
      for (int v = v0; v < v1; ++v) {
        const double x = left(v);
        mine += x;
        if (x > 0.0) last = v;
      }
      cluster_sum(mine, before, all);
      if (form == 0 && !(all > 0.0)) continue;              // (nothing beyond the drafter's: the verifier's own)
      int hit = INT_MAX;
      const double goal = r * all;
      if (before + mine > goal) {
        double run = before;
        for (int v = v0; v < v1; ++v) {
          const double x = left(v);
          run += x;
          if (x > 0.0 && run > goal) { hit = v; break; }
        }
      }
      if (tid == 0) { s_pick[0] = INT_MAX; s_pick[1] = -1; }
      __syncthreads();
      atomicMin(&s_pick[0], hit);
      atomicMax(&s_pick[1], last);
      __syncthreads();
      if (tid < 2) cluster.map_shared_rank(&s_ex, 0)->pick[tid][rank] = s_pick[tid];
      cluster.sync();
      if (rank == 0) {
        int lo = INT_MAX, hi = -1;
        for (int j = 0; j < size; ++j) { lo = min(lo, s_ex.pick[0][j]); hi = max(hi, s_ex.pick[1][j]); }
        token = lo < INT_MAX ? lo : max(hi, 0);             // (r not below one: the last token with any weight; no weight anywhere: id 0)
      }
      break;
    }
  }
  if (rank == 0) {
    const int n = first == k ? k : first + 1;
    if (tid == 0) p.n_acc[b] = n;
    for (int i = tid; i < p.kmax; i += ACCEPT_THREADS)
      p.tokens[(size_t)b * p.kmax + i] = i >= n ? -1 : i == first && how == DROP ? token : __ldg(drafts + i);
    for (int i = tid; i < k; i += ACCEPT_THREADS)
      if (__ldg(drafts + i) >= p.vocab) latch_error(p.status, AD_ERR_ARG);
  }
}

}  // namespace sampled
}  // namespace ad
