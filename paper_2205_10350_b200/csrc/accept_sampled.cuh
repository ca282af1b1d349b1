// Verification of drafted tokens against the verifier's probabilities, from given random numbers.
#pragma once

#include <cooperative_groups.h>
#include <math.h>

#include "kv_cache.cuh"      // ex2

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

// What exponents are taken against: a whole number, finite whatever the maximum is; at or above the maximum's own while that is below 2^22, within a step of FP32 beyond.
// (Roundings by additions: conversions would go through the pipe of the exponentials, which is the one that is full.)
constexpr float WHOLE = 12582912.f;                                  // 1.5 * 2^23
__device__ __forceinline__ float reference(float top, float c) { return isinf(top) ? 0.f : __fadd_ru(__fmul_rn(top, c), WHOLE) - WHOLE; }
// What brings a sum from one reference to that of a larger maximum.  Both are whole, so this is a power of two, put together from its exponent: however often
// the maximum moves, sums are not rounded for it.  At most one: from an empty sum, which has no reference (0), nothing is scaled up.
__device__ __forceinline__ float rescale(float from, float to) {
  const float k = fmaxf(fminf(from - to, 0.f), -127.f);
  return __int_as_float(__float_as_int(k + (WHOLE + 127.f)) << 23);     // (the sum's last nine bits are k + 127: the exponent, or 0)
}

__device__ __forceinline__ void join(Stat& a, const Stat& b, float c) {
  const float top = fmaxf(a.top, b.top), ref = reference(top, c);
  a.sum = a.sum * rescale(reference(a.top, c), ref) + b.sum * rescale(reference(b.top, c), ref);
  a.top = top;
}

// Largest score and sum of exponentials of part blockIdx.y of row blockIdx.x, of the verifier's scores or (blockIdx.z) the drafter's.  Scores are
// read once, 16 bytes at a time behind a ragged beginning; bound by bytes: 1970 rows of 200000 FP32 scores, verifier's and drafter's, 449 us, 7.0 TB/s;
// of BF16 264 us, 6.0 TB/s; 1656 rows of 32000 in BF16, 44 us, 4.9 TB/s, with the exponentials' pipe at 66 %.  grid = (M, parts, 1 or 2), block = STAT_THREADS.
template <typename T>
__global__ void __launch_bounds__(STAT_THREADS)
score_stats_kernel(Params p) {
  constexpr int W = 16 / sizeof(T), VECS = 2, N = VECS * W;      // scores in a vector; vectors of a round, the next of which is under way
  constexpr uint32_t NOTHING = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;      // -inf
  __shared__ float s_top[STAT_THREADS / 32], s_sum[STAT_THREADS / 32];
  pdl_launch();
  pdl_wait();
  const T* row = static_cast<const T*>(p.score[blockIdx.z]) + blockIdx.x * p.stride[blockIdx.z];
  const int head = min((int)((16 - reinterpret_cast<uintptr_t>(row) % 16) % 16 / sizeof(T)), p.vocab);
  const int vecs = (p.vocab - head) / W, tail = head + vecs * W;
  const int each = (vecs + p.parts - 1) / p.parts, v0 = min((int)blockIdx.y * each, vecs), v1 = min(v0 + each, vecs);
  const uint4* body = reinterpret_cast<const uint4*>(row + head);
  float top = -INFINITY, sum = 0.f, ref = 0.f;
  auto rebase = [&](float t) {                            // to the reference of maximum t
    const float to = reference(t, p.c);
    sum *= rescale(ref, to);
    ref = to;
    top = t;
  };
  auto load = [&](uint4* raw, int v) {
#pragma unroll
    for (int u = 0; u < VECS; ++u)
      raw[u] = v + u * STAT_THREADS < v1 ? __ldcs(body + v + u * STAT_THREADS) : make_uint4(NOTHING, NOTHING, NOTHING, NOTHING);
  };
  uint4 next[VECS];
  load(next, v0 + threadIdx.x);
  for (int v = v0 + threadIdx.x; v < v1; v += VECS * STAT_THREADS) {
    float x[N];
#pragma unroll
    for (int u = 0; u < VECS; ++u) {
      const uint32_t w[4] = {next[u].x, next[u].y, next[u].z, next[u].w};
#pragma unroll
      for (int j = 0; j < W; ++j) x[u * W + j] = __uint_as_float(sizeof(T) == 4 ? w[j % 4] : j % 2 ? w[j / 2] & 0xffff0000u : w[j / 2] << 16);
    }
    load(next, v + VECS * STAT_THREADS);
    float t = top;
#pragma unroll
    for (int j = 0; j < N; j += 2) t = kv::max3(t, x[j], x[j + 1]);
    rebase(t);
    float2 y[N / 2];
#pragma unroll
    for (int j = 0; j < N / 2; ++j) {
      y[j] = kv::fma2(make_float2(x[2 * j], x[2 * j + 1]), make_float2(p.c, p.c), make_float2(-ref, -ref));
      y[j] = make_float2(kv::ex2(y[j].x), kv::ex2(y[j].y));
    }
#pragma unroll
    for (int w = N / 4; w; w >>= 1)                       // (pairs first: a thread's sum is a chain of as many additions as it has rounds)
#pragma unroll
      for (int j = 0; j < w; ++j) y[j] = kv::add2(y[j], y[j + w]);
    sum += y[0].x + y[0].y;
  }
  if (blockIdx.y == 0) {
    const int i = threadIdx.x;
    auto one = [&](float x) { rebase(fmaxf(top, x)); sum += kv::ex2(fmaf(x, p.c, -ref)); };
    if (i < head) one(to_f32(row[i]));
    if (tail + i < p.vocab) one(to_f32(row[tail + i]));      // (fewer than W left)
  }
  // the largest score of all threads, then their sums against it
  float t = top;
#pragma unroll
  for (int w = 16; w; w >>= 1) t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, w));
  if ((threadIdx.x & 31) == 0) s_top[threadIdx.x >> 5] = t;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < STAT_THREADS / 32; ++w) t = fmaxf(t, s_top[w]);
  rebase(t);
#pragma unroll
  for (int w = 16; w; w >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, w);
  if ((threadIdx.x & 31) == 0) s_sum[threadIdx.x >> 5] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    sum = 0.f;
#pragma unroll
    for (int w = 0; w < STAT_THREADS / 32; ++w) sum += s_sum[w];
    p.stats[((size_t)blockIdx.z * p.M + blockIdx.x) * p.parts + blockIdx.y] = Stat{top, sum};
  }
}

enum Decision { KEEP = 0, STOP = 1, NEAR = 2, DROP = 3 };     // STOP: kept, and the end of the output.  NEAR: too close to call in 32 bits

namespace cg = cooperative_groups;

// exp(y), y <= 0, to the last bits of FP64: y = k ln2 / 64 + f, exp(y) = 2^(k / 64) exp(f), the first from a table of 2^(j / 64) and the exponent, the
// second from its Taylor series up to f^5 (f^6 / 720 < 4e-17), the table-driven scheme of Tang (1989).  A third of the FP64 operations of exp(), and these bound
// the kernel.
constexpr int EXP_TABLE = 64;
__device__ __forceinline__ double exp_below(double y, const double* table) {
  y = fmax(y, -746.0);
  const double ROUND = 6755399441055744.0;                                  // 1.5 * 2^52: the sum's low word is k
  const double kd = fma(y, 64.0 / 0.693147180559945309417, ROUND);
  const int k = __double2loint(kd);
  const double kr = kd - ROUND;
  const double f = fma(kr, -2.3190468138462996e-17 / 64.0, fma(kr, -0.69314718055994530942 / 64.0, y));     // ln 2 as a double, and the rest of it
  double e = fma(f, 1.0 / 120.0, 1.0 / 24.0);
  e = fma(f, e, 1.0 / 6.0);
  e = fma(f, e, 0.5);
  e = fma(f, e, 1.0);
  e = fma(f, e, 1.0) * table[k & (EXP_TABLE - 1)];
  const int n = k >> 6, h = n >> 1;                                          // (in two steps: the result may be subnormal)
  return e * __hiloint2double((h + 1023) << 20, 0) * __hiloint2double((n - h + 1023) << 20, 0);
}

// Exchange between the CTAs of a cluster, one slot per CTA.
constexpr int MAX_CLUSTER = 8;
struct Exchange {
  double sum[2][2][MAX_CLUSTER];    // (two sets, taken in turn)
  int pick[2][MAX_CLUSTER];         // [lowest hit, highest token with weight]
};
constexpr int AT_ONCE = 8;          // scores under way per thread and row

// The decision for one row, by one cluster.
//   Position i keeps its draft d while u_i q_i(d) < p_i(d).  The first one that does not gets the token at which the running sum of
//   max(p_i - q_i, 0), in the order of ids, passes r times its total, and is the last (n = i + 1); without a draft the sum is p_i's own.
// A token that is drawn depends on sums over the vocabulary to the last bit near a border, and a decision on a comparison; both have to come out as
// the formula says and alike for every way of adding up.  So decisions are taken from the 32-bit sums of score_stats_kernel only where these leave no
// doubt, and else, like the draw, from sums in 64 bits over the one position's scores, which are still in L2.  With weights w = exp((score - top) / T)
// and their sums z, p and q enter as w_p z_q and w_q z_p, multiples of the probabilities that need no division.
// Bound by latency: decisions, one sweep over the position's scores and three exchanges in a row (from a cold start 20 us for one row, 25 for 32).  KEPT: the weights of the sweep stay in shared memory
// for the sum and the draw, else they are computed again.
// grid = B clusters of CTAs that share the vocabulary, block = ACCEPT_THREADS.  Every CTA of a cluster takes the same decisions from the same numbers.
// Dynamic shared memory: KEPT, a double per score of the CTA's share, of one or two rows.
template <typename T, bool KEPT>
__global__ void __launch_bounds__(ACCEPT_THREADS)
accept_sampled_kernel(Params p) {
  constexpr int WARPS = ACCEPT_THREADS / 32;
  extern __shared__ double s_weight[];
  __shared__ double s_table[EXP_TABLE], s_warp[2][WARPS];
  __shared__ int s_first[1], s_pick[2];
  __shared__ float s_top[2];
  __shared__ Exchange s_ex;
  cg::cluster_group cluster = cg::this_cluster();
  const int rank = cluster.block_rank(), size = cluster.num_blocks(), b = blockIdx.x / size, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  pdl_launch();
  if (tid < EXP_TABLE) s_table[tid] = exp2(tid / (double)EXP_TABLE);
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
  cluster.barrier_arrive();                                 // (another CTA's shared memory may be written once that CTA runs)
  bool met = false;
  const bool two = p.score[1] != nullptr;
  const T* prow = static_cast<const T*>(p.score[0]) + (size_t)o * p.stride[0];
  const T* qrow = static_cast<const T*>(p.score[1]) + (size_t)o * p.stride[1];
  auto draft_at = [&](int i) {
    const int d = __ldg(drafts + i);
    return d < p.vocab ? d : -1;
  };

  // ---- a score's weight: 1 at the top (even where it is infinite), 0 for a NaN and where there is no top ----
  auto weight = [&](float x, float top) {
    if (x == top) return top == -INFINITY ? 0.0 : 1.0;
    return x < top && !isinf(top) ? exp_below(((double)x - (double)top) * p.inv_t, s_table) : 0.0;
  };
  auto row_stat = [&](int z, int i) {
    constexpr int PARTS = 16;                               // under way at once
    Stat s = {-INFINITY, 0.f};
    const float2* part = reinterpret_cast<const float2*>(p.stats + ((size_t)z * p.M + o + i) * p.parts);
    for (int j0 = 0; j0 < p.parts; j0 += PARTS) {
      float2 t[PARTS];
#pragma unroll
      for (int j = 0; j < PARTS; ++j) t[j] = j0 + j < p.parts ? __ldcg(part + j0 + j) : make_float2(-INFINITY, 0.f);
#pragma unroll
      for (int j = 0; j < PARTS; ++j)
        if (j0 + j < p.parts) join(s, Stat{t[j].x, t[j].y}, p.c);
    }
    return s;
  };

  // ---- a position's decision from the 32-bit sums ----
  float my_top[2] = {0.f, 0.f};
  auto decide = [&](int i) -> int {
    const int d = draft_at(i);
    const float xp = d < 0 ? 0.f : to_f32(prow[(size_t)i * p.stride[0] + d]), xq = two && d >= 0 ? to_f32(qrow[(size_t)i * p.stride[1] + d]) : 0.f;
    const Stat sp = row_stat(0, i), sq = two ? row_stat(1, i) : Stat{0.f, 1.f};
    my_top[0] = sp.top;
    my_top[1] = sq.top;
    if (d < 0) return DROP;
    const float rp = reference(sp.top, p.c), rq = reference(sq.top, p.c);
    if (!isfinite(sp.top) || !isfinite(sp.sum) || !isfinite(sq.top) || !isfinite(sq.sum)) return NEAR;
    // Scores over T beyond 2^26: FP32's steps put the reference so far from the maximum (10 exponents there, 128 and more from 2^30 on) that sums vanish.
    if (!(fabsf(rp) <= 67108864.f) || !(fabsf(rq) <= 67108864.f)) return NEAR;
    if (xp != xp || xq != xq) return NEAR;
    const double qd = two ? exp2((double)xq * p.c - rq) : 1.0;
    const double want = (double)__ldg(p.u + (size_t)b * p.kmax + i) * qd * (double)sp.sum;
    const double have = exp2((double)xp * p.c - rp) * (double)sq.sum;
    // How far off the two may be, relatively.  A sum: chains of at most 128 additions in all, 2^-24 each, and an exponential within 2^-21; 1.6e-5 for both
    // sums.  Moving maxima round nothing.  An exponent is rounded to 2^-24 of itself and the factor c is off by as much, which moves a sum by these shares of
    // the mean distance from the top (20 exponents at most, with 2^20 scores) and an exponential by one of its own distance; 4e-6 and the last term.
    const double away = (isinf(xp) ? 0.0 : (double)(sp.top - xp)) + (two && !isinf(xq) ? (double)(sq.top - xq) : 0.0);
    const double doubt = 3e-5 + 1.2e-7 * away * p.c;
    if (fabs(want - have) <= doubt * fmax(fabs(want), have)) return NEAR;
    return want < have ? (d == p.eos ? STOP : KEEP) : DROP;
  };

  // ---- sums over the cluster in the order of its threads: of x (in front of this thread's, and all), and of y (all) ----
  int turn = 0;
  auto cluster_sums = [&](double x, double y, double& before, double& all_x, double& all_y) {
    double run = x;
#pragma unroll
    for (int w = 1; w < 32; w <<= 1) {
      const double v = __shfl_up_sync(0xffffffffu, run, w);
      if (lane >= w) run += v;
      y += __shfl_xor_sync(0xffffffffu, y, w);
    }
    __syncthreads();
    if (lane == 31) { s_warp[0][warp] = run; s_warp[1][warp] = y; }
    __syncthreads();
    double mine = 0.0, front = 0.0, mine_y = 0.0;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) {
      if (w == warp) front = mine;
      mine += s_warp[0][w];
      mine_y += s_warp[1][w];
    }
    const int slot = turn & 1;
    if (!met) { cluster.barrier_wait(); met = true; }
    if (tid < 2 * size) cluster.map_shared_rank(&s_ex, tid >> 1)->sum[slot][tid & 1][rank] = tid & 1 ? mine_y : mine;
    cluster.sync();
    double ahead = 0.0;
    all_x = all_y = 0.0;
    for (int j = 0; j < size; ++j) {
      if (j == rank) ahead = all_x;
      all_x += s_ex.sum[slot][0][j];
      all_y += s_ex.sum[slot][1][j];
    }
    before = ahead + front + (run - x);
    ++turn;
  };
  // this thread's share of the vocabulary
  const int each = (p.vocab + size * ACCEPT_THREADS - 1) / (size * ACCEPT_THREADS);
  const int v0 = min((rank * ACCEPT_THREADS + tid) * each, p.vocab), v1 = min(v0 + each, p.vocab);
  // calls f(v, weight of the verifier's score v, of the drafter's) over it
  auto sweep = [&](const T* pr, const T* qr, float ptop, float qtop, auto f) {
    for (int e0 = v0; e0 < v1; e0 += AT_ONCE) {
      float xp[AT_ONCE], xq[AT_ONCE];
#pragma unroll
      for (int e = 0; e < AT_ONCE; ++e) {
        xp[e] = e0 + e < v1 ? to_f32(pr[e0 + e]) : 0.f;
        xq[e] = two && e0 + e < v1 ? to_f32(qr[e0 + e]) : 0.f;
      }
#pragma unroll
      for (int e = 0; e < AT_ONCE; ++e)
        if (e0 + e < v1) f(e0 + e, weight(xp[e], ptop), two ? weight(xq[e], qtop) : 0.0);
    }
  };
  auto kept = [&](int z, int v) -> double& { return s_weight[(size_t)(z * each + v - v0) * ACCEPT_THREADS + tid]; };

  int first = -1, how = KEEP, from = 0;      // the first position that does not simply keep its draft
  double zp = 0.0, zq = 1.0;
  float ptop = 0.f, qtop = 0.f;
  const T *pr = prow, *qr = qrow;
  for (;;) {
    if (tid == 0) s_first[0] = INT_MAX;
    __syncthreads();
    int mine_first = -1;
    for (int i = from + tid; i < k; i += ACCEPT_THREADS) {
      const int h = decide(i);
      if (h != KEEP) { mine_first = 4 * i + h; atomicMin(&s_first[0], mine_first); break; }              // (an integer minimum: no order in it)
    }
    __syncthreads();
    if (mine_first == s_first[0]) { s_top[0] = my_top[0]; s_top[1] = my_top[1]; }
    __syncthreads();
    first = s_first[0] == INT_MAX ? k : s_first[0] >> 2;
    how = s_first[0] == INT_MAX ? KEEP : s_first[0] & 3;
    if (how == KEEP || how == STOP) break;
    // the position's sums in 64 bits
    ptop = s_top[0];
    qtop = s_top[1];
    pr = prow + (size_t)first * p.stride[0];
    qr = qrow + (size_t)first * p.stride[1];
    double a = 0.0, c = 0.0, unused;
    sweep(pr, qr, ptop, qtop, [&](int v, double wp, double wq) {
      a += wp;
      c += wq;
      if (KEPT) {
        kept(0, v) = wp;
        if (two) kept(1, v) = wq;
      }
    });
    cluster_sums(a, c, unused, zp, zq);
    if (!two || !(zq > 0.0)) zq = 1.0;                      // (no drafter, or one without a distribution: its weights are 0)
    if (how == DROP) break;
    const int d = draft_at(first);
    const double pd = weight(to_f32(pr[d]), ptop), qd = two ? weight(to_f32(qr[d]), qtop) : 1.0;
    if (!((double)__ldg(p.u + (size_t)b * p.kmax + first) * qd * zp < pd * zq)) { how = DROP; break; }
    if (d == p.eos) { how = STOP; break; }
    from = first + 1;
    __syncthreads();
    if (from == k) { first = k; how = KEEP; break; }
  }

  // ---- the token of the first position that does not keep its draft ----
  int token = 0;
  if (how == DROP) {
    const int d = draft_at(first);
    const double r = (double)__ldg(p.r + b);
    for (int form = d < 0 ? 1 : 0; form < 2; ++form) {      // 0: what the verifier gives beyond the drafter; 1: the verifier's own
      auto left = [&](int v, double wp, double wq) {
        if (form == 1) return wp;
        if (!two) return v == d ? 0.0 : wp;
        return fmax(__dmul_rn(wp, zq) - __dmul_rn(wq, zp), 0.0);     // (each rounded: equal distributions leave nothing, not one product's rounding)
      };
      auto over = [&](auto f) {                             // f(v, what is left of v)
        if constexpr (KEPT) {
          for (int v = v0; v < v1; ++v) f(v, left(v, kept(0, v), two ? kept(1, v) : 0.0));
        } else {
          sweep(pr, qr, ptop, qtop, [&](int v, double wp, double wq) { f(v, left(v, wp, wq)); });
        }
      };
      double mine = 0.0, before, all, unused;
      int last = -1;
      over([&](int v, double x) {
        mine += x;
        if (x > 0.0) last = v;
      });
      if (tid == 0) { s_pick[0] = INT_MAX; s_pick[1] = -1; }
      cluster_sums(mine, 0.0, before, all, unused);
      if (form == 0 && !(all > 0.0)) continue;              // (nothing beyond the drafter's: the verifier's own)
      int hit = INT_MAX;
      const double goal = r * all;
      if (before + mine > goal) {
        double run = before;
        over([&](int v, double x) {
          run += x;
          if (x > 0.0 && run > goal) hit = min(hit, v);
        });
      }
      hit = __reduce_min_sync(0xffffffffu, hit);
      last = __reduce_max_sync(0xffffffffu, last);
      if (lane == 0) {
        atomicMin(&s_pick[0], hit);
        atomicMax(&s_pick[1], last);
      }
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
  if (!met) cluster.barrier_wait();
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
