// A pool of cache blocks that rows share: forking rows, handing out blocks with copies of what is shared, and moving what is in use to the front.
#pragma once

#include <cooperative_groups.h>
#include <limits.h>

#include "kv_cache.cuh"

namespace ad {
namespace pool {

namespace cg = cooperative_groups;

struct Pool {
  int* table;                    // [rows, stride]: block i of row b, negative: none
  int* refs;                     // [n_blocks]: entries of the table that name the block
  int rows, stride, n_blocks, block;
  __host__ __device__ __forceinline__ bool there(int id) const { return (unsigned)id < (unsigned)n_blocks; }
};

// ---- forking -----------------------------------------------------------------------------------------------------
// What a row is to be: nothing (its parent is negative), the first `held` blocks of a row of the call, or, where the wish makes no sense, as it was.
enum Wish { EMPTY = -1, AS_IT_WAS = -2 };
struct Heir { int parent, held; };
__host__ __device__ __forceinline__ Heir heir(const Pool& p, int B, int parent, int len, int& fault) {
  fault = AD_OK;
  if (parent < 0) return Heir{EMPTY, 0};
  if (parent >= B || len < 0) fault = AD_ERR_ARG;
  else if (len > p.stride * p.block) fault = AD_ERR_CAPACITY;
  if (fault != AD_OK) return Heir{AS_IT_WAS, 0};
  return Heir{parent, len / p.block + (len % p.block != 0)};
}

// Row b becomes the first len[b] tokens of what row parent[b] was.  A column of the table depends on itself alone, so a CTA takes `width` columns of
// all rows into shared memory and writes them back from there; what changes is counted in refs, by integer additions, whose order does not matter.
// Bound by latency for ordinary batches: two round trips, no other CTA to wait for.  8 rows: 5.6 us a call, 4.0 of the kernel
// alone.  512 rows of up to 2000 blocks, 8.4 MB read and written and half a million additions to counts: 15 us a call, 0.56 TB/s.
// grid = ceil(stride / width), dynamic shared memory = B * width entries.
constexpr int FORK_THREADS = 512;
__global__ void __launch_bounds__(FORK_THREADS)
cache_fork_kernel(Pool p, const int* __restrict__ parent, const int* __restrict__ len, int B, int shift, int* status) {
  extern __shared__ int s_old[];
  pdl_launch();
  pdl_wait();
  const int width = 1 << shift, c0 = blockIdx.x * width;
  for (int e = threadIdx.x; e < B << shift; e += FORK_THREADS) {
    const int col = c0 + (e & (width - 1));
    s_old[e] = col < p.stride ? p.table[(size_t)(e >> shift) * p.stride + col] : -1;
  }
  __syncthreads();
  for (int e = threadIdx.x; e < B << shift; e += FORK_THREADS) {
    const int b = e >> shift, c = e & (width - 1), col = c0 + c;
    if (col >= p.stride) continue;
    int fault;
    const Heir h = heir(p, B, __ldg(parent + b), __ldg(len + b), fault);
    if (fault != AD_OK && col == 0) latch_error(status, fault);
    if (h.parent == AS_IT_WAS) continue;
    const int old = s_old[e];
    int to = -1;
    if (h.parent >= 0 && col < h.held) {
      to = s_old[(h.parent << shift) + c];
      if (!p.there(to)) { to = -1; latch_error(status, AD_ERR_ARG); }       // (tokens that the parent has no block for)
    }
    if (to == old) continue;
    p.table[(size_t)b * p.stride + col] = to;
    if (p.there(old)) atomicAdd(p.refs + old, -1);
    if (to >= 0) atomicAdd(p.refs + to, 1);
  }
}

// ---- planning kernels: one cluster ---------------------------------------------------------------------------------
// Whatever is numbered in order (free blocks, rows' needs) is counted by ranges, one per warp of the cluster: a count, the ranges' counts added up in front of
// each, then the same walk again with its number at hand.
constexpr int PLAN_THREADS = 1024, PLAN_WARPS = PLAN_THREADS / 32, MAX_CLUSTER = 8, COUNTS = 3;      // at most (warps of a CTA: a power of two)
struct Move { int src, dst, live; };       // `live` tokens of block src go to block dst
struct Plan {
  Pool p;
  int2* claim;                   // reserve, [n_blocks]: rows that write the block although others hold it, and the first of them
  int* list;                     // reserve: free blocks in order; compact: holes, then, behind n_blocks of them, movers
  int* map;                      // compact, [n_blocks]: where a block goes
  Move* moves;
  int* n_moves;
};

struct Counting {
  int warp[COUNTS][PLAN_WARPS];
  int cta[COUNTS];
};
// n[i] of this warp's range -> what lies in front of it in all ranges of the cluster, and all there is.  Every lane of a warp has the same n.
// Barriers of the whole cluster on both sides.
template <int N>
__device__ __forceinline__ void cluster_counts(cg::cluster_group& cluster, Counting& s, const int (&n)[N], int (&front)[N], int (&all)[N]) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, rank = cluster.block_rank();
  if (lane == 0)
#pragma unroll
    for (int i = 0; i < N; ++i) s.warp[i][warp] = n[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int x = lane < (int)blockDim.x / 32 ? s.warp[i][lane] : 0;
    front[i] = __reduce_add_sync(0xffffffffu, lane < warp ? x : 0);
    const int sum = __reduce_add_sync(0xffffffffu, x);
    if (threadIdx.x == 0) s.cta[i] = sum;
  }
  cluster.sync();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    all[i] = 0;
    for (int r = 0; r < (int)cluster.num_blocks(); ++r) {
      if (r == rank) front[i] += all[i];
      all[i] += *cluster.map_shared_rank(&s.cta[i], r);
    }
  }
  cluster.sync();
}
// A warp's part of n things that lie in order.
__device__ __forceinline__ void warp_range(cg::cluster_group& cluster, int n, int& lo, int& hi) {
  const int each = blockDim.x >> 5, warps = cluster.num_blocks() * each, w = cluster.block_rank() * each + (threadIdx.x >> 5);
  lo = (int)((long long)n * w / warps);
  hi = (int)((long long)n * (w + 1) / warps);
}
// Calls f(id, whether it is in the range, refs[id]) for ids lo .. hi - 1, 32 at a time, several loads under way.
template <typename F>
__device__ __forceinline__ void walk_refs(const int* refs, int lo, int hi, F f) {
  constexpr int AHEAD = 8;
  const int lane = threadIdx.x & 31;
  for (int i0 = lo; i0 < hi; i0 += 32 * AHEAD) {
    int x[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) x[u] = i0 + u * 32 + lane < hi ? __ldcg(refs + i0 + u * 32 + lane) : 0;
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
      if (i0 + u * 32 < hi) f(i0 + u * 32 + lane, i0 + u * 32 + lane < hi, x[u]);
  }
}

// ---- handing out blocks ------------------------------------------------------------------------------------------
// The blocks first .. last of a row that its new tokens are written to; false: none, or not to be served.
struct Span { int first, last, live; };      // live: tokens in front of the new ones in block `first`
__host__ __device__ __forceinline__ bool span_of(const Pool& p, int off0, int off1, int len, Span& s, int& fault) {
  fault = AD_OK;
  if (off1 == off0) return false;
  const long long n = (long long)off1 - off0;
  if (off0 < 0 || n < 0 || len < 0) fault = AD_ERR_ARG;
  else if (n + len > (long long)p.stride * p.block) fault = AD_ERR_CAPACITY;
  if (fault != AD_OK) return false;
  s.first = len / p.block;
  s.last = (int)((n + len - 1) / p.block);
  s.live = len % p.block;
  return true;
}

// Rows get the blocks that they lack for new tokens off[b] .. off[b + 1] behind their first len[b], and blocks of their own in place of those that others hold
// too.  Of the rows that write the same block the first keeps it where nobody else holds it; all others leave it.  Fresh blocks are the free ones
// in ascending order, handed out in the order of rows and of blocks within a row: nothing here depends on the order in which threads run.  A pool with too few
// of them latches AD_ERR_CAPACITY and stays as it is.  moves[b]: what the copy kernel is to do for row b.
// Bound by latency: eight barriers, as many round trips, and its own instructions, which come from memory when others have run in between (8 rows: 10 us alone and cold, of
// which 3 are spent on loops that have nothing to do).  256 rows of 1678 blocks, a cluster: 15 us.  (Claims and lists of a single CTA in shared memory, with barriers of
// its own: the same.)
// grid = one cluster, block = PLAN_THREADS or less.
__global__ void __launch_bounds__(PLAN_THREADS)
cache_reserve_kernel(Plan a, const int* __restrict__ off, const int* __restrict__ len, int B, int* status) {
  __shared__ Counting s_count;
  cg::cluster_group cluster = cg::this_cluster();
  const Pool& p = a.p;
  const int lane = threadIdx.x & 31;
  pdl_launch();
  pdl_wait();
  int row0, row1, id0, id1;
  warp_range(cluster, B, row0, row1);
  warp_range(cluster, p.n_blocks, id0, id1);
  // f(entry's place in the table, block of the row, what it names or -1) for every entry that row b writes, by all lanes of a warp
  auto entries = [&](int b, const Span& s, auto f) {
    for (int i0 = s.first; i0 <= s.last; i0 += 32) {
      const int i = i0 + lane;
      const bool in = i <= s.last;
      const int at = b * p.stride + i;               // (fewer than 2^31 entries)
      const int e = in ? __ldcg(p.table + at) : -1;
      f(at, i, in, p.there(e) ? e : -1);
    }
  };
  auto span = [&](int b, Span& s, bool tell) {
    int fault;
    const bool some = span_of(p, __ldg(off + b), __ldg(off + b + 1), __ldg(len + b), s, fault);
    if (tell && fault != AD_OK && lane == 0) latch_error(status, fault);
    return some;
  };
  for (int id = id0 + lane; id < id1; id += 32) a.claim[id] = make_int2(0, INT_MAX);
  cluster.sync();
  Span s;
  for (int b = row0; b < row1; ++b)
    if (span(b, s, true))
      entries(b, s, [&](int at, int, bool, int e) {
        if (e >= 0 && __ldcg(p.refs + e) > 1) {
          atomicAdd(&a.claim[e].x, 1);
          atomicMin(&a.claim[e].y, at);
        }
      });
  cluster.sync();
  // Whether an entry gets another block.  `writers` of a block that others hold: more than none; only the first of them looks at refs, and changes it below.
  auto fresh = [&](int at, bool in, int e, int& writers, bool& first) {
    if (e < 0) return in;
    const int2 c = __ldcg(a.claim + e);
    writers = c.x;
    first = c.x > 0 && c.y == at;
    return c.x > 0 && !(first && __ldcg(p.refs + e) == c.x);
  };
  int need = 0, spare = 0;
  for (int b = row0; b < row1; ++b)
    if (span(b, s, false))
      entries(b, s, [&](int at, int, bool in, int e) {
        int writers;
        bool first;
        need += __popc(__ballot_sync(0xffffffffu, fresh(at, in, e, writers, first)));
      });
  walk_refs(p.refs, id0, id1, [&](int, bool in, int refs) { spare += __popc(__ballot_sync(0xffffffffu, in && refs == 0)); });
  int front[2], all[2];
  cluster_counts(cluster, s_count, {need, spare}, front, all);
  const bool enough = all[0] <= all[1];
  if (!enough && threadIdx.x == 0 && cluster.block_rank() == 0) latch_error(status, AD_ERR_CAPACITY);
  if (enough && front[1] < all[0]) {
    int at = front[1];
    walk_refs(p.refs, id0, id1, [&](int id, bool in, int refs) {
      const unsigned free = __ballot_sync(0xffffffffu, in && refs == 0);
      const int mine = at + __popc(free & ((1u << lane) - 1u));
      if ((free >> lane & 1u) && mine < all[0]) a.list[mine] = id;
      at += __popc(free);
    });
  }
  cluster.sync();
  int at_list = front[0];
  for (int b = row0; b < row1; ++b) {
    if (lane == 0) a.moves[b] = Move{-1, 0, 0};
    __syncwarp();
    if (!enough || !span(b, s, false)) continue;
    entries(b, s, [&](int at, int i, bool in, int e) {
      int writers = 0;
      bool first = false;
      const bool mine = fresh(at, in, e, writers, first);
      const unsigned some = __ballot_sync(0xffffffffu, mine);
      if (mine) {
        const int id = __ldcg(a.list + at_list + __popc(some & ((1u << lane) - 1u)));
        p.table[at] = id;
        p.refs[id] = 1;
        if (e >= 0 && i == s.first && s.live > 0) a.moves[b] = Move{e, id, s.live};
      }
      // those that leave: all writers but a first one that keeps it
      if (first) p.refs[e] = __ldcg(p.refs + e) - (mine ? writers : writers - 1);
      at_list += __popc(some);
    });
  }
}

// ---- moving what is in use to the front --------------------------------------------------------------------------
// With U blocks in use, those from U on go to the free ones in front of U, both in ascending order.  Bound by latency, as above: 6.5 us alone and cold.
// grid = one cluster, block = PLAN_THREADS or less.
__global__ void __launch_bounds__(PLAN_THREADS)
cache_compact_kernel(Plan a, int* n_used) {
  __shared__ Counting s_count;
  cg::cluster_group cluster = cg::this_cluster();
  const Pool& p = a.p;
  const int lane = threadIdx.x & 31;
  pdl_launch();
  pdl_wait();
  int id0, id1, used = 0, movers = 0;
  warp_range(cluster, p.n_blocks, id0, id1);
  walk_refs(p.refs, id0, id1, [&](int, bool in, int refs) { used += __popc(__ballot_sync(0xffffffffu, in && refs > 0)); });
  int front[1], all[1], unused[1];
  cluster_counts(cluster, s_count, {used}, front, all);
  const int U = all[0];
  int at = front[0];
  walk_refs(p.refs, id0, id1, [&](int id, bool in, int refs) {
    const unsigned busy = __ballot_sync(0xffffffffu, in && refs > 0);
    const int before = at + __popc(busy & ((1u << lane) - 1u));          // blocks in use in front of id
    if (in && id < U && refs <= 0) a.list[id - before] = id;              // the holes, in order
    if (in && id >= U) {
      if (refs > 0) a.list[p.n_blocks + U - 1 - before] = id;            // the movers, from the last one on
      else a.map[id] = id;
    }
    at += __popc(busy);
    movers += __popc(__ballot_sync(0xffffffffu, in && id >= U && refs > 0));
  });
  cluster_counts(cluster, s_count, {movers}, unused, all);
  const int H = all[0];                                                   // (as many holes in front of U as blocks in use behind it)
  for (int j = cluster.block_rank() * blockDim.x + threadIdx.x; j < H; j += cluster.num_blocks() * blockDim.x) {
    const int dst = __ldcg(a.list + j), src = __ldcg(a.list + p.n_blocks + H - 1 - j);
    a.moves[j] = Move{src, dst, p.block};
    a.map[src] = dst;
    p.refs[dst] = __ldcg(p.refs + src);
    p.refs[src] = 0;
  }
  if (threadIdx.x == 0 && cluster.block_rank() == 0) {
    *a.n_moves = H;
    *n_used = U;
  }
}

// ---- moving contents -----------------------------------------------------------------------------------------------
struct Layer {
  uint8_t* codes[2];
  float* scale[2];
  int heads, dim;
};
constexpr int MAX_LAYERS = 64;
struct Contents {
  Layer layer[MAX_LAYERS];
  int n_layers;
  const Move* moves;
  const int* n_moves;            // null: n of them
  int n, block;
  // compact: entries of the table that get another number (null: none)
  int* table;
  long long entries;
  const int* map;
  const int* n_used;
  int n_blocks;
};
// Does the moves, in every layer: codes of the live tokens and the scales, head by head, each of which lies in one piece.  A warp takes a head's keys or values
// at a time, 16 bytes a lane and up to eight of them under way.  Bound by bytes: 64 rows of
// 700-2100 tokens, six layers of 8 heads of 128 (1.14 GB read and written): 172 us, 6.6 TB/s; copies of partly filled blocks for 224 of 256 rows
// (186 MB): 24 us, 7.8 TB/s, part of it from L2.
// grid = (CTAs a layer, layers, and one more row of CTAs for the table), block = COPY_THREADS.
constexpr int COPY_THREADS = 256, COPY_AHEAD = 8;
__global__ void __launch_bounds__(COPY_THREADS)
cache_move_kernel(const __grid_constant__ Contents a) {
  pdl_launch();
  pdl_wait();
  const int lane = threadIdx.x & 31;
  if ((int)blockIdx.y == a.n_layers) {
    const int used = __ldcg(a.n_used);
    for (long long i = (long long)blockIdx.x * COPY_THREADS + threadIdx.x; i < a.entries; i += (long long)gridDim.x * COPY_THREADS) {
      const int e = a.table[i];
      if (e >= used && e < a.n_blocks) a.table[i] = __ldcg(a.map + e);
    }
    return;
  }
  const Layer& l = a.layer[blockIdx.y];
  const int n = a.n_moves ? __ldcg(a.n_moves) : a.n, each = 2 * l.heads;
  const long long items = (long long)n * each;
  for (long long item = (long long)blockIdx.x * (COPY_THREADS / 32) + (threadIdx.x >> 5); item < items; item += (long long)gridDim.x * (COPY_THREADS / 32)) {
    const int j = (int)(item / each), r = (int)(item % each), head = r >> 1;
    const Move m = {__ldcg(&a.moves[j].src), __ldcg(&a.moves[j].dst), __ldcg(&a.moves[j].live)};
    if (m.src < 0) continue;
    uint8_t* codes = r & 1 ? l.codes[1] : l.codes[0];
    float* scale = r & 1 ? l.scale[1] : l.scale[0];
    const size_t from = (size_t)m.src * l.heads + head, to = (size_t)m.dst * l.heads + head;
    const int bytes = m.live * l.dim;                          // a multiple of 32
    const uint8_t* src = codes + from * a.block * l.dim;
    uint8_t* dst = codes + to * a.block * l.dim;
    if (lane == 0) scale[to] = __ldcg(scale + from);
    for (int o = lane * 16; o < bytes; o += 512 * COPY_AHEAD) {
      uint4 v[COPY_AHEAD];
#pragma unroll
      for (int u = 0; u < COPY_AHEAD; ++u)
        if (o + u * 512 < bytes) v[u] = __ldcs(reinterpret_cast<const uint4*>(src + o + u * 512));
#pragma unroll
      for (int u = 0; u < COPY_AHEAD; ++u)
        if (o + u * 512 < bytes) __stcs(reinterpret_cast<uint4*>(dst + o + u * 512), v[u]);
    }
  }
}

}  // namespace pool
}  // namespace ad
