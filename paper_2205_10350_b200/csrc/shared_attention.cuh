// Attention over the 8-bit key/value cache for rows that share prefixes: the shared positions once for all rows of a group, on the tensor cores' own memory.
#pragma once

#include "cache_attention.cuh"
#include "gemm_tc.cuh"

namespace ad {
namespace shr {

using kv::Cache;

constexpr int KEYS = 128;              // keys of a tile
constexpr int SUB = 64;                // ... of which scores are worked on so many at a time
constexpr int M_ROWS = 128;            // rows of an MMA
constexpr int ITEM_ROWS = 256;         // most rows of an item, and the distance of CTAs' parts in scratch

// What is worked on: a line for every group, its rows' queries over the blocks that they share.  A line has `heads` times `tiles` (of its rows) items, each over all
// of its keys; an item is `per` granules: FIXED ones, and `weight`, one or two, for every tile of keys.  The CTAs share all granules evenly, in order.  What the rows have besides is left to the
// attention row by row; behind the groups' lines each row of the batch has one that says which queries are its own, and of which group.
// `row`: the one whose table names the group's blocks.
struct Line {
  long long front, rows_front;         // granules and rows of results in front of it
  int o, n, keys;                      // tokens o .. o + n - 1; keys that they share
  int row, tiles, per, weight, group, pad[4];
};
static_assert(sizeof(Line) == 64, "four 16-byte loads");
struct Start { int line, pad; long long at; };
struct Total {
  long long all, each;                 // granules of all lines; of a CTA, in order (the last ones may get fewer, or none)
  int own_whole;                       // no row has so many positions of its own that they are split
};

struct Params {
  Cache c;
  const void* q;
  size_t q_stride;
  void* out;
  int n_heads, M, max_new, B, G;
  const int* off;
  const int* len;
  const int* group;
  const int* shared;
  int causal;
  float scale;                         // softmax scale times log2(e)
  int* status;
  int grid, item_rows;                 // CTAs; rows of an item
  long long part_rows;                 // rows of results of one half
  // scratch
  Total* total;
  Line* lines;                         // [G + B]
  Start* start;                        // [grid]
  int* own_first;                      // [B] blocks that row b shares, and positions behind them (negative: the row is left out)
  int* own_len;
  float2* ml;                          // [2][part_rows] maxima and sums
  float* part;                         // [2][part_rows][dim] means of values
  float2* own_ml;                      // [M][n_heads] the same of the rows' own positions, where one CTA worked on them
  float* own_part;                     // [M][n_heads][dim]
  kv::Parts own;                       // ... and where several did
};

constexpr int FIXED = 3;
__host__ __device__ __forceinline__ int key_tiles(int keys) { return (keys + KEYS - 1) / KEYS; }
// The tile that granule x of an item starts with.
__host__ __device__ __forceinline__ int tile_at(int x, int weight) { return x <= FIXED ? 0 : (x - FIXED + weight - 1) >> (weight - 1); }

// Units of keys that a row has of its own.
__device__ __forceinline__ int own_units(const Params& a, int len, int n) { return (len + (a.causal ? n : 0) + kv::UNIT - 1) / kv::UNIT; }

// ---- plan ----------------------------------------------------------------------------------------------------------
constexpr int PLAN_THREADS = 256;
__device__ __forceinline__ long long block_scan(long long x, long long* s_warp, long long& all) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  long long run = x;
#pragma unroll
  for (int w = 1; w < 32; w <<= 1) {
    const long long y = __shfl_up_sync(0xffffffffu, run, w);
    if (lane >= w) run += y;
  }
  __syncthreads();
  if (lane == 31) s_warp[warp] = run;
  __syncthreads();
  long long front = run - x;
  all = 0;
  for (int w = 0; w < PLAN_THREADS / 32; ++w) {
    if (w < warp) front += s_warp[w];
    all += s_warp[w];
  }
  return front;
}
// Tokens of group g, and the positions that its rows share; false: it makes no sense.
__device__ __forceinline__ bool group_of(const Params& a, int g, int& first, int& last, int& o, int& n, int& keys) {
  first = __ldcg(a.group + g);
  last = __ldcg(a.group + g + 1);
  keys = __ldcg(a.shared + g);
  bool good = first >= 0 && last >= first && last <= a.B && keys >= 0 && keys <= a.c.table_stride * a.c.block;
  o = n = 0;
  if (good && first < last) {
    o = __ldcg(a.off + first);
    const long long d = (long long)__ldcg(a.off + last) - o;
    good = o >= 0 && d >= 0 && o + d <= a.M;
    n = good ? (int)d : 0;
  }
  if (!good) latch_error(a.status, AD_ERR_ARG);
  return good;
}
// Bound by latency: four round trips one after another for rows and groups, two more for the CTAs' starts, 6 us alone and cold.  (With 1024 threads 9.5 us.  Starts found by one thread, line after
// line with a 64-bit division for each: 10 more.)
// grid = 1, block = PLAN_THREADS.
__global__ void __launch_bounds__(PLAN_THREADS)
shared_plan_kernel(const __grid_constant__ Params a) {
  __shared__ long long s_warp[PLAN_THREADS / 32];
  pdl_launch();
  pdl_wait();
  const int per_kv = a.n_heads / a.c.heads, tid = threadIdx.x;
  // rows: which group they are of, and what is left for the attention row by row
  bool own_long = false;
  for (int b = tid; b < a.B; b += PLAN_THREADS) {
    Line x = {};
    int lo = 0, hi = a.G - 1;                                // the last group that starts at b or in front of it
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (__ldcg(a.group + mid) <= b) lo = mid;
      else hi = mid - 1;
    }
    x.row = b;
    x.group = lo;
    int first, last, go, gn, keys, p;
    a.own_first[b] = 0;
    a.own_len[b] = -1;
    if (kv::row_tokens(a.c, a.off, a.len, b, a.M, a.max_new, !a.causal, a.status, x.o, x.n, p)) {
      if (group_of(a, lo, first, last, go, gn, keys) && first <= b && b < last && keys <= p && x.o >= go && x.o + x.n <= go + gn) {
        a.own_first[b] = keys / a.c.block;
        a.own_len[b] = p - keys / a.c.block * a.c.block;
        own_long = own_long || own_units(a, a.own_len[b], x.n) >= 2 * a.own.granule;
      } else {
        latch_error(a.status, AD_ERR_ARG);
        x.n = 0;
      }
    } else {
      x.n = 0;
    }
    a.lines[a.G + b] = x;
  }
  own_long = __syncthreads_or(own_long);
  long long granules_front = 0, tokens_front = 0;
  for (int l0 = 0; l0 < a.G; l0 += PLAN_THREADS) {
    const int l = l0 + tid;
    Line x = {};
    if (l < a.G) {
      int last;
      if (!group_of(a, l, x.row, last, x.o, x.n, x.keys)) x.keys = 0;
      if (x.n > 0 && __ldcg(a.off + x.row + 1) <= x.o) {      // the first row that brings tokens: others may have been given up
        int hi = last - 1;
        while (x.row < hi) {
          const int mid = (x.row + hi) >> 1;
          if (__ldcg(a.off + mid + 1) > x.o) hi = mid;
          else x.row = mid + 1;
        }
      }
      x.keys -= x.keys % a.c.block;                           // (whole blocks; the rest is the rows' own)
    }
    // no more results than there is room for, whatever the offsets
    long long all_t, all;
    const long long front = tokens_front + block_scan(x.n, s_warp, all_t);
    if (front + x.n > a.M) {
      x.n = 0;
      latch_error(a.status, AD_ERR_ARG);
    }
    const int rows = x.n * per_kv;
    x.rows_front = front * a.n_heads;
    x.tiles = x.keys > 0 ? (rows + a.item_rows - 1) / a.item_rows : 0;
    x.weight = a.item_rows > M_ROWS && rows > M_ROWS ? 2 : 1;
    x.per = key_tiles(x.keys) * x.weight + FIXED;
    x.front = granules_front + block_scan((long long)a.c.heads * x.tiles * x.per, s_warp, all);
    if (l < a.G) a.lines[l] = x;
    granules_front += all;
    tokens_front += all_t;
  }
  const long long total = granules_front, each = (total + a.grid - 1) / a.grid;
  if (tid == 0) *a.total = Total{total, each, !own_long};
  __syncthreads();
  for (int c = tid; c * each < total; c += PLAN_THREADS) {   // where each CTA starts: in the last line that has begun there
    const long long g = c * each;
    int lo = 0, hi = a.G - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (a.lines[mid].front <= g) lo = mid;
      else hi = mid - 1;
    }
    a.start[c] = Start{lo, 0, g - a.lines[lo].front};
  }
}

// ---- a CTA's way through its share ---------------------------------------------------------------------------------
struct Segment {
  int row, kvh, o;                     // as the line's
  int r0, rows;                        // rows r0 .. of the line's n * per_kv
  int t0, t1, keys;                    // tiles of keys; keys of the line
  bool two;                            // two tiles of rows, each over all keys; else two halves of the keys
  long long part;                      // where its results go
};
struct Walk {
  Line x;
  long long at, cur, end;
  int line, loaded;
  __device__ __forceinline__ void load(const Params& a) {
    const uint4* src = reinterpret_cast<const uint4*>(a.lines + line);
    uint4* dst = reinterpret_cast<uint4*>(&x);
#pragma unroll
    for (int i = 0; i < 4; ++i) dst[i] = __ldcg(src + i);
    loaded = line;
  }
  __device__ __forceinline__ bool begin(const Params& a) {
    const long long total = __ldcg(&a.total->all), each = __ldcg(&a.total->each);
    cur = blockIdx.x * each;
    end = min(cur + each, total);
    if (cur >= end) return false;
    const Start* s = a.start + blockIdx.x;
    line = __ldcg(&s->line);
    at = __ldcg(&s->at);
    loaded = -1;
    return true;
  }
  __device__ __forceinline__ bool next(const Params& a, Segment& s) {
    const int per_kv = a.n_heads / a.c.heads;
    while (cur < end) {
      if (loaded != line) load(a);
      const long long all = (long long)a.c.heads * x.tiles * x.per;
      if (at >= all) { ++line; at = 0; continue; }
      const int item = (int)(at / x.per), g0 = (int)(at % x.per), take = (int)min((long long)(x.per - g0), end - cur);
      at += take;
      cur += take;
      const int rows = x.n * per_kv;
      s.row = x.row; s.o = x.o; s.keys = x.keys;
      s.kvh = item / x.tiles;
      s.r0 = item % x.tiles * a.item_rows;
      s.rows = min(a.item_rows, rows - s.r0);
      s.two = s.rows > M_ROWS;
      const int kt = key_tiles(x.keys);
      s.t0 = min(tile_at(g0, x.weight), kt);
      s.t1 = min(tile_at(g0 + take, x.weight), kt);
      s.part = x.rows_front + (long long)s.kvh * rows + s.r0 + (long long)blockIdx.x * ITEM_ROWS;
      if (s.t0 < s.t1) return true;
    }
    return false;
  }
};

// ---- shared memory ---------------------------------------------------------------------------------------------
// Operands lie as the MMA reads them: 64 numbers of FP16 a row of 128 bytes, its 16-byte pieces exchanged by the row's last three bits, 8 rows a group of
// 1024 bytes; 128 wide, two such tiles behind each other.
template <int DIM, bool WIDE>
struct Layout {
  static constexpr int DP = DIM < 64 ? 64 : DIM;               // (32 wide: the upper half is zeros)
  static constexpr int TILE = KEYS * DP * 2;                   // FP16 keys or values of a tile; also 128 rows of queries
  static constexpr int RAW = KEYS * DIM;                       // their codes
  static constexpr int N_TILES = DIM == 128 ? 4 : 6, N_RAW = DIM == 128 ? 2 : 8;
  static constexpr int Q = 0, F16 = Q + 2 * TILE;              // queries: two tiles of rows, or (WIDE) two halves of their bits
  static constexpr int CODES = F16 + N_TILES * TILE;
  static constexpr int BYTES = CODES + N_RAW * RAW;
  // Tiles whose scales are kept.  When the codes of tile i are asked for, those of N_RAW / 2 tiles in front have been converted and the operands of N_TILES / 2 in
  // front of these have been read, so that at most N_RAW / 2 + N_TILES / 2 + 3 tiles are in use.
  static constexpr int N_INFO = DIM == 128 ? 8 : 16;
  static_assert(N_RAW / 2 + N_TILES / 2 + 3 <= N_INFO, "scales stay until they have been used");
};
struct alignas(16) Info { float ks[8], ve[8], lv[8]; int whole[4]; };                   // scales of the keys (negative: no such block), log2 of the values' (rounded up, and
                                                               // itself); whether all blocks are there, of each 64 keys

// What else lies in shared memory, behind the tiles.
// Segments that are told ahead.  The warp that asks for codes looks three tiles ahead and asks for a tile's values along with the next one's keys, so the segment whose
// place it waits for has to be the fifth in front, or none of its values would come.
constexpr int N_SEGMENTS = 8;
template <int DIM, bool WIDE>
struct Small {
  typedef Layout<DIM, WIDE> L;
  uint64_t raw_full[L::N_RAW], raw_empty[L::N_RAW], full[L::N_TILES], empty[L::N_TILES], s[2][2], p[2][2], o[2][2], drain, seg_full[N_SEGMENTS], seg_empty[N_SEGMENTS];
  uint64_t q[N_SEGMENTS];              // queries of the segment in that place.  (The place is not told again before both halves' products have waited for them: none gets two phases behind.)
  Info info[L::N_INFO];
  Segment segment[N_SEGMENTS];         // what the warp that asks for codes has come to, for all others; t1 = 0: that was all
  uint8_t exponent[2][M_ROWS];          // of the rows' largest numbers
  uint32_t tmem;
  int abort;
};
template <int DIM, bool WIDE>
__host__ __device__ constexpr int smem_bytes() { return Layout<DIM, WIDE>::BYTES + (int)sizeof(Small<DIM, WIDE>); }

// Warps: 8 for the softmax (two halves, either of 128 rows), 4 that turn codes into operands, one for each half that issues its products, one that asks for codes.
constexpr int SOFTMAX_WARPS = 8, CONVERT_WARPS = 4;
constexpr int W_CONVERT = SOFTMAX_WARPS, W_MMA = W_CONVERT + CONVERT_WARPS, W_LOAD = W_MMA + 2, THREADS = 32 * (W_LOAD + 1);

__device__ __forceinline__ void mbar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ void umma_f16_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) { tc::umma_bf16(d, a, b, idesc, accumulate); }
// A from tensor memory.
__device__ __forceinline__ void umma_f16_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
// FP16 A and B, FP32 sums; MN_B: B lies with its N side in rows (values: a key's dims next to each other).
__device__ __forceinline__ uint32_t idesc_f16(int m, int n, bool mn_b) {
  return (1u << 4) | (mn_b ? 1u << 16 : 0u) | (static_cast<uint32_t>(n >> 3) << 17) | (static_cast<uint32_t>(m >> 4) << 24);
}
// Values as the second product's B: rows of 64 dims, 8 keys a group; groups 1024 bytes apart (stride byte offset), the dims from 64 on a whole
// tile further (leading byte offset).
__device__ __forceinline__ uint64_t value_desc(uint32_t addr) {
  uint64_t d = 0;
  d |= static_cast<uint64_t>((addr >> 4) & 0x3FFF);
  d |= static_cast<uint64_t>((KEYS * 128) >> 4) << 16;
  d |= static_cast<uint64_t>(1024 >> 4) << 32;
  d |= static_cast<uint64_t>(1) << 46;
  d |= static_cast<uint64_t>(2) << 61;
  return d;
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_store8(uint32_t taddr, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]),
               "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}
__device__ __forceinline__ void tmem_load8(uint32_t taddr, uint32_t* r) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr));
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < 8; ++i) asm volatile("" : "+r"(r[i]));
}
__device__ __forceinline__ void before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void to_async_proxy() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// Order in which a CTA's tiles g = 0, 1, .. become operands: keys 0, keys 1, values 0, keys 2, values 1, .., so that scores are never waited for behind values whose
// room is still taken.  (What would follow the last values is left out.)
__host__ __device__ __forceinline__ int keys_fill(int g) { return g == 0 ? 0 : 2 * g - 1; }
__host__ __device__ __forceinline__ int values_fill(int g) { return 2 * g + 2; }

// A ring's place: which slot, and the parity of its phase.
struct Turn {
  int slot = 0;
  uint32_t phase = 0;
  __device__ __forceinline__ void step(int n) {
    if (++slot == n) { slot = 0; phase ^= 1u; }
  }
};

// A wait by a whole warp, bounded in time, once a first look has found nothing.  (Short, and out of line: with the polls unrolled the kernel had 140 KB of instructions instead
// of 92; its time was the same.)
__device__ __noinline__ bool wait_on(uint32_t bar, uint32_t parity, volatile int* abort, int* status) {
  const unsigned long long t0 = tc::global_ns();
  for (;;) {
#pragma unroll 1
    for (int i = 0; i < 64; ++i)
      if (__all_sync(0xffffffffu, tc::mbar_try_wait(bar, parity))) return true;
    if (__any_sync(0xffffffffu, *abort != 0)) return false;
    if (__any_sync(0xffffffffu, tc::global_ns() - t0 > tc::WAIT_BUDGET_NS)) break;
  }
  *abort = 1;
  latch_error(status, AD_ERR_TIMEOUT);
  return false;
}

// S = Q K^T, P = 2^(factor S - m), O = P V over the positions that a group shares, for all of its rows' queries: with per_kv heads on one key/value head, n tokens are n per_kv rows
// of the same matrices, so that 128 of them fill an MMA's rows where the attention row by row has 4 to 32.
// Codes are exact in FP16, and so are BF16 queries times a power of two (FP32 ones and their probabilities go in as two FP16 numbers: twice the products); a block's scale meets
// the scores behind the product, and the probabilities in front of the next one, rounded to 11 bits (22) as in the attention row by row, sums in FP32.  References m and d
// (of scores, and of probability times scale) are whole exponents: what changes when they move is exact.
// Scores lie in tensor memory, probabilities replace them there in half the columns and are the second product's A as they lie.  A CTA works on two halves, each 128 rows of its own (or, with no
// more than 128 rows, every other tile of keys for the same rows), in steps of 64 keys whose scores are issued two steps ahead, so that tensor cores and exponentials of the
// halves take turns.  Exponents are worked out against the references as they are, and again only where one of the warp's rows passes them.
// The CTAs take equal shares of all granules: an item's fixed part is what queries, results and the first tiles' latency cost (9600 cycles), a tile of 128 keys 3440 cycles with one tile
// of rows and 5700 with two.
// Bound by the softmax's latency: of a step's 2900 cycles with two tiles of rows its eight warps wait 290 for scores, look at them for 620 (loads from tensor memory among it),
// take 1000 for exponents and 930 for powers of two, store and hand over for 300, while products and powers of two of both halves need 1024 each.  Sixteen softmax warps, two
// a row, with references exchanged through shared memory, were slower (registers: 64 scores a thread are held at once); so was a branch of its own for keys that are not there.
// 109 rows of 3-8 queries behind 4 prefixes of 6000-16000, 32 heads on 8 of 128, INT8: 195 us, 104 GFLOP, 535 TFLOP/s of 1668 measured; 64 single queries behind 32000: 81 us, 418
// TFLOP/s.  (All of it by the attention row by row: 682 and 598 us with what follows.)
// grid = (CTAs that the plan is for), block = THREADS; dynamic shared memory: smem_bytes.
template <typename T, typename F, int DIM>
__global__ void __launch_bounds__(THREADS, 1)
shared_attention_kernel(const __grid_constant__ Params a) {
  constexpr bool WIDE = sizeof(T) == 4;
  typedef Layout<DIM, WIDE> L;
  constexpr int DP = L::DP, KSTEPS = DIM / 16;
  constexpr float SLACK = 2.f;
  extern __shared__ __align__(1024) unsigned char smem_p[];
  const int warp = tc::uniform_warp(), lane = threadIdx.x & 31, per_kv = a.n_heads / a.c.heads;
  const uint32_t smem = tc::smem_u32(smem_p);
  if (smem & 1023u) {                                          // (nothing else lies in shared memory that could move it)
    latch_error(a.status, AD_ERR_CUDA);
    return;
  }
  Small<DIM, WIDE>& sm = *reinterpret_cast<Small<DIM, WIDE>*>(smem_p + L::BYTES);
  auto bar = [](uint64_t& b) { return tc::smem_u32(&b); };
  if (threadIdx.x == 0) {
    for (int i = 0; i < L::N_RAW; ++i) { tc::mbar_init(bar(sm.raw_full[i]), 1); tc::mbar_init(bar(sm.raw_empty[i]), CONVERT_WARPS); }
    for (int i = 0; i < L::N_TILES; ++i) { tc::mbar_init(bar(sm.full[i]), CONVERT_WARPS); tc::mbar_init(bar(sm.empty[i]), 2); }
    for (int i = 0; i < 2; ++i) { tc::mbar_init(bar(sm.s[i][0]), 1); tc::mbar_init(bar(sm.s[i][1]), 1); tc::mbar_init(bar(sm.p[i][0]), 4); tc::mbar_init(bar(sm.p[i][1]), 4); tc::mbar_init(bar(sm.o[i][0]), 1); tc::mbar_init(bar(sm.o[i][1]), 1); }
    for (int i = 0; i < N_SEGMENTS; ++i) { tc::mbar_init(bar(sm.q[i]), SOFTMAX_WARPS); tc::mbar_init(bar(sm.seg_full[i]), 1); tc::mbar_init(bar(sm.seg_empty[i]), SOFTMAX_WARPS + CONVERT_WARPS + 2); }
    tc::mbar_init(bar(sm.drain), 2);
    sm.abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == W_MMA) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tc::smem_u32(&sm.tmem)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  if (DIM < 64)                                                // values' dims that there are none of
    for (int i = threadIdx.x; i < L::N_TILES * L::TILE / 16; i += THREADS) reinterpret_cast<uint4*>(smem_p + L::F16)[i] = make_uint4(0u, 0u, 0u, 0u);
  to_async_proxy();
  before_sync();
  __syncthreads();
  after_sync();
  pdl_launch();
  pdl_wait();
  const uint32_t tmem = __shfl_sync(0xffffffffu, sm.tmem, 0);
  auto col_s = [&](int t) { return tmem + t * 128; };          // scores, and over them probabilities
  auto col_o = [&](int t) { return tmem + 256 + t * DP; };
  auto aborted = [&]() { return *reinterpret_cast<volatile int*>(&sm.abort) != 0; };
  auto drain = [&](uint64_t& b, uint32_t parity) {             // waits whether or not somebody has given up
    int never = 0;
    wait_on(bar(b), parity, &never, a.status);
  };
  auto wait_warp = [&](uint64_t& b, uint32_t parity) {
    if (__all_sync(0xffffffffu, tc::mbar_try_wait(bar(b), parity))) return true;
    return wait_on(bar(b), parity, &sm.abort, a.status);
  };
  const bool work = Walk().begin(a);
  // Segments in their order, for the warps that read them.
  Turn seg;
  auto segment = [&]() -> const Segment* {                     // the next one; null: that was all, or a wait has run out
    if (!wait_warp(sm.seg_full[seg.slot], seg.phase)) return nullptr;
    const Segment* s = &sm.segment[seg.slot];
    return s->t1 == 0 ? nullptr : s;
  };
  auto done_with = [&](int slot) {
    __syncwarp();
    if (lane == 0) mbar_arrive(bar(sm.seg_empty[slot]));
  };

  if (work && warp == W_LOAD) {
    // ================= codes and scales: table -> scales -> copies, each a tile ahead of the next =================
    struct Tile { int row, kvh, pos, hi; bool there; };
    Walk walk;
    walk.begin(a);
    Segment s;
    int t = 0, told = 0;
    auto next_segment = [&]() {                                 // goes on, and tells the others
      const bool more = walk.next(a, s);
      if (!more) s.t0 = s.t1 = 0;
      if (told >= N_SEGMENTS) wait_warp(sm.seg_empty[seg.slot], seg.phase ^ 1u);
      if (lane == 0) {
        sm.segment[seg.slot] = s;
        mbar_arrive(bar(sm.seg_full[seg.slot]));
      }
      __syncwarp();
      seg.step(N_SEGMENTS);
      ++told;
      t = s.t0;
      return more;
    };
    bool more = next_segment();
    auto next_tile = [&]() {
      Tile x;
      x.there = more;
      if (!more) return x;
      x.row = s.row; x.kvh = s.kvh; x.pos = t * KEYS; x.hi = s.keys;
      if (++t == s.t1) more = next_segment();
      return x;
    };
    const int block = a.c.block, shift = __ffs(block) - 1, n_blocks = KEYS / block + 1;
    auto find = [&](const Tile& x) {                           // lane i: the tile's i-th block; -2: none
      const int i = (x.pos >> shift) + lane;
      if (!x.there || lane >= n_blocks || i << shift >= min(x.hi, x.pos + KEYS)) return -2;
      return a.c.find(x.row, i);
    };
    auto scales = [&](const Tile& x, int id, float& ks, float& vs) {      // lane j < 8: 16 keys each
      const int pos = x.pos + 16 * lane;
      const int mine = __shfl_sync(0xffffffffu, id, ((pos >> shift) - (x.pos >> shift)) & 31);
      ks = -1.f;
      vs = 1.f;
      if (x.there && lane < 8 && pos < x.hi && mine >= 0) {
        ks = __ldcg(a.c.scale[0] + (size_t)mine * a.c.heads + x.kvh);
        vs = __ldcg(a.c.scale[1] + (size_t)mine * a.c.heads + x.kvh);
      }
    };
    Tile x0 = {}, x1 = {};
    int id0 = -2, id1 = -2;
    float ks = -1.f, vs = 1.f;
    Turn raw;
    int g = 0, issued = 0;
    // what this lane copies of a tile: bytes, from where, to where in the tile; of all lanes
    uint32_t bytes = 0, to = 0, all = 0, bytes0 = 0, to0 = 0, all0 = 0;
    size_t src = 0, src0 = 0;
    bool ok = true;
    for (int round = 0; ok; ++round) {                           // (the first two rounds only fill the line)
      const Tile x2 = next_tile();
      const int id2 = find(x2);
      float ks1, vs1;
      scales(x1, id1, ks1, vs1);
      if (round >= 2) {
        if (id0 == -1) latch_error(a.status, AD_ERR_ARG);
        const int first = max(((x0.pos >> shift) + lane) << shift, x0.pos), last = min(min(((x0.pos >> shift) + lane + 1) << shift, x0.pos + KEYS), x0.hi);
        bytes = x0.there && id0 >= 0 && last > first ? (last - first) * DIM : 0;
        all = __reduce_add_sync(0xffffffffu, bytes);
        to = (first - x0.pos) * DIM;
        src = (((size_t)max(id0, 0) * a.c.heads + x0.kvh) * block + (first & (block - 1))) * DIM;
#pragma unroll 1
        for (int z = 0; z < 2; ++z) {
          if (z == 0 ? !x0.there : g == 0) continue;
          if (issued >= L::N_RAW) ok = wait_warp(sm.raw_empty[raw.slot], raw.phase ^ 1u);
          if (!ok) break;
          if (z == 0) {
            Info& info = sm.info[g & (L::N_INFO - 1)];
            if (lane < 8) {
              info.ks[lane] = ks;
              const float whole = kv::whole_lg2(vs);
              info.ve[lane] = whole;
              info.lv[lane] = kv::lg2(vs, whole);
            }
            const unsigned gone = __ballot_sync(0xffffffffu, ks < 0.f);
            if (lane < 2) info.whole[lane] = (gone >> (4 * lane) & 15u) == 0;
            __syncwarp();
          }
          const uint32_t full = bar(sm.raw_full[raw.slot]), n = z == 0 ? bytes : bytes0;
          if (lane == 0) tc::mbar_expect_tx(full, z == 0 ? all : all0);
          __syncwarp();
          if (n) bulk_load(smem + L::CODES + raw.slot * L::RAW + (z == 0 ? to : to0), a.c.codes[z] + (z == 0 ? src : src0), n, full);
          raw.step(L::N_RAW);
          ++issued;
        }
        if (!x0.there) break;
        bytes0 = bytes; to0 = to; all0 = all; src0 = src;
        ++g;
      }
      x0 = x1; x1 = x2; id0 = id1; id1 = id2; ks = ks1; vs = vs1;
    }
    for (int i = max(0, issued - L::N_RAW); i < issued; ++i)   // nothing is under way when the CTA ends, whoever gave up
      drain(sm.raw_full[i % L::N_RAW], (uint32_t)(i / L::N_RAW) & 1u);
  } else if (work && warp >= W_CONVERT && warp < W_MMA) {
    // ================= codes to FP16 =================
    constexpr int PIECES = DIM / 8, STEP = 32 * CONVERT_WARPS / PIECES, N = KEYS / STEP;      // pieces of a key; keys between a thread's pieces; its pieces
    const int ct = threadIdx.x - 32 * W_CONVERT, key0 = ct / PIECES, piece = ct % PIECES;
    const int src0 = key0 * DIM + piece * 8, dst0 = (piece >> 3) * KEYS * 128 + key0 * 128 + (((piece & 7) ^ (key0 & 7)) << 4);
    Turn raw;
    int g = 0, left0 = 0;                                       // keys of the tile in front, whose values come behind this one's keys
    bool ok = true, more = true;
    const Segment* s = segment();
    int t = s ? s->t0 : 0;
    for (; ok && more; ++g) {
      int left = 0;
      more = s != nullptr;
      if (more) {
        left = s->keys - t * KEYS;
        if (++t == s->t1) {
          done_with(seg.slot);
          seg.step(N_SEGMENTS);
          s = segment();
          t = s ? s->t0 : 0;
        }
      }
#pragma unroll 1
      for (int z = 0; z < 2; ++z) {                              // keys of tile g, values of the one in front
        if (z == 0 ? !more : g == 0) continue;
        const int fill = z == 0 ? keys_fill(g) : values_fill(g - 1), slot = fill % L::N_TILES, info = (z == 0 ? g : g - 1) & (L::N_INFO - 1);
        const int keys = z == 0 ? left : left0;
        {
          ok = wait_warp(sm.raw_full[raw.slot], raw.phase);
          if (ok && fill >= L::N_TILES) ok = wait_warp(sm.empty[slot], (uint32_t)(fill / L::N_TILES - 1) & 1u);
          if (!ok) break;
          const unsigned char* src = smem_p + L::CODES + raw.slot * L::RAW + src0;
          unsigned char* dst = smem_p + L::F16 + slot * L::TILE + dst0;
          const bool whole = keys >= KEYS && sm.info[info].whole[0] && sm.info[info].whole[1];
          constexpr int AT_ONCE = N < 8 ? N : 8;
#pragma unroll 1
          for (int i0 = 0; i0 < N; i0 += AT_ONCE) {
            uint2 w[AT_ONCE];
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) w[i] = *reinterpret_cast<const uint2*>(src + (i0 + i) * STEP * DIM);
            if (!whole) {
#pragma unroll
              for (int i = 0; i < AT_ONCE; ++i) {
                const int key = key0 + (i0 + i) * STEP;
                if (key >= keys || sm.info[info].ks[key >> 4] < 0.f) w[i] = make_uint2(0u, 0u);
              }
            }
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) {
              uint4 v;
              kv::codes_f16(F(), w[i].x, v.x, v.y);
              kv::codes_f16(F(), w[i].y, v.z, v.w);
              *reinterpret_cast<uint4*>(dst + (i0 + i) * STEP * 128) = v;
            }
          }
          to_async_proxy();
          __syncwarp();
          if (lane == 0) {
            mbar_arrive(bar(sm.raw_empty[raw.slot]));
            mbar_arrive(bar(sm.full[slot]));
          }
          raw.step(L::N_RAW);
        }
      }
      left0 = left;
    }
  } else if (work && warp < W_LOAD && warp >= W_MMA) {
    // ================= products of one half =================
    const int t = warp - W_MMA;
    const uint32_t idesc_s = idesc_f16(M_ROWS, SUB, false), idesc_o = idesc_f16(M_ROWS, DP, true);
    uint32_t p_phase = 0;
    int next_k = 0;                                            // the CTA's tiles in front of the segment
    bool ok = true;
    while (const Segment* s = ok ? segment() : nullptr) {
      const int n = __shfl_sync(0xffffffffu, s->t1 - s->t0, 0);      // (so that the compiler knows it to be the same in all lanes)
      const bool two = __shfl_sync(0xffffffffu, (int)s->two, 0) != 0;
      const int last_subs = __shfl_sync(0xffffffffu, s->keys > (s->t1 - 1) * KEYS + SUB ? 2 : 1, 0);      // steps of the last tile
      // (A half without steps waits as well: nothing else would keep it from falling behind.)
      ok = wait_warp(sm.q[seg.slot], seg.phase);
      done_with(seg.slot);
      seg.step(N_SEGMENTS);
      after_sync();
      // The half's tiles of keys: all of them for its rows (two), or every other one for the same rows; each in two steps of 64 keys, whose scores lie side by
      // side.  Scores two steps ahead; then, step by step, probabilities times values and the scores of two steps on: the softmax always finds some.
      const int stride = two ? 1 : 2, first = two ? 0 : t, steps = first < n ? 2 * ((n - 1 - first) / stride) + ((n - 1 - first) % stride == 0 ? last_subs : 2) : 0;
      for (int u = 0; u < steps + 2 && steps > 0 && ok; ++u) {
        const int sub = u & 1;
        if (u >= 2) {
          const int i = first + ((u - 2) >> 1) * stride, fill = values_fill(next_k + i), slot = fill % L::N_TILES;
          ok = wait_warp(sm.full[slot], (uint32_t)(fill / L::N_TILES) & 1u) && wait_warp(sm.p[t][sub], p_phase >> sub & 1u);
          p_phase ^= 1u << sub;
          if (!ok) break;
          after_sync();
          if (tc::elect_one()) {
            const uint32_t v = smem + L::F16 + slot * L::TILE + sub * (SUB / 16) * 2048;
#pragma unroll
            for (int j = 0; j < SUB / 16; ++j) {
#pragma unroll
              for (int h = WIDE ? 1 : 0; h >= 0; --h)
                umma_f16_ts(col_o(t), col_s(t) + SUB * sub + 16 * j + 8 * h, value_desc(v + j * 2048), idesc_o, (u > 2 || j > 0 || (WIDE && h == 0)) ? 1u : 0u);
            }
            tc::umma_commit(bar(sm.o[t][sub]));
            if (sub == 1 || u - 2 == steps - 1) {
              tc::umma_commit(bar(sm.empty[slot]));
              if (!two) tc::umma_commit(bar(sm.empty[slot]));      // (for the other half, which has no use for it)
            }
          }
          __syncwarp();
        }
        if (u < steps) {
          const int i = first + (u >> 1) * stride, fill = keys_fill(next_k + i), slot = fill % L::N_TILES;
          ok = wait_warp(sm.full[slot], (uint32_t)(fill / L::N_TILES) & 1u);
          if (!ok) break;
          after_sync();
          if (tc::elect_one()) {
            const uint32_t k = smem + L::F16 + slot * L::TILE + sub * SUB * 128;
#pragma unroll
            for (int h = WIDE ? 1 : 0; h >= 0; --h) {
              const uint32_t q = smem + L::Q + (WIDE ? h : two ? t : 0) * L::TILE;
#pragma unroll
              for (int j = 0; j < KSTEPS; ++j) {
                const uint32_t at = (j >> 2) * KEYS * 128 + (j & 3) * 32;
                umma_f16_ss(col_s(t) + SUB * sub, tc::make_smem_desc(q + at), tc::make_smem_desc(k + at), idesc_s, (j > 0 || (WIDE && h == 0)) ? 1u : 0u);
              }
            }
            tc::umma_commit(bar(sm.s[t][sub]));
            if (sub == 1 || u == steps - 1) {
              tc::umma_commit(bar(sm.empty[slot]));
              if (!two) tc::umma_commit(bar(sm.empty[slot]));
            }
          }
          __syncwarp();
        }
      }
      next_k += n;
    }
    // (what was issued is through before tensor memory is given back)
    if (tc::elect_one()) tc::umma_commit(bar(sm.drain));
    __syncwarp();
    if (t == 0) drain(sm.drain, 0);
  } else if (work && warp < SOFTMAX_WARPS) {
    // ================= probabilities, results =================
    const int half = warp >> 2, r = threadIdx.x & (M_ROWS - 1);
    const uint32_t quad = (uint32_t)(warp & 3) << 21;           // the warp's lanes of tensor memory
    uint32_t s_phase = 0, o_phase = 0;                          // a bit for either step of a tile
    int behind = 0;                                             // which of the two was the last one
    int info0 = 0, before = -1;                                 // the slot of the segment in front, whose results are stored late
    float m = -INFINITY, d = -INFINITY, l = 0.f, factor = 0.f, rest = 1.f;
    bool large = false;                                         // scores whose steps in FP32 are a quarter and more
    // queries of a segment: a thread a row, its power of two, FP16
    auto load_queries = [&](const Segment& x) {
      const int row = x.r0 + (x.two ? half * M_ROWS : 0) + r;
      if ((x.two || half == 0) && row < x.r0 + x.rows) {
        const T* q = static_cast<const T*>(a.q) + (size_t)(x.o + row / per_kv) * a.q_stride + ((size_t)x.kvh * per_kv + row % per_kv) * DIM;
        constexpr int PART = 32;                                // numbers at a time (twice through: the largest first)
        float top = 0.f;
#pragma unroll
        for (int i0 = 0; i0 < DIM; i0 += 8) {
          float y[8];
          kv::load8(q + i0, y);
#pragma unroll
          for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(y[i]));
        }
        const uint32_t e = min(max(__float_as_uint(top) >> 23, 27u), 253u);
        const float up = __uint_as_float((267u - e) << 23);      // 2^(13 - exponent)
#pragma unroll 1
        for (int i0 = 0; i0 < DIM; i0 += PART) {
#pragma unroll
          for (int i = 0; i < PART; i += 8) {
            float y[8];
            kv::load8(q + i0 + i, y);
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] *= up;
            uint32_t hi[4], lo[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              hi[j] = kv::pack_f16(y[2 * j], y[2 * j + 1]);
              if (WIDE) lo[j] = kv::rest_f16(y[2 * j], y[2 * j + 1], hi[j]);
            }
            const int c = (i0 + i) >> 3, at = (c >> 3) * KEYS * 128 + r * 128 + (((c & 7) ^ (r & 7)) << 4);
            unsigned char* dst = smem_p + L::Q + (!WIDE && x.two ? half * L::TILE : 0) + at;
            *reinterpret_cast<uint4*>(dst) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
            if (WIDE) *reinterpret_cast<uint4*>(dst + L::TILE) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
          }
        }
        sm.exponent[half][r] = (uint8_t)e;
      }
      to_async_proxy();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(sm.q[seg.slot]));
    };
    auto store = [&](const Segment& x) {                        // results of the segment that has come to its end
      const int row = x.two ? half * M_ROWS + r : r;
      const bool mine = row < x.rows, any = x.two || x.t1 - x.t0 > half;
      if (any) {
        if (!wait_warp(sm.o[half][behind], (o_phase >> behind & 1u) ^ 1u)) return;
        after_sync();
      }
      const long long at = x.part + row + (x.two ? 0 : half * a.part_rows);
      const bool some = any && l != 0.f;
      if (mine) a.ml[at] = make_float2(some ? m : -INFINITY, some ? l : 0.f);
      if (any) {
        // means, not sums, which FP32 may have no room for; factor after factor, as they may have none together
        const float share = some ? 1.f / l * kv::P_ONE : 0.f, unit = some ? kv::ex2(d) : 0.f;
#pragma unroll 1
        for (int c0 = 0; c0 < DIM; c0 += 16) {
          uint32_t y[16];
          tc::tmem_issue16(col_o(half) + c0 + quad, y);
          tmem_wait_ld();
          tc::tmem_landed16(y);
          if (mine && some) {
#pragma unroll
            for (int i = 0; i < 16; i += 4)
              *reinterpret_cast<float4*>(a.part + at * DIM + c0 + i) =
                  make_float4(__uint_as_float(y[i]) * share * unit, __uint_as_float(y[i + 1]) * share * unit, __uint_as_float(y[i + 2]) * share * unit,
                              __uint_as_float(y[i + 3]) * share * unit);
          }
        }
        before_sync();
      }
    };
    for (;;) {
      const Segment* next = segment();
      // Queries in front have been read: both halves have had their last scores.  All threads go on, or none.  A warp whose wait has run out goes through
      // the barriers like the others, with what it finds: every later wait of it ends at once.
      uint32_t over = !next || aborted();
      asm volatile(
          "{\n\t.reg .pred p, q;\n\t"
          "setp.ne.u32 p, %0, 0;\n\t"
          "barrier.cta.red.or.pred q, 1, %1, p;\n\t"
          "selp.u32 %0, 1, 0, q;\n\t}"
          : "+r"(over)
          : "n"(32 * SOFTMAX_WARPS)
          : "memory");
      if (over) break;
      const Segment& s = *next;
      load_queries(s);
      if (before >= 0) {
        store(sm.segment[before]);
        done_with(before);
      }
      before = seg.slot;
      seg.step(N_SEGMENTS);
      asm volatile("barrier.cta.sync 1, %0;" ::"n"(32 * SOFTMAX_WARPS) : "memory");
      const int n = s.t1 - s.t0, row = s.r0 + (s.two ? half * M_ROWS : 0) + r, last_row = s.r0 + s.rows - 1;
      const bool mine = row <= last_row, busy = __any_sync(0xffffffffu, mine);      // (rows that there are none of hold anything, and decide on nothing)
      {
        // scale / up: the part within 2^-120 .. 2^121 meets the keys' scale first, what is left of the powers of two their product
        const int power = (mine ? (int)sm.exponent[s.two ? half : 0][r] : 140) - 140, room = 247 - (int)(__float_as_uint(a.scale) >> 23),
                  first = min(max(power, room - 240), room);
        factor = ldexpf(a.scale, first);
        rest = ldexpf(1.f, power - first);
      }
      m = d = -INFINITY;
      l = 0.f;
      large = false;
      const int stride = s.two ? 1 : 2, base = s.t0 * KEYS;
      const int begin = (s.two ? 0 : half) * (KEYS / SUB);
      for (int u = begin, k = 0; u < n * (KEYS / SUB) && base + u * SUB < s.keys; ++k, u += u & 1 ? 1 + (stride - 1) * (KEYS / SUB) : 1) {      // steps of 64 keys
        const int sub = u & 1, pos = base + u * SUB;
        const uint32_t cols = col_s(half) + SUB * sub + quad;
        wait_warp(sm.s[half][sub], s_phase >> sub & 1u);
        s_phase ^= 1u << sub;
        after_sync();
        if (busy) {
          const Info& info = sm.info[(info0 + (u >> 1)) & (L::N_INFO - 1)];
          const float *ks = info.ks + 4 * sub, *ve = info.ve + 4 * sub, *lv = info.lv + 4 * sub;
          const float4 ks4 = *reinterpret_cast<const float4*>(ks), lv4 = *reinterpret_cast<const float4*>(lv);
          // Scores are changed where they lie, in short loops of their own, before they are looked at: one form of the rest for all tiles.
          if (pos + SUB > s.keys || !info.whole[sub]) {          // keys that are not there
            const int hi = s.keys - pos;
#pragma unroll 1
            for (int j = 0; j < 4; ++j) {
              uint32_t y[16];
              tc::tmem_issue16(cols + 16 * j, y);
              const bool gone = ks[j] < 0.f;
              tmem_wait_ld();
              tc::tmem_landed16(y);
#pragma unroll
              for (int c = 0; c < 16; ++c)
                if (gone || 16 * j + c >= hi) y[c] = 0xff800000u;
              tmem_store8(cols + 16 * j, y);
              tmem_store8(cols + 16 * j + 8, y + 8);
            }
            tmem_wait_st();
          }
          auto factor_of = [&](int j) {                          // (not 0 times -inf)
            return fmaxf(factor * fabsf(j == 0 ? ks4.x : j == 1 ? ks4.y : j == 2 ? ks4.z : ks4.w) * rest, FLT_MIN);
          };
          // Probabilities times their values' scale, as shares of 2^15 at the references m of the scores and d of the products.  With the references as they are, at
          // first, and if any row's turn out too large for FP16 or for the sum, again once these have moved.
          auto unit_of = [&](int j) {                            // exponent of what a probability of one becomes
            return (float)kv::P_BITS + fminf(fmaxf((j == 0 ? lv4.x : j == 1 ? lv4.y : j == 2 ? lv4.z : lv4.w) - d, -kv::SPAN), kv::SPAN);
          };
          // Exponents first, with the references as they are, or, where any row's probabilities would be too large for FP16 or for their sum, once these have moved.
          uint32_t y[4][16];                                     // the row's scores, then exponents
          for (bool as_they_are = k > 0 && !large;; as_they_are = false) {
#pragma unroll
            for (int j = 0; j < 4; ++j) tc::tmem_issue16(cols + 16 * j, y[j]);
            tmem_wait_ld();
#pragma unroll
            for (int j = 0; j < 4; ++j) tc::tmem_landed16(y[j]);
            if (!as_they_are) {
              // (References are whole numbers, so that what goes from one to another is an exact power of two.)
              bool again = false;
              for (float to = m == -INFINITY ? 0.f : m;;) {
                float most = -INFINITY, ve_max = -INFINITY, beyond = -INFINITY;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                  auto v = [&](int c) { return __uint_as_float(y[j][c]); };
                  float t0 = kv::max3(v(0), v(1), v(2));
#pragma unroll
                  for (int c = 3; c < 15; c += 2) t0 = kv::max3(t0, v(c), v(c + 1));
                  const float x = ceilf(fmaxf(t0, v(15)) * factor_of(j)), e = ve[j];
                  most = fmaxf(most, x);
                  ve_max = fmaxf(ve_max, e);
                  beyond = fmaxf(beyond, x - to + e);
                }
                const bool moves = mine && (most > m || beyond > d || ve_max - kv::SPAN > d);
                if (!again) {
                  if (!__any_sync(0xffffffffu, moves)) break;
                  // some row's do: how far p * scale goes beyond the new one, the same again
                  if (most > m) to = most + SLACK;
                  again = true;
                  continue;
                }
                float keep_o = 1.f;
                if (moves) {
                  const float top = most > m ? to : m, less = m - to;
                  const float tod = fmaxf(beyond > d + less ? beyond + SLACK : d + less, ve_max - kv::SPAN);
                  keep_o = tod == -INFINITY ? 0.f : kv::ex2(less + (d - tod));
                  m = top;
                  d = tod;
                  l *= kv::ex2(less);
                }
                if (k > 0) {                                    // (the half's first step has no results in front)
                  wait_warp(sm.o[half][behind], (o_phase >> behind & 1u) ^ 1u);      // (the products in front; those before them are, as these scores are)
                  after_sync();
#pragma unroll 1
                  for (int c0 = 0; c0 < DP; c0 += 8) {
                    uint32_t z[8];
                    tmem_load8(col_o(half) + c0 + quad, z);
#pragma unroll
                    for (int c = 0; c < 8; ++c) z[c] = __float_as_uint(__uint_as_float(z[c]) * keep_o);
                    tmem_store8(col_o(half) + c0 + quad, z);
                  }
                }
                break;
              }
              large = __any_sync(0xffffffffu, mine && fabsf(m) > 4194304.f && m != -INFINITY);
            }
            float ref = m == -INFINITY ? 0.f : m;
            if (large) {                                        // scores in steps of a quarter and more: a difference of rounded ones
#pragma unroll
              for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int c = 0; c < 16; ++c) y[j][c] = __float_as_uint(__fsub_rn(__fmul_rn(__uint_as_float(y[j][c]), factor_of(j)), ref));
              ref = 0.f;
            }
            bool fits = fmaxf(fmaxf(lv4.x, lv4.y), fmaxf(lv4.z, lv4.w)) - kv::SPAN <= d;
            const float most = m == -INFINITY ? -INFINITY : 15.9f;      // (2^16 is beyond FP16)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float e = unit_of(j), from = e - ref, t = large ? 1.f : factor_of(j);
              float top = -INFINITY;
#pragma unroll
              for (int c = 0; c < 16; c += 2) {
                const float2 v = kv::fma2(make_float2(__uint_as_float(y[j][c]), __uint_as_float(y[j][c + 1])), make_float2(t, t), make_float2(from, from));
                y[j][c] = __float_as_uint(v.x);
                y[j][c + 1] = __float_as_uint(v.y);
                top = kv::max3(top, v.x, v.y);
              }
              fits = fits && top <= fminf(most, e + 1.f);
            }
            if (!as_they_are || __all_sync(0xffffffffu, fits || !mine)) break;
          }
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            float2 sum;
            uint32_t hi[8], lo[8];
#pragma unroll
            for (int c = 0; c < 16; c += 2) {
              const float2 v = make_float2(kv::ex2(__uint_as_float(y[j][c])), kv::ex2(__uint_as_float(y[j][c + 1])));
              sum = c == 0 ? v : kv::add2(sum, v);
              hi[c / 2] = kv::pack_f16(v.x, v.y);
              if (WIDE) lo[c / 2] = kv::rest_f16(v.x, v.y, hi[c / 2]);
            }
            l = fmaf(sum.x + sum.y, kv::ex2(-unit_of(j)), l);
            tmem_store8(cols + 16 * j, hi);
            if (WIDE) tmem_store8(cols + 16 * j + 8, lo);
          }
          tmem_wait_st();
        }
        before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(sm.p[half][sub]));
        o_phase ^= 1u << sub;
        behind = sub;
      }
      info0 += n;
    }
    if (before >= 0 && !aborted()) store(sm.segment[before]);
  }
  before_sync();
  __syncthreads();
  after_sync();
  if (warp == W_MMA) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512));
}

// Joins the parts of every query: of its group's items, and of its row's own positions (one, or what several CTAs of the attention row by row left), with out = sum of mean_i s_i 2^(m_i - m) / sum of s_i 2^(m_i - m).  A warp a query and head.
// Bound by latency: lines, maxima, means, one after another; five means under way and four CTAs an SM: 600 queries of 32 heads with 3 to 7 parts each 29 us alone and cold, 64 with about 20
// 15 us.  (With the rows' own parts joined in front of it 25 and 13, and 14 and 6 for that.)  The parts' borders are worked out in 32 bits where they fit, as 64-bit divisions took a tenth of its time.
// grid = (enough for max_new * n_heads warps, B), block = JOIN_THREADS.
constexpr int JOIN_THREADS = 256;
template <typename T, int DIM>
__global__ void __launch_bounds__(JOIN_THREADS, 4)
shared_join_kernel(const __grid_constant__ Params a) {
  constexpr int PER = DIM / 32;
  pdl_launch();
  pdl_wait();
  const int lane = threadIdx.x & 31, b = blockIdx.y, per_kv = a.n_heads / a.c.heads;
  auto load_line = [&](int l) {
    Line x;
    const uint4* src = reinterpret_cast<const uint4*>(a.lines + l);
#pragma unroll
    for (int i = 0; i < 4; ++i) reinterpret_cast<uint4*>(&x)[i] = __ldcg(src + i);
    return x;
  };
  auto load = [&](const float* p, float* y) {
    p += lane * PER;
    if constexpr (PER == 4) { const float4 t = __ldcg(reinterpret_cast<const float4*>(p)); y[0] = t.x; y[1] = t.y; y[PER - 2] = t.z; y[PER - 1] = t.w; }
    else if constexpr (PER == 2) { const float2 t = __ldcg(reinterpret_cast<const float2*>(p)); y[0] = t.x; y[PER - 1] = t.y; }
    else y[0] = __ldcg(p);
  };
  const Line row = load_line(a.G + b);
  const int own_len = __ldcg(a.own_len + b), own_whole = __ldcg(&a.total->own_whole);
  if ((long long)blockIdx.x * (JOIN_THREADS / 32) + (threadIdx.x >> 5) >= (long long)row.n * a.n_heads) return;      // (below 2^30)
  const int w = blockIdx.x * (JOIN_THREADS / 32) + (threadIdx.x >> 5), i = w / a.n_heads, head = w - i * a.n_heads, kvh = head / per_kv;
  const Line grp = load_line(row.group);
  if (grp.n == 0) return;                                      // (a group that overlaps others, and that there was no room for: left out)
  // the row's own positions, by one CTA or several
  const size_t own = (size_t)(row.o + i) * a.n_heads + head;
  const int r_own = i * per_kv + head % per_kv, pieces = a.own.granule && !own_whole ? (own_units(a, own_len, row.n) + a.own.fixed + a.own.granule / 2) / a.own.granule : 1;
  int own0 = 0, slot0 = 0, own_parts = 1;
  if (pieces > 1) {
    const long long total = __ldcg(a.own.prefix + a.B), ctas = min((long long)a.own.grid, total);
    const long long first = __ldcg(a.own.prefix + b) + ((long long)kvh * ((row.n * per_kv + a.own.tile_rows - 1) / a.own.tile_rows) + r_own / a.own.tile_rows) * pieces;
    auto cta = [&](long long g) { return total * ctas >> 32 ? kv::cta_of(total, g, ctas) : (int)((unsigned)((g + 1) * ctas - 1) / (unsigned)total); };
    own0 = cta(first);
    own_parts = cta(first + pieces - 1) - own0 + 1;
    slot0 = 2 * own0 + (total * own0 < first * ctas ? 1 : 0);   // (its last segment, unless it starts there)
  }
  const long long each = __ldcg(&a.total->each);
  // part u, of its own or its group's: maximum and sum, and where its means are; all there are
  const int rows = grp.n * per_kv, r = (row.o - grp.o + i) * per_kv + head % per_kv, tile = r / a.item_rows, kt = key_tiles(grp.keys);
  const long long first = grp.front + ((long long)kvh * grp.tiles + tile) * grp.per, at = grp.rows_front + (long long)kvh * rows + r;
  const int halves = min(a.item_rows, rows - tile * a.item_rows) > M_ROWS ? 1 : 2;
  auto cta_of = [&](long long g) { return (int)((g | each) >> 32 ? g / each : (unsigned)g / (unsigned)each); };
  int c0 = 0, parts = own_parts;
  if (grp.tiles > 0) {
    c0 = cta_of(first);
    parts += (cta_of(first + grp.per - 1) - c0 + 1) * halves;
  }
  auto part = [&](int u, const float*& means) {
    if (u < own_parts) {
      const size_t slot = (size_t)(u == 0 ? slot0 : 2 * (own0 + u)) * a.own.tile_rows + r_own % a.own.tile_rows;
      means = own_parts == 1 ? a.own_part + own * DIM : a.own.part + slot * DIM;
      return __ldcg(own_parts == 1 ? a.own_ml + own : reinterpret_cast<const float2*>(a.own.part + 2 * (size_t)a.own.grid * a.own.tile_rows * DIM) + slot);
    }
    if (u >= parts) return make_float2(-INFINITY, 0.f);
    u -= own_parts;
    const int c = c0 + (halves == 2 ? u >> 1 : u);
    const long long where = at + (long long)c * ITEM_ROWS + (halves == 2 && (u & 1) ? a.part_rows : 0);
    means = a.part + where * DIM;
    const int g0 = (int)(max(c * each, first) - first), g1 = (int)(min((c + 1) * each, first + grp.per) - first);
    return min(tile_at(g0, grp.weight), kt) < min(tile_at(g1, grp.weight), kt) ? __ldcg(a.ml + where) : make_float2(-INFINITY, 0.f);
  };
  // the largest maximum and the sum against it; then means times their shares (sums of values may be more than FP32 has room for)
  float top = -INFINITY, sum = 0.f, x[PER];
  const float* means = a.part;
  float2 v = make_float2(-INFINITY, 0.f);
  for (int u0 = 0; u0 < parts; u0 += 32) {
    v = part(u0 + lane, means);
    float most = v.y != 0.f ? v.x : -INFINITY;
#pragma unroll
    for (int s = 16; s; s >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, s));
    most = fmaxf(top, most);
    float more = v.y == 0.f ? 0.f : v.x == most ? v.y : v.y * kv::ex2(v.x - most);
#pragma unroll
    for (int s = 16; s; s >>= 1) more += __shfl_xor_sync(0xffffffffu, more, s);
    sum = (top == most ? sum : sum * kv::ex2(top - most)) + more;
    top = most;
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  auto share = [&](float2 v) { return v.y == 0.f ? 0.f : (v.x == top ? v.y : v.y * kv::ex2(v.x - top)) * inv; };
#pragma unroll
  for (int j = 0; j < PER; ++j) x[j] = 0.f;
  for (int u0 = 0; u0 < parts; u0 += 32) {
    if (parts > 32) v = part(u0 + lane, means);
    const float f = share(v);
    for (unsigned left = __ballot_sync(0xffffffffu, v.y != 0.f); left;) {
      constexpr int AHEAD = 5;
      float y[AHEAD][PER], g[AHEAD];
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) {
        const int src = left ? __ffs(left) - 1 : 0;
        g[k] = left ? __shfl_sync(0xffffffffu, f, src) : 0.f;
        const float* from = reinterpret_cast<const float*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(means), src));
#pragma unroll
        for (int j = 0; j < PER; ++j) y[k][j] = 0.f;
        if (left) load(from, y[k]);
        left &= left - 1;
      }
#pragma unroll
      for (int k = 0; k < AHEAD; ++k)
#pragma unroll
        for (int j = 0; j < PER; ++j) x[j] = fmaf(y[k][j], g[k], x[j]);
    }
  }
  T* out = static_cast<T*>(a.out) + ((size_t)(row.o + i) * a.n_heads + head) * DIM + lane * PER;
#pragma unroll
  for (int j = 0; j < PER; ++j) out[j] = from_f32<T>(x[j]);
}

}  // namespace shr
}  // namespace ad
