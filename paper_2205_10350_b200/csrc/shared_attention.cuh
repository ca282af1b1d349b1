// Attention over the 8-bit key/value cache for rows that share prefixes: the shared positions once for all rows of a group, on the tensor cores' own memory.
#pragma once

#include "cache_attention.cuh"
#include "gemm_tc.cuh"

namespace ad {
namespace shr {

using kv::Cache;

constexpr int KEYS = 128;              // keys of a tile
constexpr int M_ROWS = 128;            // rows of an MMA
constexpr int ITEM_ROWS = 256;         // most rows of an item, and the distance of CTAs' parts in scratch

// What is worked on: first the groups' shared positions, then the rows' own ones.  A line has `heads` times `tiles` (of its rows) items, each over the keys
// lo .. of it; an item is `per` granules: FIXED ones, and `weight` for every tile of keys.  The CTAs share all granules evenly, in order.
struct Line {
  long long front, rows_front;         // granules and rows of results in front of it
  int o, n, lo, p;                     // tokens o .. o + n - 1; keys lo .. p + causal * (query + 1)
  int row, causal, tiles, per, weight, group, pad[2];
};
static_assert(sizeof(Line) == 64, "four 16-byte loads");
struct Start { int line, pad; long long at; };

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
  int grid, item_rows;                 // CTAs; rows of a group's item
  long long part_rows;                 // rows of results of one half
  // scratch
  long long* total;                    // granules of all lines
  Line* lines;                         // [G + B]
  Start* start;                        // [grid]
  float2* ml;                          // [2][part_rows] maxima and sums
  float* part;                         // [2][part_rows][dim] means of values
};

constexpr int FIXED = 4;
__host__ __device__ __forceinline__ int key_base(int lo) { return lo & ~15; }         // (scales change every 16 keys at most)
__host__ __device__ __forceinline__ int key_tiles(int lo, int hi) { return hi > lo ? (hi - key_base(lo) + KEYS - 1) / KEYS : 0; }
// The tile that granule x of an item starts with.
__host__ __device__ __forceinline__ int tile_at(int x, int weight) { return x <= FIXED ? 0 : (x - FIXED + weight - 1) / weight; }

// ---- plan ----------------------------------------------------------------------------------------------------------
constexpr int PLAN_THREADS = 1024;
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
// Tokens and shared positions of group g; false: it makes no sense, or holds nothing.
__device__ __forceinline__ bool group_of(const Params& a, int g, int& first, int& last, int& o, int& n, int& keys) {
  first = __ldcg(a.group + g);
  last = __ldcg(a.group + g + 1);
  keys = __ldcg(a.shared + g);
  if (first < 0 || last < first || last > a.B || keys < 0 || keys > a.c.table_stride * a.c.block) { latch_error(a.status, AD_ERR_ARG); return false; }
  if (first == last) return false;
  o = __ldcg(a.off + first);
  const long long d = (long long)__ldcg(a.off + last) - o;
  if (o < 0 || d < 0 || o + d > a.M) { latch_error(a.status, AD_ERR_ARG); return false; }
  n = (int)d;
  return n > 0;
}
// grid = 1, block = PLAN_THREADS.
__global__ void __launch_bounds__(PLAN_THREADS)
shared_plan_kernel(Params a) {
  __shared__ long long s_warp[PLAN_THREADS / 32];
  pdl_launch();
  pdl_wait();
  const int lines = a.G + a.B, per_kv = a.n_heads / a.c.heads, tid = threadIdx.x;
  long long granules_front = 0, tokens_front = 0, row_tokens_front = 0;
  for (int l0 = 0; l0 < lines; l0 += PLAN_THREADS) {
    const int l = l0 + tid;
    Line x = {};
    int hi = 0;
    bool some = false;
    if (l < a.G) {
      int first, last;
      some = group_of(a, l, first, last, x.o, x.n, x.p) && x.p > 0;
      x.row = first;
      hi = x.p;
    } else if (l < lines) {
      const int b = l - a.G;
      int lo = 0, hi_g = a.G - 1;                            // the last group that starts at b or in front of it
      while (lo < hi_g) {
        const int mid = (lo + hi_g + 1) >> 1;
        if (__ldcg(a.group + mid) <= b) lo = mid;
        else hi_g = mid - 1;
      }
      int first, last, go, gn;
      x.row = b;
      x.causal = a.causal;
      x.group = lo;
      if (kv::row_tokens(a.c, a.off, a.len, b, a.M, a.max_new, !a.causal, a.status, x.o, x.n, x.p)) {
        some = group_of(a, lo, first, last, go, gn, x.lo) && first <= b && b < last && x.lo <= x.p && x.o >= go && x.o + x.n <= go + gn;
        if (!some) latch_error(a.status, AD_ERR_ARG);
      }
      hi = x.causal ? x.p + x.n : x.p;
    }
    // no more results than there is room for, whatever the offsets
    long long all_g, all_r;
    const long long tf = tokens_front + block_scan(some && l < a.G ? x.n : 0, s_warp, all_g);
    const long long rf = row_tokens_front + block_scan(some && l >= a.G ? x.n : 0, s_warp, all_r);
    if (some && (l < a.G ? tf : rf) + x.n > a.M) {
      some = false;
      latch_error(a.status, AD_ERR_ARG);
    }
    const int item_rows = l < a.G ? a.item_rows : M_ROWS, rows = x.n * per_kv;
    x.rows_front = ((l < a.G ? tf : a.M + rf)) * a.n_heads;
    x.tiles = some ? (rows + item_rows - 1) / item_rows : 0;
    x.weight = l < a.G && item_rows > M_ROWS && rows > M_ROWS ? 2 : 1;
    const int kt = key_tiles(x.lo, hi);
    x.per = kt ? kt * x.weight + FIXED : 0;
    if (!some) x.n = 0;
    long long all;
    x.front = granules_front + block_scan((long long)a.c.heads * x.tiles * x.per, s_warp, all);
    if (l < lines) a.lines[l] = x;
    granules_front += all;
    tokens_front += all_g;
    row_tokens_front += all_r;
  }
  const long long total = granules_front, ctas = min((long long)a.grid, total);
  if (tid == 0) *a.total = total;
  for (int l = tid; l < lines; l += PLAN_THREADS) {
    const Line x = a.lines[l];                               // (written by this thread)
    const long long n = (long long)a.c.heads * x.tiles * x.per;
    if (n == 0) continue;
    long long c = kv::cta_of(total, x.front, ctas);
    if (kv::cta_start(total, c, ctas) < x.front) ++c;
    for (; c < ctas && kv::cta_start(total, c, ctas) < x.front + n; ++c) a.start[c] = Start{l, 0, kv::cta_start(total, c, ctas) - x.front};
  }
}

// ---- a CTA's way through its share ---------------------------------------------------------------------------------
struct Segment {
  int row, kvh, o, lo, p, causal;      // as the line's
  int r0, rows;                        // rows r0 .. of the line's n * per_kv
  int t0, t1, hi;                      // tiles of keys; end of the keys that any of the rows sees
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
    const long long total = __ldcg(a.total), ctas = min((long long)a.grid, total);
    if (blockIdx.x >= ctas) return false;
    cur = kv::cta_start(total, blockIdx.x, ctas);
    end = kv::cta_start(total, blockIdx.x + 1, ctas);
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
      const bool is_group = line < a.G;
      const int item_rows = is_group ? a.item_rows : M_ROWS, rows = x.n * per_kv;
      s.row = x.row; s.o = x.o; s.lo = x.lo; s.p = x.p; s.causal = x.causal;
      s.kvh = item / x.tiles;
      s.r0 = item % x.tiles * item_rows;
      s.rows = min(item_rows, rows - s.r0);
      s.two = s.rows > M_ROWS;
      s.hi = x.causal ? x.p + (s.r0 + s.rows - 1) / per_kv + 1 : x.p;
      const int kt = key_tiles(x.lo, s.hi);
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
  static constexpr int N_TILES = DIM == 128 ? 3 : 6, N_RAW = DIM == 128 ? 4 : 8;
  static constexpr int Q = 0, F16 = Q + 2 * TILE;              // queries: two tiles of rows, or (WIDE) two halves of their bits
  static constexpr int CODES = F16 + N_TILES * TILE;
  static constexpr int BYTES = CODES + N_RAW * RAW;
  // Tiles whose scales are kept.  When the codes of tile i are asked for, those of N_RAW / 2 tiles in front have been converted and the operands of N_TILES / 2 in
  // front of these have been read, so that at most N_RAW / 2 + N_TILES / 2 + 3 tiles are in use.
  static constexpr int N_INFO = DIM == 128 ? 8 : 16;
  static_assert(N_RAW / 2 + N_TILES / 2 + 3 <= N_INFO, "scales stay until they have been used");
};
struct Info { float ks[8], ve[8], lv[8]; };                   // scales of the keys (negative: no such block), log2 of the values' (rounded up, and itself)

// What else lies in shared memory, behind the tiles.
template <int DIM, bool WIDE>
struct Small {
  typedef Layout<DIM, WIDE> L;
  uint64_t raw_full[L::N_RAW], raw_empty[L::N_RAW], full[L::N_TILES], empty[L::N_TILES], s[2], p[2][2], o[2], q, seg, drain;
  Info info[L::N_INFO];
  Segment segment[2];                  // for the softmax's warps, whose registers are short; two: the one in front is stored late
  int exponent[M_ROWS];                // of the rows' largest numbers, where both halves of the keys want them
  uint32_t tmem;
  int abort;
};
template <int DIM, bool WIDE>
__host__ __device__ constexpr int smem_bytes() { return 1023 + Layout<DIM, WIDE>::BYTES + (int)sizeof(Small<DIM, WIDE>); }

constexpr int SOFTMAX_WARPS = 8, CONVERT_WARPS = 4;
constexpr int W_CONVERT = SOFTMAX_WARPS, W_MMA = W_CONVERT + CONVERT_WARPS, W_LOAD = W_MMA + 1, THREADS = 512;      // (four warpgroups, for the sake of their registers)
// Registers of a thread by warpgroup, from the 128 of the launch: 2 * 144 + 2 * 112 = 4 * 128.
constexpr int SOFTMAX_REGS = 144, OTHER_REGS = 112;

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
__device__ __forceinline__ void tmem_issue32(uint32_t taddr, uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),
        "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
        "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr));
}
// (orders every use of r behind the wait)
__device__ __forceinline__ void tmem_landed32(uint32_t (&r)[32]) {
#pragma unroll
  for (int i = 0; i < 32; ++i) asm volatile("" : "+r"(r[i]));
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_store8(uint32_t taddr, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]),
               "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}
__device__ __forceinline__ void before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void to_async_proxy() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// A ring's place: which slot, and the parity of its phase.
struct Turn {
  int slot = 0;
  uint32_t phase = 0;
  __device__ __forceinline__ void step(int n) {
    if (++slot == n) { slot = 0; phase ^= 1u; }
  }
};

// The rest of a wait by a whole warp whose first look found nothing.  (Out of line: the kernel's roles compete for the SM's instruction cache.)
__device__ __noinline__ bool wait_on(uint32_t bar, uint32_t parity, volatile int* abort, int* status) {
  if (__any_sync(0xffffffffu, *abort != 0) || !tc::mbar_wait_warp(bar, parity, status)) {
    *abort = 1;
    return false;
  }
  return true;
}

template <typename T, typename F, int DIM>
__global__ void __launch_bounds__(THREADS, 1)
shared_attention_kernel(const __grid_constant__ Params a) {
  constexpr bool WIDE = sizeof(T) == 4;
  typedef Layout<DIM, WIDE> L;
  constexpr int DP = L::DP, KSTEPS = DIM / 16;
  constexpr float SLACK = 2.f;
  extern __shared__ __align__(16) unsigned char smem_raw[];
  const int warp = tc::uniform_warp(), lane = threadIdx.x & 31, per_kv = a.n_heads / a.c.heads;
  const uint32_t smem = (tc::smem_u32(smem_raw) + 1023u) & ~1023u;
  unsigned char* smem_p = smem_raw + (smem - tc::smem_u32(smem_raw));
  Small<DIM, WIDE>& sm = *reinterpret_cast<Small<DIM, WIDE>*>(smem_p + L::BYTES);
  auto bar = [](uint64_t& b) { return tc::smem_u32(&b); };
  if (threadIdx.x == 0) {
    for (int i = 0; i < L::N_RAW; ++i) { tc::mbar_init(bar(sm.raw_full[i]), 1); tc::mbar_init(bar(sm.raw_empty[i]), CONVERT_WARPS); }
    for (int i = 0; i < L::N_TILES; ++i) { tc::mbar_init(bar(sm.full[i]), CONVERT_WARPS); tc::mbar_init(bar(sm.empty[i]), 1); }
    for (int i = 0; i < 2; ++i) { tc::mbar_init(bar(sm.s[i]), 1); tc::mbar_init(bar(sm.p[i][0]), 4); tc::mbar_init(bar(sm.p[i][1]), 4); tc::mbar_init(bar(sm.o[i]), 1); }
    tc::mbar_init(bar(sm.q), SOFTMAX_WARPS);
    tc::mbar_init(bar(sm.seg), 1);
    tc::mbar_init(bar(sm.drain), 1);
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
  auto wait_warp = [&](uint64_t& b, uint32_t parity) {
    if (__all_sync(0xffffffffu, tc::mbar_try_wait(bar(b), parity))) return true;
    return wait_on(bar(b), parity, &sm.abort, a.status);
  };
  Walk walk;
  const bool work = walk.begin(a);

  if (work) {
    if (warp < SOFTMAX_WARPS) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(SOFTMAX_REGS));
    else asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(OTHER_REGS));
  }
  if (work && warp == W_LOAD) {
    // ================= codes and scales: table -> scales -> copies, each a tile ahead of the next =================
    struct Tile { int row, kvh, pos, lo, hi; bool there; };
    Segment s;
    int t = 0;
    bool more = walk.next(a, s);
    if (more) t = s.t0;
    auto next_tile = [&]() {
      Tile x;
      x.there = more;
      if (!more) return x;
      x.row = s.row; x.kvh = s.kvh; x.pos = key_base(s.lo) + t * KEYS; x.lo = s.lo; x.hi = s.hi;
      if (++t == s.t1) {
        more = walk.next(a, s);
        if (more) t = s.t0;
      }
      return x;
    };
    const int block = a.c.block, n_blocks = KEYS / block + 1;
    auto find = [&](const Tile& x) {                           // lane i: the tile's i-th block; -2: none
      const int i = x.pos / block + lane;
      if (!x.there || lane >= n_blocks || i * block >= min(x.hi, x.pos + KEYS)) return -2;
      return a.c.find(x.row, i);
    };
    auto scales = [&](const Tile& x, int id, float& ks, float& vs) {      // lane j < 8: 16 keys each
      const int pos = x.pos + 16 * lane;
      const int mine = __shfl_sync(0xffffffffu, id, (pos / block - x.pos / block) & 31);
      ks = -1.f;
      vs = 1.f;
      if (x.there && lane < 8 && pos < x.hi && mine >= 0) {
        ks = __ldcg(a.c.scale[0] + (size_t)mine * a.c.heads + x.kvh);
        vs = __ldcg(a.c.scale[1] + (size_t)mine * a.c.heads + x.kvh);
      }
    };
    Tile x0 = next_tile(), x1 = next_tile();
    int id0 = find(x0), id1 = find(x1);
    float ks, vs;
    scales(x0, id0, ks, vs);
    Turn raw;
    int info = 0;
    bool ok = true;
    int issued = 0;
    while (x0.there && ok) {
      const Tile x2 = next_tile();
      const int id2 = find(x2);
      float ks1, vs1;
      scales(x1, id1, ks1, vs1);
      if (id0 == -1) latch_error(a.status, AD_ERR_ARG);
      // this lane's block: what of it falls into the tile
      const int first = max((x0.pos / block + lane) * block, x0.pos), last = min(min((x0.pos / block + lane + 1) * block, x0.pos + KEYS), x0.hi);
      const int bytes = id0 >= 0 && last > first ? (last - first) * DIM : 0;
      const int all = __reduce_add_sync(0xffffffffu, bytes);
      const size_t src = (((size_t)max(id0, 0) * a.c.heads + x0.kvh) * block + (first & (block - 1))) * DIM;
#pragma unroll
      for (int z = 0; z < 2; ++z) {
        if (issued >= L::N_RAW) ok = wait_warp(sm.raw_empty[raw.slot], raw.phase ^ 1u);
        if (!ok) break;
        if (z == 0) {
          if (lane < 8) {
            sm.info[info].ks[lane] = ks;
            const float whole = kv::whole_lg2(vs);
            sm.info[info].ve[lane] = whole;
            sm.info[info].lv[lane] = kv::lg2(vs, whole);
          }
          info = (info + 1) & (L::N_INFO - 1);
          __syncwarp();
        }
        const uint32_t full = bar(sm.raw_full[raw.slot]);
        if (lane == 0) tc::mbar_expect_tx(full, (uint32_t)all);
        __syncwarp();
        if (bytes) bulk_load(smem + L::CODES + raw.slot * L::RAW + (first - x0.pos) * DIM, a.c.codes[z] + src, (uint32_t)bytes, full);
        raw.step(L::N_RAW);
        ++issued;
      }
      x0 = x1; x1 = x2; id0 = id1; id1 = id2; ks = ks1; vs = vs1;
    }
    for (int i = max(0, issued - L::N_RAW); i < issued; ++i)   // nothing is under way when the CTA ends, whoever gave up
      tc::mbar_wait_warp(bar(sm.raw_full[i % L::N_RAW]), (uint32_t)(i / L::N_RAW) & 1u, a.status);
  } else if (work && warp >= W_CONVERT && warp < W_MMA) {
    // ================= codes to FP16 =================
    constexpr int PIECES = DIM / 8, STEP = 128 / PIECES, N = KEYS / STEP;      // pieces of a key; keys between a thread's pieces; its pieces
    const int ct = threadIdx.x - 32 * W_CONVERT, key0 = ct / PIECES, piece = ct % PIECES;
    const int src0 = key0 * DIM + piece * 8, dst0 = (piece >> 3) * KEYS * 128 + key0 * 128 + (((piece & 7) ^ (key0 & 7)) << 4);
    Segment s;
    Turn raw, f16;
    int info = 0, done = 0;
    bool ok = true;
    while (ok && walk.next(a, s)) {
      for (int t = s.t0; t < s.t1 && ok; ++t) {
        const int pos = key_base(s.lo) + t * KEYS;
#pragma unroll 1
        for (int z = 0; z < 2; ++z) {
          ok = wait_warp(sm.raw_full[raw.slot], raw.phase);
          if (ok && done >= L::N_TILES) ok = wait_warp(sm.empty[f16.slot], f16.phase ^ 1u);
          if (!ok) break;
          const unsigned char* src = smem_p + L::CODES + raw.slot * L::RAW + src0;
          unsigned char* dst = smem_p + L::F16 + f16.slot * L::TILE + dst0;
          bool whole = pos >= s.lo && pos + KEYS <= s.hi;
#pragma unroll
          for (int j = 0; j < 8; ++j) whole = whole && sm.info[info].ks[j] >= 0.f;
          constexpr int AT_ONCE = 4;
#pragma unroll 1
          for (int i0 = 0; i0 < N; i0 += AT_ONCE) {
            uint2 w[AT_ONCE];
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) w[i] = *reinterpret_cast<const uint2*>(src + (i0 + i) * STEP * DIM);
            if (!whole) {
#pragma unroll
              for (int i = 0; i < AT_ONCE; ++i) {
                const int key = key0 + (i0 + i) * STEP;
                if (pos + key < s.lo || pos + key >= s.hi || sm.info[info].ks[key >> 4] < 0.f) w[i] = make_uint2(0u, 0u);
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
            mbar_arrive(bar(sm.full[f16.slot]));
          }
          raw.step(L::N_RAW);
          f16.step(L::N_TILES);
          ++done;
        }
        info = (info + 1) & (L::N_INFO - 1);
      }
    }
  } else if (work && warp == W_MMA) {
    // ================= products =================
    const uint32_t idesc_s = idesc_f16(M_ROWS, KEYS, false), idesc_o = idesc_f16(M_ROWS, DP, true);
    Segment s;
    uint32_t q_phase = 0, p_phase[2] = {0, 0};
    int next_k = 0;                                            // fills of the ring in front of the segment: keys 2 i, values 2 i + 1
    bool ok = true;
    auto slot_of = [&](int fill) { return fill % L::N_TILES; };
    auto phase_of = [&](int fill) { return (uint32_t)(fill / L::N_TILES) & 1u; };
    // scores of tile `fill` / 2 for half t; last: the keys are not read again
    auto scores = [&](int t, int q_tile, int fill, bool last) {
      const int slot = slot_of(fill);
      if (!wait_warp(sm.full[slot], phase_of(fill))) return false;
      after_sync();
      if (tc::elect_one()) {
        const uint32_t k = smem + L::F16 + slot * L::TILE;
#pragma unroll
        for (int h = WIDE ? 1 : 0; h >= 0; --h) {
          const uint32_t q = smem + L::Q + (WIDE ? h : q_tile) * L::TILE;
#pragma unroll
          for (int j = 0; j < KSTEPS; ++j) {
            const uint32_t at = (j >> 2) * KEYS * 128 + (j & 3) * 32;
            umma_f16_ss(col_s(t), tc::make_smem_desc(q + at), tc::make_smem_desc(k + at), idesc_s, (j > 0 || (WIDE && h == 0)) ? 1u : 0u);
          }
        }
        tc::umma_commit(bar(sm.s[t]));
        if (last) tc::umma_commit(bar(sm.empty[slot]));
      }
      __syncwarp();
      return true;
    };
    auto values = [&](int t, int fill, bool first, bool last, bool end) {
      const int slot = slot_of(fill);
      if (!wait_warp(sm.full[slot], phase_of(fill))) return false;
      const uint32_t v = smem + L::F16 + slot * L::TILE;
#pragma unroll
      for (int part = 0; part < 2; ++part) {                   // (probabilities come in two halves)
        if (!wait_warp(sm.p[t][part], p_phase[t])) return false;
        after_sync();
        if (tc::elect_one()) {
#pragma unroll
          for (int j = part * KEYS / 32; j < (part + 1) * KEYS / 32; ++j) {
#pragma unroll
            for (int h = WIDE ? 1 : 0; h >= 0; --h)
              umma_f16_ts(col_o(t), col_s(t) + 16 * j + 8 * h, value_desc(v + j * 2048), idesc_o, (!first || j > 0 || (WIDE && h == 0)) ? 1u : 0u);
          }
          if (part == 1) {
            if (last) tc::umma_commit(bar(sm.empty[slot]));
            if (end) tc::umma_commit(bar(sm.o[t]));
          }
        }
        __syncwarp();
      }
      p_phase[t] ^= 1u;
      return true;
    };
    int turn = 0;
    auto publish = [&](bool more) {                            // (t1 = 0: that was all)
      if (lane == 0) {
        if (!more) s.t0 = s.t1 = 0;
        sm.segment[turn] = s;
        mbar_arrive(bar(sm.seg));
      }
      __syncwarp();
      turn ^= 1;
    };
    bool more = walk.next(a, s);
    publish(more);
    while (ok && more) {
      ok = wait_warp(sm.q, q_phase);
      q_phase ^= 1u;
      after_sync();
      const int n = __shfl_sync(0xffffffffu, s.t1 - s.t0, 0);      // (so that the compiler knows it to be the same in all lanes)
      const bool two = __shfl_sync(0xffffffffu, (int)s.two, 0) != 0;
      // The halves take turns: while one's scores become probabilities, the other's are multiplied.  Each is a tile of rows over all tiles of keys (two), or
      // every other tile of keys for the same rows.
      const int last = two ? 2 * n : n;
      for (int u = 0; u < last + 2 && ok; ++u) {
        const int t = u & 1;
        if (u >= 2) ok = values(t, next_k + 2 * (two ? (u - 2) >> 1 : u - 2) + 1, u < 4, !two || t == 1, u >= last);
        if (u < last && ok) ok = scores(t, two ? t : 0, next_k + 2 * (two ? u >> 1 : u), !two || t == 1);
      }
      next_k += 2 * n;
      more = walk.next(a, s);
      publish(more);
    }
    // (what was issued is through before tensor memory is given back)
    if (tc::elect_one()) tc::umma_commit(bar(sm.drain));
    __syncwarp();
    if (!tc::mbar_wait_warp(bar(sm.drain), 0, a.status)) sm.abort = 1;
  } else if (work && warp < SOFTMAX_WARPS) {
    // ================= probabilities, results =================
    const int half = warp >> 2, r = threadIdx.x & (M_ROWS - 1);
    const uint32_t quad = (uint32_t)(warp & 3) << 21;           // the warp's lanes of tensor memory
    uint32_t s_phase = 0, o_phase = 0, seg_phase = 0;
    int info0 = 0, turn = 0;
    float m = -INFINITY, d = -INFINITY, l = 0.f, factor = 0.f, rest = 1.f;
    bool ok = true, pending = false;
    // scale / up: the part within 2^-120 .. 2^121 meets the keys' scale first, what is left of the powers of two their product
    auto factors = [&](int e) {
      const int power = e - 140, room = 247 - (int)(__float_as_uint(a.scale) >> 23), first = min(max(power, room - 240), room);
      factor = ldexpf(a.scale, first);
      rest = ldexpf(1.f, power - first);
    };
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
        factors((int)e);
        if (!x.two) sm.exponent[r] = (int)e;
      }
      to_async_proxy();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(sm.q));
    };
    auto store = [&](const Segment& x) {                        // results of the segment that has come to its end
      const int row = x.two ? half * M_ROWS + r : r;
      const bool mine = row < x.rows, any = x.two || x.t1 - x.t0 > half;
      if (any) {
        if (!ok || !wait_warp(sm.o[half], o_phase)) { ok = false; return; }
        o_phase ^= 1u;
        after_sync();
      }
      const long long at = x.part + row + (x.two ? 0 : half * a.part_rows);
      const bool some = any && l != 0.f;
      if (mine) a.ml[at] = make_float2(some ? m : -INFINITY, some ? l : 0.f);
      if (any) {
        // means, not sums, which FP32 may have no room for; factor after factor, as they may have none together
        const float share = some ? 1.f / l * kv::P_ONE : 0.f, unit = some ? kv::ex2(d) : 0.f;
#pragma unroll 1
        for (int c0 = 0; c0 < DIM; c0 += 32) {
          uint32_t y[32];
          tmem_issue32(col_o(half) + c0 + quad, y);
          tmem_wait_ld();
          tmem_landed32(y);
          if (mine && some) {
#pragma unroll
            for (int i = 0; i < 32; i += 4)
              *reinterpret_cast<float4*>(a.part + at * DIM + c0 + i) =
                  make_float4(__uint_as_float(y[i]) * share * unit, __uint_as_float(y[i + 1]) * share * unit, __uint_as_float(y[i + 2]) * share * unit,
                              __uint_as_float(y[i + 3]) * share * unit);
          }
        }
        before_sync();
      }
    };
    for (;;) {
      // (one that has given up goes on to where it is not waited for any more: every wait of its ends at once)
      const bool there = wait_warp(sm.seg, seg_phase);
      seg_phase ^= 1u;
      ok = ok && there;
      const Segment& s = sm.segment[turn];
      turn ^= 1;
      // Queries in front have been read: both halves have had their last scores.  All threads go on, or none.
      uint32_t over = !ok || aborted() || s.t0 == s.t1;
      asm volatile(
          "{\n\t.reg .pred p, q;\n\t"
          "setp.ne.u32 p, %0, 0;\n\t"
          "barrier.cta.red.or.pred q, 1, 256, p;\n\t"
          "selp.u32 %0, 1, 0, q;\n\t}"
          : "+r"(over)
          :
          : "memory");
      if (over) break;
      load_queries(s);
      if (pending) store(sm.segment[turn]);
      asm volatile("barrier.cta.sync 1, 256;" ::: "memory");
      if (!s.two && half == 1 && r < s.rows) factors(sm.exponent[r]);
      m = d = -INFINITY;
      l = 0.f;
      const int n = s.t1 - s.t0, row = s.r0 + (s.two ? half * M_ROWS : 0) + r, last_row = s.r0 + s.rows - 1;
      const int sees = s.causal ? s.p + min(row, last_row) / per_kv + 1 : s.p;
      const bool mine = row <= last_row, busy = __any_sync(0xffffffffu, mine);      // (rows that there are none of hold anything, and decide on nothing)
      for (int i = s.two ? 0 : half; i < n && ok; i += s.two ? 1 : 2) {
        ok = wait_warp(sm.s[half], s_phase);
        if (!ok) break;
        s_phase ^= 1u;
        after_sync();
        auto hand_over = [&](int part) {
          tmem_wait_st();
          before_sync();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(sm.p[half][part]));
        };
        if (busy) {
          const Info& info = sm.info[(info0 + i) & (L::N_INFO - 1)];
          const int pos = key_base(s.lo) + (s.t0 + i) * KEYS;
          bool whole = pos >= s.lo && pos + KEYS <= sees;
#pragma unroll
          for (int j = 0; j < 8; ++j) whole = whole && info.ks[j] >= 0.f;
          // Scores are changed where they lie, in short loops of their own, before they are looked at: one form of the rest for all tiles, as instructions that are
          // not in the SM's cache cost more than any of these loops.
          if (!__all_sync(0xffffffffu, whole)) {                // keys that are not there, or not seen by some row of the warp
            const int lo = s.lo - pos, hi = sees - pos;
#pragma unroll 1
            for (int j = 0; j < 8; ++j) {
              uint32_t y[16];
              tc::tmem_issue16(col_s(half) + 16 * j + quad, y);
              const bool gone = info.ks[j] < 0.f;
              tmem_wait_ld();
              tc::tmem_landed16(y);
#pragma unroll
              for (int c = 0; c < 16; ++c)
                if (gone || 16 * j + c < lo || 16 * j + c >= hi) y[c] = 0xff800000u;
              tmem_store8(col_s(half) + 16 * j + quad, y);
              tmem_store8(col_s(half) + 16 * j + 8 + quad, y + 8);
            }
            tmem_wait_st();
          }
          // ---- the largest score of every 16 keys: do references move? ----
          auto factor_of = [&](int j) { return fmaxf(factor * fabsf(info.ks[j]) * rest, FLT_MIN); };      // (not 0 times -inf)
          // (references are whole numbers, so that what goes from one to another is an exact power of two)
          float keep_o = 1.f;
          bool moved = false;
          for (float to = m == -INFINITY ? 0.f : m;;) {
            float most = -INFINITY, ve_max = -INFINITY, beyond = -INFINITY;
            uint32_t y[2][16];
            tc::tmem_issue16(col_s(half) + quad, y[0]);
#pragma unroll 1
            for (int g = 0; g < 4; ++g) {
#pragma unroll
              for (int k = 0; k < 2; ++k) {
                tmem_wait_ld();
                tc::tmem_landed16(y[k]);
                if (k == 0 || g < 3) tc::tmem_issue16(col_s(half) + 32 * g + 16 * (k + 1) + quad, y[k ^ 1]);
                auto v = [&](int c) { return __uint_as_float(y[k][c]); };
                float t0 = kv::max3(v(0), v(1), v(2)), t1 = kv::max3(v(3), v(4), v(5));
                t0 = kv::max3(t0, v(6), v(7)); t1 = kv::max3(t1, v(8), v(9));
                t0 = kv::max3(t0, v(10), v(11)); t1 = kv::max3(t1, v(12), v(13));
                t0 = kv::max3(t0, v(14), v(15));
                const float x = ceilf(fmaxf(t0, t1) * factor_of(2 * g + k)), ve = info.ve[2 * g + k];
                most = fmaxf(most, x);
                ve_max = fmaxf(ve_max, ve);
                beyond = fmaxf(beyond, x - to + ve);
              }
            }
            if (!moved) {
              moved = mine && (most > m || beyond > d || ve_max - kv::SPAN > d);
              if (!__any_sync(0xffffffffu, moved)) break;
              if (moved && most > m) to = most + SLACK;         // ... and how far p * scale goes beyond that: the same again
              moved = true;
              continue;
            }
            // reference m of the row's scores, and exponent d of p * scale beyond m's own
            if (mine && (most > m || beyond > d || ve_max - kv::SPAN > d)) {
              const float top = most > m ? to : m, less = m - to;
              const float tod = fmaxf(beyond > d + less ? beyond + SLACK : d + less, ve_max - kv::SPAN);
              keep_o = tod == -INFINITY ? 0.f : kv::ex2(less + (d - tod));
              m = top;
              d = tod;
              l *= kv::ex2(less);
            }
            if (i > (s.two ? 0 : 1)) {                          // (the half's first tile has no results in front)
#pragma unroll 1
              for (int c0 = 0; c0 < DP; c0 += 16) {
                uint32_t y[16];
                tc::tmem_issue16(col_o(half) + c0 + quad, y);
                tmem_wait_ld();
                tc::tmem_landed16(y);
#pragma unroll
                for (int c = 0; c < 16; ++c) y[c] = __float_as_uint(__uint_as_float(y[c]) * keep_o);
                tmem_store8(col_o(half) + c0 + quad, y);
                tmem_store8(col_o(half) + c0 + 8 + quad, y + 8);
              }
            }
            break;
          }
          float ref = m == -INFINITY ? 0.f : m;
          const bool large = __any_sync(0xffffffffu, mine && fabsf(ref) > 4194304.f);
          if (large) {                                          // scores in steps of a quarter and more: a difference of rounded ones
#pragma unroll 1
            for (int j = 0; j < 8; ++j) {
              uint32_t y[16];
              tc::tmem_issue16(col_s(half) + 16 * j + quad, y);
              const float t = factor_of(j);
              tmem_wait_ld();
              tc::tmem_landed16(y);
#pragma unroll
              for (int c = 0; c < 16; ++c) y[c] = __float_as_uint(__fsub_rn(__fmul_rn(__uint_as_float(y[c]), t), ref));
              tmem_store8(col_s(half) + 16 * j + quad, y);
              tmem_store8(col_s(half) + 16 * j + 8 + quad, y + 8);
            }
            tmem_wait_st();
            ref = 0.f;
          }
          // ---- probabilities times their values' scale, as shares of 2^15 at the references ----
          uint32_t y[2][16];
          tc::tmem_issue16(col_s(half) + quad, y[0]);
#pragma unroll 1
          for (int g = 0; g < 4; ++g) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              const float e = (float)kv::P_BITS + fminf(fmaxf(info.lv[2 * g + k] - d, -kv::SPAN), kv::SPAN), from = e - ref, t = large ? 1.f : factor_of(2 * g + k);
              tmem_wait_ld();
              tc::tmem_landed16(y[k]);
              if (k == 0 || g < 3) tc::tmem_issue16(col_s(half) + 32 * g + 16 * (k + 1) + quad, y[k ^ 1]);
              float2 sum;
              uint32_t hi[8], lo[8];
#pragma unroll
              for (int c = 0; c < 16; c += 2) {
                float2 v = make_float2(__uint_as_float(y[k][c]), __uint_as_float(y[k][c + 1]));
                v = kv::fma2(v, make_float2(t, t), make_float2(from, from));
                v.x = kv::ex2(v.x);
                v.y = kv::ex2(v.y);
                sum = c == 0 ? v : kv::add2(sum, v);
                hi[c / 2] = kv::pack_f16(v.x, v.y);
                if (WIDE) lo[c / 2] = kv::rest_f16(v.x, v.y, hi[c / 2]);
              }
              l = fmaf(sum.x + sum.y, kv::ex2(-e), l);
              tmem_store8(col_s(half) + 32 * g + 16 * k + quad, hi);
              if (WIDE) tmem_store8(col_s(half) + 32 * g + 16 * k + 8 + quad, lo);
            }
            if (g == 1) hand_over(0);                            // (the second product begins with the first half)
          }
        } else {
          hand_over(0);
        }
        hand_over(1);
      }
      info0 += n;
      pending = true;
    }
    if (pending && ok && !aborted()) store(sm.segment[turn]);
  }
  before_sync();
  __syncthreads();
  after_sync();
  if (warp == W_MMA) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512));
}

// Joins the parts of every query: of its group's items and of its row's.  A warp a query and head.
// grid = (enough for max_new * n_heads warps, B), block = JOIN_THREADS.
constexpr int JOIN_THREADS = 256;
template <typename T, int DIM>
__global__ void __launch_bounds__(JOIN_THREADS)
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
  const Line row = load_line(a.G + b);
  const long long w = (long long)blockIdx.x * (JOIN_THREADS / 32) + (threadIdx.x >> 5);
  if (w >= (long long)row.n * a.n_heads) return;
  const Line grp = load_line(row.group);
  const long long total = __ldcg(a.total), ctas = min((long long)a.grid, total);
  const int i = (int)(w / a.n_heads), head = (int)(w % a.n_heads), kvh = head / per_kv;
  float top = -INFINITY, sum = 0.f, x[PER];
#pragma unroll
  for (int j = 0; j < PER; ++j) x[j] = 0.f;
  auto add = [&](const Line& ln, bool is_group) {
    if (ln.per == 0 || ln.tiles == 0) return;
    const int item_rows = is_group ? a.item_rows : M_ROWS, rows = ln.n * per_kv, r = (row.o - ln.o + i) * per_kv + head % per_kv, tile = r / item_rows;
    const int n_rows = min(item_rows, rows - tile * item_rows), last = tile * item_rows + n_rows - 1;
    const int hi = ln.causal ? ln.p + last / per_kv + 1 : ln.p, kt = key_tiles(ln.lo, hi);
    const long long first = ln.front + ((long long)kvh * ln.tiles + tile) * ln.per;
    const int c0 = kv::cta_of(total, first, ctas), c1 = kv::cta_of(total, first + ln.per - 1, ctas), halves = n_rows > M_ROWS ? 1 : 2;
    const long long at = ln.rows_front + (long long)kvh * rows + r;
    // lane u: part u (32 at a time)
    for (int u0 = 0; u0 < (c1 - c0 + 1) * halves; u0 += 32) {
      const int u = u0 + lane, c = c0 + u / halves;
      float2 v = make_float2(-INFINITY, 0.f);
      long long where = 0;
      if (c <= c1) {
        const int g0 = (int)(max(kv::cta_start(total, c, ctas), first) - first), g1 = (int)(min(kv::cta_start(total, c + 1, ctas), first + ln.per) - first);
        where = at + (long long)c * ITEM_ROWS + (u % halves) * a.part_rows;
        if (min(tile_at(g0, ln.weight), kt) < min(tile_at(g1, ln.weight), kt)) v = __ldcg(a.ml + where);
      }
      const unsigned some = __ballot_sync(0xffffffffu, v.y != 0.f);
      float most = v.y != 0.f ? v.x : -INFINITY;
#pragma unroll
      for (int s = 16; s; s >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, s));
      const float to = fmaxf(top, most), back = top == to ? 1.f : kv::ex2(top - to);
      sum *= back;
#pragma unroll
      for (int j = 0; j < PER; ++j) x[j] *= back;
      top = to;
      const float f = v.y == 0.f ? 0.f : v.x == top ? v.y : v.y * kv::ex2(v.x - top);
      for (unsigned left = some; left;) {
        constexpr int AHEAD = 4;
        float y[AHEAD][PER], g[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
          const int src = left ? __ffs(left) - 1 : 0;
          g[k] = __shfl_sync(0xffffffffu, f, src);
          const long long from = __shfl_sync(0xffffffffu, where, src);
          if (!left) g[k] = 0.f;
#pragma unroll
          for (int j = 0; j < PER; ++j) y[k][j] = 0.f;
          if (left) {
            const float* p = a.part + from * DIM + lane * PER;
            if constexpr (PER == 4) { const float4 t = __ldcg(reinterpret_cast<const float4*>(p)); y[k][0] = t.x; y[k][1] = t.y; y[k][PER - 2] = t.z; y[k][PER - 1] = t.w; }
            else if constexpr (PER == 2) { const float2 t = __ldcg(reinterpret_cast<const float2*>(p)); y[k][0] = t.x; y[k][PER - 1] = t.y; }
            else y[k][0] = __ldcg(p);
          }
          left &= left - 1;
        }
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
          sum += g[k];
#pragma unroll
          for (int j = 0; j < PER; ++j) x[j] = fmaf(y[k][j], g[k], x[j]);
        }
      }
    }
  };
  add(grp, true);
  add(row, false);
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  T* out = static_cast<T*>(a.out) + ((size_t)(row.o + i) * a.n_heads + head) * DIM + lane * PER;
#pragma unroll
  for (int j = 0; j < PER; ++j) out[j] = from_f32<T>(x[j] * inv);
}

}  // namespace shr
}  // namespace ad
