// tree_wide.cuh -- tree attention for many query rows of a KV head: tcgen05
// products on tiles of 128 rows.
//
// With R rows per KV head a byte of the cache takes R flops or more: beyond 16 rows more
// than tiles of 16 keep up with.  A block takes 128 rows, one KV head and one
// item of pages, a page of 64 tokens a step:
//
//   S = Q K^T    [128 rows][64 tokens] in tensor memory; Q and K from shared memory
//   P = 2^(S' - m), by four warps, one thread per row: a row is a lane of
//       tensor memory, so its maximum and sum never leave the thread
//   O += P V     P in tensor memory, over S's place; V^T pages from shared memory
//
// Four more warps fetch K and V^T by TMA (both lie in the cache as K-major operands)
// and issue the S and the O products: to issue a copy takes a thread 300 to 400
// cycles, a product about 110, so that one thread for all of them would bound the block
// (1580 cycles a page at head dim 64, for which the softmax takes 1250).  S has three places (two
// at head dim 128), so that the products of the next pages run during the
// softmax of this one.  The softmax warps take over registers of the other four: at
// 128 to a thread they would spill.
//
// With a split that the caller gives, a block takes one item.  With an open one the
// blocks share all pages of all trees evenly, in the order of tree, head, tile and
// page: a block's share is a few segments, each of one tile, and those that are not
// a whole tile's pages leave their part to the joining kernel.  So no block waits for a
// longer one, and what a row's table could hold does not matter.  The tiles of one head
// read the same pages: they go to as many neighbouring blocks (a team), which share the
// pages as one block would, and so read them at the same time, from L2.  (As clusters that
// multicast each page the teams were slower, one document of 65,001 tokens and 264 rows
// 97 us: fewer blocks fit, and each waits for the others at every page.)
//
// m is a score as it comes from the product (see weights_of), and moves only when a row's maximum
// rises by more than 8 in the exponent (O is rescaled then; the result does not depend on m but for
// rounding).  In fp16 its own weight is 2^7, so P is at most 2^15, whatever the scores' size,
// and a weight of 2^-21 of the largest has all its bits, one of 2^-31 some.  P is rounded to the
// cache's type for the product (2^-11 in fp16, 2^-8 in bf16, as the output is; the tensor cores
// take no wider operand at their full rate), the sum takes it unrounded, in fp32.
//
// Pages that hold masked tokens clear, in shared memory, the values that no row
// sees.  Values that some rows see and that are not finite are taken out and added to
// those rows' O by hand.
//
// Measured: fp16, 16 / 8 heads of 64, 32 trees of 17 nodes over 1024 to 6144 tokens 56.5 us (a
// floor of 35 by the cache's bytes); bf16, 32 / 4 heads of 128, one tree over 65,001 tokens 40
// us with 4 nodes (32 rows), 43 with 16, 57 with 33, 71 with 64 (floors of 20, and of 36 by the
// products for the last).  With 16 nodes the pages come in at 90 per cent of the memory's rate,
// for 22 of the 43 us; the rest is a block's start, its end and the joining.  With 17 (the 32
// trees) the softmax warps' chain bounds a page, 1250 cycles: wait 180, scores 100, maximum 220,
// powers 430, P passed on 100, the way round 190 (stamped before the maxima were kept unscaled, which
// changed no time by more than 0.5 per cent); a block's start takes 5300, a change of segment
// 5500.  What shortened the chain was less code (waits written out in a few instructions, 61 to
// 57 us; the next segment found during the last one, 55; waiting for the last arrivals added
// one), not fewer powers: two or four threads to a row where the tile's rows leave room took 1
// us off, and added 2 at head dim 128.
#pragma once
#include "internal.h"
#include "tree_common.cuh"

namespace gs {
namespace {

constexpr int kWideRows = 128;                       // query rows of a block
constexpr int kSoftWarps = 4, kSoftThreads = 128;
constexpr int kFetchKWarp = kSoftWarps, kFetchVWarp = kSoftWarps + 1, kScoreWarp = kSoftWarps + 2,
              kValueWarp = kSoftWarps + 3;
constexpr int kWideThreads = 256;
// Registers of a softmax thread and of the others: what 256 threads of 128 have.
constexpr int kSoftRegs = 184, kWorkRegs = 72;
static_assert(kSoftThreads * kSoftRegs + (kWideThreads - kSoftThreads) * kWorkRegs == kWideThreads * 128);
constexpr int kTmemCols = 256;                       // the places of S (and P), and O
constexpr int kMostShared = 1024;                    // trees whose pages are shared evenly
constexpr int kFewPages = 4;                         // the least share of a block
constexpr float kRise = 8.f;                         // log2 units
template <bool BF16>
constexpr float kSet = BF16 ? 0.f : 7.f;             // the weight of the score that m was set to

template <int D>
struct WideSmem {
  static constexpr int H = D / 64;                   // 64-dim halves
  static constexpr int stages = D == 64 ? 4 : 2;     // pages in flight
  static constexpr int places = D == 64 ? 3 : 2;     // of S, 64 columns each; O behind them
  static constexpr int o_col = 64 * places;
  static constexpr int q_bytes = H * kWideRows * 128;
  static constexpr int page_bytes = D * 128;         // K: [half][64 tokens][64 dims]; V^T: [dims][64 tokens]
  static constexpr int k_at = q_bytes, v_at = k_at + stages * page_bytes;
  static constexpr int bars_at = v_at + stages * page_bytes;
  static constexpr int total = bars_at + 256 + 1024;    // (1024: the start is aligned by hand)
};

// Byte offset of 16-byte chunk `chunk` of row `row` in a tile with 128-byte swizzle.
__device__ __forceinline__ uint32_t swizzled(int row, int chunk) {
  return static_cast<uint32_t>(row * 128 + ((chunk ^ (row & 7)) << 4));
}

__device__ __forceinline__ float max3(float x, float y, float z) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(x), "f"(y), "f"(z));
  return r;
}

// 32 lanes x 16 columns, with the wait.
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
        "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]),
        "=r"(r[14]), "=r"(r[15])
      : "r"(taddr));
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
      "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}

// D += A B with A (two 16-bit values per column) in tensor memory.
__device__ __forceinline__ void umma_f16_ta(uint32_t tmem_d, uint32_t tmem_a, uint64_t bdesc,
                                            uint32_t idesc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.eq.u32 p, %3, %3;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(tmem_d),
      "r"(tmem_a), "l"(bdesc), "r"(idesc)
      : "memory");
}

template <bool BF16>
constexpr uint32_t wide_idesc(int N) {   // both operands bf16: format 1 at bits 7 and 10
  return umma_idesc_f16(kWideRows, N) | (BF16 ? (1u << 7) | (1u << 10) : 0u);
}

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* m, int x, int y, int z,
                                            uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(m)), "r"(x), "r"(y), "r"(z), "r"(bar)
      : "memory");
}
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* m, int x, int y, int z,
                                            int w, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(m)), "r"(x), "r"(y), "r"(z), "r"(w), "r"(bar)
      : "memory");
}

// A row of shared memory to global memory, with the wait.
__device__ __forceinline__ void store_bulk(void* to, uint32_t from, uint32_t bytes) {
  asm volatile(
      "cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;\n\t"
      "cp.async.bulk.commit_group;\n\t"
      "cp.async.bulk.wait_group 0;" ::"l"(to),
      "r"(from), "r"(bytes)
      : "memory");
}

__device__ __forceinline__ void block_barrier() {    // all warps, wherever they are
  __syncwarp();
  asm volatile("bar.sync 2, 256;" ::: "memory");
}
__device__ __forceinline__ void soft_barrier() {     // the softmax warps
  __syncwarp();
  asm volatile("bar.sync 1, 128;" ::: "memory");
}

// The pages that a tree's nodes see: its first, and how many (0 without nodes).
struct Pages {
  int first, count;
};
__device__ __forceinline__ Pages tree_pages(const TreeArgs& a, const TreeNums& t) {
  const int lo = a.window > 0 ? first_key(0, t.n, a.window) : 0;   // (of positions from n on)
  const int first = min(min(lo, t.n) / kPageTokens, a.cache.pt_stride - 1);
  return {first, t.count > 0 ? max(1, (t.keys + kPageTokens - 1) / kPageTokens - first) : 0};
}
__device__ __forceinline__ int tree_tiles(const TreeArgs& a, int count) {
  return (count * a.G + kWideRows - 1) / kWideRows;
}

// One block's next piece of work.
struct Segment {
  int tree, head, tile, rows;            // rows: in use in this tile; 0: nothing is left
  int n, keys, lo_most;
  int seq, page, pages;                  // pages of the sequence's table
  int64_t part;                          // its row of parts, -1: the whole tile
};

// Blocks that take the tiles of one head, this block's place among them.
struct Team {
  int size, rank;
};

// The order of all work, walked by one warp.  Lane l holds tree 32 chunk + l.
struct Walk {
  int64_t at, end, total;                // this block's pages
  int64_t before;                        // pages of the trees before the chunk
  int64_t work, upto;                    // the lane's tree: its pages, and with those before
  TreeNums nums;                         // its numbers
  int chunk, blocks;
};
// It rests in shared memory between two segments.
struct WalkRest {
  int64_t at, end, work[32], upto[32];
  TreeNums nums[32];
  int chunk;
};
__device__ __forceinline__ void walk_rest(WalkRest& r, const Walk& w, int lane) {
  r.work[lane] = w.work;
  r.upto[lane] = w.upto;
  r.nums[lane] = w.nums;
  if (lane == 0) r.at = w.at, r.end = w.end, r.chunk = w.chunk;
  __syncwarp();
}
__device__ __forceinline__ void walk_wake(const WalkRest& r, Walk& w, int lane) {
  w.work = r.work[lane];
  w.upto = r.upto[lane];
  w.nums = r.nums[lane];
  w.at = r.at;
  w.end = r.end;
  w.chunk = r.chunk;
  __syncwarp();
}
__device__ __forceinline__ int64_t walk_load(const TreeArgs& a, int trees, int lane, Team team, Walk& w,
                                             bool tell) {
  const int tree = w.chunk * 32 + lane;
  w.work = 0;
  w.nums = {0, 0, 0, 0, false};
  int pages = 0;
  if (tree < trees) {
    w.nums = read_tree(a, tree);
    pages = tree_pages(a, w.nums).count;
    w.work = static_cast<int64_t>(pages) * a.cache.Hkv *
             ((tree_tiles(a, w.nums.count) + team.size - 1) / team.size);
    if (tell && w.nums.bad) atomicExch(a.err, kErrBounds);
  }
  w.upto = w.work;
#pragma unroll
  for (int x = 1; x < 32; x *= 2) {
    const int64_t y = __shfl_up_sync(0xFFFFFFFFu, w.upto, x);
    if (lane >= x) w.upto += y;
  }
  const int64_t sum = __shfl_sync(0xFFFFFFFFu, w.upto, 31);
  w.upto += w.before;
  if (tell && tree < trees) a.part_n[tree] = {w.upto - w.work, pages, w.nums.count};
  return sum;
}
__device__ __forceinline__ void walk_begin(const TreeArgs& a, int trees, int lane, Team team, Walk& w) {
  const bool tell = blockIdx.x == 0;
  w.before = 0;
  const int chunks = (trees + 31) / 32;
  for (w.chunk = 0; w.chunk < chunks; ++w.chunk) w.before += walk_load(a, trees, lane, team, w, tell);
  w.total = w.before;
  const int64_t most = max(static_cast<int64_t>(1), w.total / kFewPages);
  const int64_t mine = blockIdx.x / team.size;       // the team's number
  w.blocks = static_cast<int>(min(static_cast<int64_t>(gridDim.x / team.size), most));
  if (tell && lane == 0) a.part_all[0] = w.total, a.part_all[1] = w.blocks;
  w.at = w.end = 0;
  if (mine < w.blocks) {
    w.at = w.total * mine / w.blocks;
    w.end = w.total * (mine + 1) / w.blocks;
  }
  w.before = 0;
  w.chunk = 0;
  if (chunks > 1 && w.at < w.end) walk_load(a, trees, lane, team, w, false);   // (the only one is there)
}
// The first cached key that all of a tree's nodes see (one warp).
__device__ __forceinline__ int last_first_key(const TreeArgs& a, int tree, const TreeNums& t, int lane) {
  if (a.window == 0) return 0;
  int lo = 0;
  for (int i = lane; i < t.count; i += 32)
    lo = max(lo, first_key(a.pos[static_cast<int64_t>(tree) * a.nodes + i], t.n, a.window));
  return __reduce_max_sync(0xFFFFFFFFu, lo);
}
__device__ __forceinline__ void walk_next(const TreeArgs& a, int trees, int lane, Team team, Walk& w,
                                          Segment& s) {
  if (w.at >= w.end) {
    if (lane == 0) s.rows = 0;
    return;
  }
  uint32_t in;
  while (!(in = __ballot_sync(0xFFFFFFFFu, w.upto > w.at)) && (w.chunk + 1) * 32 < trees) {
    w.before = __shfl_sync(0xFFFFFFFFu, w.upto, 31);
    ++w.chunk;
    walk_load(a, trees, lane, team, w, false);
  }
  const int l = in ? __ffs(in) - 1 : 31;
  const int64_t first = __shfl_sync(0xFFFFFFFFu, w.upto - w.work, l);
  const int tree = w.chunk * 32 + l;
  const TreeNums t = {__shfl_sync(0xFFFFFFFFu, w.nums.seq, l), __shfl_sync(0xFFFFFFFFu, w.nums.n, l),
                      __shfl_sync(0xFFFFFFFFu, w.nums.keys, l), __shfl_sync(0xFFFFFFFFu, w.nums.count, l),
                      false};
  const Pages p = tree_pages(a, t);
  const int tiles = tree_tiles(a, t.count);
  const int lo_most = last_first_key(a, tree, t, lane);
  if (lane == 0) {
    const int64_t in_tree = w.at - first;
    const int groups = max((tiles + team.size - 1) / team.size, 1);
    const int unit = in && p.count > 0 ? static_cast<int>(in_tree / p.count) : 0;
    const int from = in && p.count > 0 ? static_cast<int>(in_tree % p.count) : 0;
    const int pages = static_cast<int>(min(static_cast<int64_t>(p.count - from), w.end - w.at));
    s.tree = tree;
    s.head = unit / groups;
    s.tile = unit % groups * team.size + team.rank;
    s.rows = in && pages > 0 && unit < a.cache.Hkv * groups
                 ? (s.tile < tiles ? min(kWideRows, t.count * a.G - s.tile * kWideRows) : -1)
                 : 0;
    s.n = t.n, s.keys = t.keys, s.lo_most = lo_most;
    s.seq = t.seq;
    s.page = p.first + from;
    s.pages = pages;
    // a team's first segment may go on with a tile, its last leave one unfinished
    const int64_t mine = blockIdx.x / team.size;
    s.part = pages == p.count ? -1
                              : ((2 * mine + (from == 0 ? 1 : 0)) * team.size + team.rank) * kWideRows;
  }
  w.at += __shfl_sync(0xFFFFFFFFu, lane == 0 ? max(s.pages, 1) : 0, 0);
}

// The block's next segment: of its share, or its one item.
__device__ __forceinline__ void next_segment(const TreeArgs& a, int trees, int lane, Team team,
                                             int seg, WalkRest& rest, Segment& s) {
  if (a.items == 0) {
    Walk walk;
    walk_wake(rest, walk, lane);
    int rows;
    do {                                 // (a tree may have fewer tiles than the team blocks)
      walk_next(a, trees, lane, team, walk, s);
      rows = __shfl_sync(0xFFFFFFFFu, lane == 0 ? s.rows : 0, 0);
    } while (rows < 0);
    walk_rest(rest, walk, lane);
    return;
  }
  const int tree = blockIdx.z, head = blockIdx.y / a.tiles, tile = blockIdx.y % a.tiles;
  const TreeNums t = read_tree(a, tree);
  const Pages p = tree_pages(a, t);
  const int lo_most = last_first_key(a, tree, t, lane);
  if (lane == 0) {
    const int from = blockIdx.x * a.split;
    const bool any = seg == 0 && from < p.count;
    s = {tree, head, tile, any ? min(kWideRows, t.count * a.G - tile * kWideRows) : 0, t.n, t.keys,
         lo_most, t.seq, p.first + from, min(a.split, p.count - from), p.count > a.split ? 0 : -1};
    if (blockIdx.x == 0 && blockIdx.y == 0 && seg == 0) {
      if (t.bad) atomicExch(a.err, kErrBounds);
      a.part_n[tree] = {0, p.count, t.count};
    }
  }
}

template <bool BF16, int D>
__global__ void __launch_bounds__(kWideThreads, 2)
tree_wide_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                 const TreeArgs a, int trees, int team_size) {
  using L = WideSmem<D>;
  constexpr int H = L::H, ST = L::stages, NP = L::places, O = L::o_col;
  extern __shared__ uint8_t smem_raw[];
  __shared__ Segment s_segs[2];            // this one, the next
  __shared__ WalkRest s_walk;
  __shared__ uint32_t s_some[2][kSoftWarps], s_all[2][kSoftWarps], s_odd[2];
  __shared__ int64_t s_place[kWideRows];   // of each row: its query, then its output
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~static_cast<uintptr_t>(1023));
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + L::bars_at);
  const uint32_t k_full = smem_u32(bars), k_empty = k_full + 8 * ST, v_full = k_empty + 8 * ST,
                 v_empty = v_full + 8 * ST, s_full = v_empty + 8 * ST, p_full = s_full + 8 * NP,
                 pv_done = p_full + 8 * NP, q_full = pv_done + 8 * NP;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 4 * ST + 3 * NP + 1);
  pdl_trigger();   // the joining kernel may take its place; it waits for this one's end
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const bool shared = a.items == 0;      // an open split
  const Team team = {team_size, static_cast<int>(blockIdx.x % team_size)};
  if (warp == kFetchKWarp && shared) {
    Walk walk;
    walk_begin(a, trees, lane, team, walk);
    walk_rest(s_walk, walk, lane);
  }
  if (threadIdx.x == 0) {
    tma_prefetch_desc(&map_k);
    tma_prefetch_desc(&map_v);
    for (int i = 0; i < ST; ++i) {
      mbar_init(k_full + 8 * i, 1);
      mbar_init(k_empty + 8 * i, 1);
      mbar_init(v_full + 8 * i, 1);
      mbar_init(v_empty + 8 * i, 1);
    }
    for (int i = 0; i < NP; ++i) {
      mbar_init(s_full + 8 * i, 1);
      mbar_init(p_full + 8 * i, kSoftWarps);
      mbar_init(pv_done + 8 * i, 1);
    }
    mbar_init(q_full, kSoftWarps);
    fence_mbar_init();
  }
  if (warp == kScoreWarp) tmem_alloc(smem_u32(tmem_slot), kTmemCols);
  bool ok = true;
  // pages are counted over all segments: page j uses ring place j % ST; `at`, the
  // place of S, and `turn`, its uses so far mod 2, are counted along
  int base = 0, at = 0;
  uint32_t turn = 0;
  auto step = [&] {
    if (++at == NP) at = 0, turn ^= 1;
  };
  if (warp >= kSoftWarps) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kWorkRegs));
    int issued = 0;                      // pages whose products this warp has issued
    for (int seg = 0;; ++seg) {
      // (found while the last one's pages are still at work)
      if (warp == kFetchKWarp) next_segment(a, trees, lane, team, seg, s_walk, s_segs[seg & 1]);
      tc_fence_before();
      block_barrier();                   // the last segment's memory is done with, this one is known
      tc_fence_after();
      const Segment& s_seg = s_segs[seg & 1];
      const int pages = s_seg.pages, end = base + pages;
      if (s_seg.rows <= 0) break;
      const uint32_t tmem = *tmem_slot;
      if (warp == kFetchKWarp || warp == kFetchVWarp) {
        // ---- TMA: the segment's pages; lane l holds the number of page 32 i + l
        const bool value = warp == kFetchVWarp;
        const uint32_t full = value ? v_full : k_full, empty = value ? v_empty : k_empty;
        const uint32_t ring = smem_u32(smem + (value ? L::v_at : L::k_at));
        const int32_t* table = a.cache.page_table +
                               static_cast<int64_t>(s_seg.seq) * a.cache.pt_stride + s_seg.page - base;
        const int which = (value ? a.cache.Hkv : 0) + s_seg.head;
        int ids = 0, fetched = base;
        for (int j = base; j < end && ok; ++j) {
          const int i = (j - base) & 31;
          if (i == 0 && j + lane < end) {
            ids = table[j + lane];
            if (ids < 0 || ids >= a.cache.n_pages) {
              atomicExch(a.err, kErrBounds);
              ids = 0;
            }
          }
          const int block = 2 * a.cache.Hkv * __shfl_sync(0xFFFFFFFFu, ids, i) + which;
          if (lane == 0) {
            const uint32_t bar = full + 8 * (j % ST), dst = ring + j % ST * L::page_bytes;
            if (j >= ST) ok = wait_for(empty + 8 * (j % ST), (j / ST + 1) & 1, a.err);
            if (ok) {
              mbar_arrive_expect_tx(bar, L::page_bytes);
              if (value) {
                tma_load_3d(dst, &map_v, 0, 0, block, bar);
              } else {
#pragma unroll
                for (int h = 0; h < H; ++h)
                  tma_load_4d(dst + h * kPageTokens * 128, &map_k, 0, h, 0, block, bar);
              }
              fetched = j + 1;
            }
          }
          ok = __shfl_sync(0xFFFFFFFFu, ok, 0);
        }
        // the ring outlives its copies
        if (lane == 0)
          for (int j = max(base, fetched - ST); j < fetched; ++j)
            wait_for(full + 8 * (j % ST), (j / ST) & 1, a.err);
      } else if (lane == 0 && warp == kScoreWarp) {
        // ---- S, where an earlier page's P was
        const uint64_t qd = umma_desc_sw128(smem_u32(smem));
        ok = ok && wait_for(q_full, seg & 1, a.err);
        for (int j = base; j < end && ok; ++j) {
          const int st = j % ST;
          ok = (j < NP || wait_for(pv_done + 8 * at, turn ^ 1, a.err)) &&
               wait_for(k_full + 8 * st, (j / ST) & 1, a.err);
          if (!ok) break;
          tc_fence_after();
          const uint64_t kd = umma_desc_sw128(smem_u32(smem + L::k_at + st * L::page_bytes));
#pragma unroll
          for (int k = 0; k < D / 16; ++k)
            umma_f16(tmem + 64 * at, qd + (k / 4) * (kWideRows * 128 >> 4) + (k % 4) * 2,
                     kd + (k / 4) * (kPageTokens * 128 >> 4) + (k % 4) * 2,
                     wide_idesc<BF16>(kPageTokens), k > 0);
          umma_commit(s_full + 8 * at);
          umma_commit(k_empty + 8 * st);
          issued = j + 1;
          step();
        }
      } else if (lane == 0) {
        // ---- O += P V
        for (int j = base; j < end && ok; ++j) {
          const int st = j % ST;
          ok = wait_for(v_full + 8 * st, (j / ST) & 1, a.err) &&
               wait_for(p_full + 8 * at, turn, a.err);
          if (!ok) break;
          tc_fence_after();
          const uint64_t vd = umma_desc_sw128(smem_u32(smem + L::v_at + st * L::page_bytes));
#pragma unroll
          for (int k = 0; k < kPageTokens / 16; ++k)
            umma_f16_ta(tmem + O, tmem + 64 * at + 8 * k, vd + k * 2, wide_idesc<BF16>(D));
          umma_commit(pv_done + 8 * at);
          umma_commit(v_empty + 8 * st);
          issued = j + 1;
          step();
        }
      }
      __syncwarp();
      base = end;
    }
    // the block outlives its arrivals: nobody waits for the last pages' places
    if (lane == 0 && (warp == kScoreWarp || warp == kValueWarp))
      for (int j = max(0, issued - ST); j < issued; ++j)
        wait_for((warp == kScoreWarp ? k_empty : v_empty) + 8 * (j % ST), (j / ST) & 1, a.err);
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftRegs));
    for (int seg = 0;; ++seg) {
      tc_fence_before();
      block_barrier();
      tc_fence_after();
      const Segment& s_seg = s_segs[seg & 1];
      const uint32_t tmem = *tmem_slot;
      const int rows = s_seg.rows, pages = s_seg.pages;
      if (rows <= 0) break;
      const int head = s_seg.head, page0 = s_seg.page;
      // ---- softmax: thread = row = lane of tensor memory
      const int r = threadIdx.x;
      const bool live = r < rows, busy = warp * 32 < rows;   // the row, any row of the warp is in use
      const int of = live ? s_seg.tile * kWideRows + r : 0, node = of / a.G;
      const int q_head = head * a.G + of % a.G, n = s_seg.n, lo_most = s_seg.lo_most;
      const int64_t row = static_cast<int64_t>(s_seg.tree) * a.nodes + node;
      // queries, a row's 16-byte pieces by neighbouring threads (rows not in use
      // hold anything: they meet no other, and never rise)
      s_place[r] = live ? row * a.ld_q + static_cast<int64_t>(q_head) * D : -1;
      soft_barrier();
#pragma unroll 4
      for (int i = 0; i < D / 8; ++i) {
        const int e = r + i * kSoftThreads, qr = e / (D / 8), c = e % (D / 8);
        const uint32_t to = smem_u32(smem) + (c / 8) * kWideRows * 128 + swizzled(qr, c % 8);
        if (qr < rows)
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(a.q + s_place[qr] + 8 * c)
                       : "memory");
      }
      const uint32_t trow = tmem + (static_cast<uint32_t>(warp * 32) << 16);
      if (busy) {
        uint32_t zero[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) zero[i] = 0u;
#pragma unroll
        for (int c = 0; c < D / 16; ++c) tmem_st16(trow + O + 16 * c, zero);
        tmem_wait_st();
      }
      uint64_t mask = 0;
      int lo = n;
      if (live) {
        mask = a.mask[row];
        if (s_seg.keys - n < 64) mask &= (1ull << (s_seg.keys - n)) - 1;
        lo = a.window > 0 ? min(first_key(a.pos[row], n, a.window), lo_most) : 0;
      }
      asm volatile("cp.async.wait_all;" ::: "memory");
      fence_proxy_async_smem();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(q_full);
      // waits are warp-uniform; after a failure the warp stops waiting
      auto wait = [&](uint32_t bar, uint32_t phase) {
        if (ok) ok = __all_sync(0xFFFFFFFFu, wait_for(bar, phase, a.err)) != 0;
        return ok;
      };
      const F32x2 scale2 = join2(a.scale_log2, a.scale_log2), set2 = join2(kSet<BF16>, kSet<BF16>);
      float m = -INFINITY, l = 0.f;
      for (int j = 0; j < pages; ++j) {
        const int tok0 = (page0 + j) * kPageTokens;
        const bool edge = tok0 < lo_most || tok0 + kPageTokens > n;
        // the products of the page before this one
        const int was = at == 0 ? NP - 1 : at - 1;
        const uint32_t was_turn = at == 0 ? turn ^ 1 : turn;
        wait(s_full + 8 * at, turn);
        tc_fence_after();
        if (busy) {
          uint32_t s[2][32];
          tmem_ld32_nowait(trow + 64 * at, s[0]);
          tmem_ld32_nowait(trow + 64 * at + 32, s[1]);
          tmem_wait_ld();
          if (edge) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const uint32_t v = row_view(mask, lo, n, tok0 + 32 * h);
#pragma unroll
              for (int i = 0; i < 32; ++i)
                if (!((v >> i) & 1)) s[h][i] = 0xFF800000u;
            }
          }
          float x[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            x[e] = fmaxf(__uint_as_float(s[0][e]), __uint_as_float(s[1][e]));
#pragma unroll
            for (int i = 4; i < 32; i += 4)
              x[e] = max3(x[e], __uint_as_float(s[0][i + e]), __uint_as_float(s[1][i + e]));
          }
          const float mx = fmaxf(max3(x[0], x[1], x[2]), x[3]);
          const bool rise = live && (mx - m) * a.scale_log2 > kRise;   // (m = -inf: any score)
          if (__any_sync(0xFFFFFFFFu, rise)) {
            const float f = rise ? moved_max(m, mx, a.scale_log2) : 1.f;   // (mx is above -inf)
            l *= f;
            if (rise) m = mx;
            if (j > 0 && wait(pv_done + 8 * was, was_turn)) {
              tc_fence_after();
#pragma unroll 1
              for (int c = 0; c < D / 16; ++c) {
                uint32_t o[16];
                tmem_ld16(trow + O + 16 * c, o);
#pragma unroll
                for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(f * __uint_as_float(o[i]));
                tmem_st16(trow + O + 16 * c, o);
              }
            }
          }
          const float z = finite_max(m);
          const F32x2 z2 = join2(-z, -z);
          F32x2 sum2[2] = {join2(0.f, 0.f), join2(0.f, 0.f)};
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            uint32_t p[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const float2 e = split2(fma2(
                  add2(join2(__uint_as_float(s[h][2 * i]), __uint_as_float(s[h][2 * i + 1])), z2), scale2, set2));
              const float u = ex2(e.x), w = ex2(e.y);
              sum2[i & 1] = add2(sum2[i & 1], join2(u, w));
              p[i] = pack2<BF16>(u, w);
            }
            tmem_st16(trow + 64 * at + 16 * h, p);
          }
          const float2 sum = split2(add2(sum2[0], sum2[1]));
          l += sum.x + sum.y;
          tmem_wait_st();
        }
        if (edge) {
          // values that no row sees are cleared; those that are not finite and that
          // some rows see go to their O by hand
          const int st = (base + j) % ST;
          uint8_t* v = smem + L::v_at + st * L::page_bytes;
#pragma unroll
          for (int w = 0; w < 2; ++w) {
            const uint32_t x = row_view(mask, lo, n, tok0 + 32 * w);
            const uint32_t some = __reduce_or_sync(0xFFFFFFFFu, live ? x : 0u),
                           all = __reduce_and_sync(0xFFFFFFFFu, live ? x : 0xFFFFFFFFu);
            if (lane == 0) s_some[w][warp] = some, s_all[w][warp] = all;
          }
          if (r < 2) s_odd[r] = 0u;
          wait(v_full + 8 * st, ((base + j) / ST) & 1);
          soft_barrier();
          // chunk = 8 tokens of a dim
#pragma unroll 1
          for (int e = r; e < D * 8; e += kSoftThreads) {
            const int chunk = e % 8, dim = e / 8, w = chunk / 4, shift = chunk % 4 * 8;
            uint32_t some = 0u, all = 0xFFFFFFFFu;
#pragma unroll
            for (int k = 0; k < kSoftWarps; ++k) some |= s_some[w][k], all &= s_all[w][k];
            const uint32_t keep = some >> shift, part = (some & ~all) >> shift;
            if ((keep & 0xFF) == 0xFF && !(part & 0xFF)) continue;
            uint4* to = reinterpret_cast<uint4*>(v + swizzled(dim, chunk));
            const uint4 x = *to;
            uint32_t word[4] = {x.x, x.y, x.z, x.w}, odd = 0u;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              if (!((keep >> (2 * k)) & 1)) word[k] &= 0xFFFF0000u;
              if (!((keep >> (2 * k + 1)) & 1)) word[k] &= 0x0000FFFFu;
              const uint32_t nf = not_finite<BF16>(word[k]);
              odd |= ((nf & 1u) | (nf >> 30 & 2u)) << (2 * k) & part;
            }
            *to = make_uint4(word[0], word[1], word[2], word[3]);
            if (odd & 0xFFu) atomicOr(&s_odd[w], (odd & 0xFFu) << shift);
          }
          soft_barrier();
          if (s_odd[0] | s_odd[1]) {
            if (j > 0) wait(pv_done + 8 * was, was_turn);
            tc_fence_after();
#pragma unroll 1
            for (int c = 0; c < D / 16; ++c) {
              uint32_t o[16];
              tmem_ld16(trow + O + 16 * c, o);
#pragma unroll 1
              for (int w = 0; w < 2; ++w)
#pragma unroll 1
                for (uint32_t left = s_odd[w] & row_view(mask, lo, n, tok0 + 32 * w); left;
                     left &= left - 1) {
                  const int tok = 32 * w + __ffs(left) - 1;
#pragma unroll
                  for (int i = 0; i < 16; ++i) {
                    const uint32_t h = *reinterpret_cast<const uint16_t*>(
                        v + swizzled(16 * c + i, tok / 8) + tok % 8 * 2);
                    if (not_finite<BF16>(h))
                      o[i] = __float_as_uint(__uint_as_float(o[i]) + unpack2<BF16>(h).x);
                  }
                }
              __syncwarp();
              tmem_st16(trow + O + 16 * c, o);
            }
            tmem_wait_st();
            soft_barrier();
#pragma unroll 1
            for (int e = r; e < D * 8; e += kSoftThreads) {
              const int chunk = e % 8, dim = e / 8;
              const uint32_t odd = s_odd[chunk / 4] >> (chunk % 4 * 8);
              if (!(odd & 0xFF)) continue;
              uint4* to = reinterpret_cast<uint4*>(v + swizzled(dim, chunk));
              const uint4 x = *to;
              uint32_t word[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                const uint32_t sel = ((odd >> (2 * k)) & 1 ? 0x0000FFFFu : 0u) |
                                     ((odd >> (2 * k + 1)) & 1 ? 0xFFFF0000u : 0u);
                word[k] &= ~(not_finite<BF16>(word[k]) & sel);
              }
              *to = make_uint4(word[0], word[1], word[2], word[3]);
            }
          }
          soft_barrier();                  // the words above are free for the next page
          fence_proxy_async_smem();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_full + 8 * at);
        step();
      }
      // ---- the rows' end.  The last O is done, and so are all products and copies:
      // their shared memory takes the rows.  A part's row is copied from there in one piece,
      // an output's is written a row's pieces by neighbours.
      wait(pv_done + 8 * (at == 0 ? NP - 1 : at - 1), at == 0 ? turn ^ 1 : turn);
      tc_fence_after();
      const int64_t out_at = row * a.Hq + q_head, part = s_seg.part;
      const bool whole = part < 0;
      constexpr int P = D + 4;
      float* so = reinterpret_cast<float*>(smem);
      const float inv = !whole ? 1.f : l != 0.f ? 1.f / l : 0.f;
      if (busy) {
#pragma unroll 1
        for (int c = 0; c < D / 16; ++c) {
          uint32_t o[16];
          tmem_ld16(trow + O + 16 * c, o);
#pragma unroll
          for (int i = 0; i < 16; i += 4)
            *reinterpret_cast<float4*>(so + r * P + 16 * c + i) =
                make_float4(__uint_as_float(o[i]) * inv, __uint_as_float(o[i + 1]) * inv,
                            __uint_as_float(o[i + 2]) * inv, __uint_as_float(o[i + 3]) * inv);
        }
      }
      fence_proxy_async_smem();            // (bulk copies follow, and those of the next segment)
      if (!whole) {
        if (live) {
          const int64_t slot = shared ? part + r : out_at * a.items + blockIdx.x;
          a.part_ml[slot] = make_float2(m, l);
          store_bulk(a.part_o + slot * D, smem_u32(so + r * P), D * 4);
        }
      } else {
        if (live) {
          if (a.lse) a.lse[out_at] = row_lse(a, m, l);
          s_place[r] = row * a.ld_out + static_cast<int64_t>(q_head) * D;
        }
        soft_barrier();
#pragma unroll 4
        for (int e = r; e < rows * (D / 4); e += kSoftThreads) {
          const int i = e / (D / 4), d = e % (D / 4) * 4;
          const float4 v = *reinterpret_cast<const float4*>(so + i * P + d);
          *reinterpret_cast<uint2*>(a.out + s_place[i] + d) =
              make_uint2(pack2<BF16>(v.x, v.y), pack2<BF16>(v.z, v.w));
        }
        fence_proxy_async_smem();
      }
      base += pages;
    }
  }
  if (warp == kScoreWarp) {
    __syncwarp();
    tmem_dealloc(*tmem_slot, kTmemCols);
  }
}

// The pool as the kernels' TMA boxes see it: blocks (a page's K or V^T of a KV
// head) of K as [64 tokens][halves][64 dims], of V^T as [dims][64 tokens].
inline bool pool_maps(const gs_cache& c, CUtensorMap* k, CUtensorMap* v) {
  const uint64_t D = c.head_dim, blocks = 2ull * c.n_pages * c.n_kv_heads;
  const uint64_t kd[4] = {64, D / 64, kPageTokens, blocks}, ks[3] = {128, D * 2, D * kPageTokens * 2};
  const uint32_t kb[4] = {64, 1, kPageTokens, 1};
  const uint64_t vd[3] = {64, D, blocks}, vs[2] = {128, D * kPageTokens * 2};
  const uint32_t vb[3] = {64, static_cast<uint32_t>(D), 1};
  return make_map_nd(k, c.kv, 4, kd, ks, kb) && make_map_nd(v, c.kv, 3, vd, vs, vb);
}

}  // namespace
}  // namespace gs
