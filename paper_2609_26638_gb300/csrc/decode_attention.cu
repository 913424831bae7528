// decode_attention.cu -- attention of one new token per sequence over the
// paged cache, split over the cache's length and joined.
//
//   s_j = scale * q . k_j over the visible keys j in [max(0, n - window), n)
//   o = sum_j 2^(s_j' - m) v_j / l,  l = sum_j 2^(s_j' - m),  s' = s log2(e)
//
// Each key and value is read once for its group of query heads, with 4 G
// flops per 4 bytes, so HBM bounds every group that shares a KV head.  The
// work is cut into items of `split` pages; a block takes one item of one KV
// head (and up to 16 of its query heads), its warps take the item's pages in
// turn.  A warp is its own pipeline: lane 0 streams the warp's pages, K block
// then V^T block (each contiguous), by bulk copies into a private ring of
// shared-memory blocks, the warp computes and gives the block back with a
// warp-level barrier, so no two warps ever wait for each other before the
// item's end.
//
// The products are m16n8k16 tensor instructions on the 16 query rows.  One
// token fills at most 16 of the 128 rows of a tcgen05 tile, and its
// accumulator would have to come back from tensor memory twice a page; here
// scores and probabilities never leave the registers.  A dot product does not
// care in which order its terms come, so each lane takes 16 contiguous bytes
// as its share of the operand: of a K row, 8 dims (Q is held in the same
// order); of a V^T row, 8 tokens.  The S tile's columns are given to the tokens
// in the order in which the accumulators of one lane are again the P operand of
// the 8 tokens whose values it reads, so P needs no exchange either.
//
// Running max (log2 units), sum and accumulators are fp32.  P is rounded to
// the cache's type for the second product: at most 1, relative error 2^-12
// (fp16) or 2^-9 (bf16), below the output's own rounding after averaging; the
// sum l takes the unrounded P.
#include <cmath>

#include "internal.h"
#include "step_common.cuh"

namespace gs {
namespace {

constexpr int kRows = 16;            // query heads of one block
constexpr size_t kErrBytes = 256;    // the error word at the scratch's start
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

struct DecodeArgs {
  const uint16_t* q;
  int64_t ld_q;
  const int32_t *seq, *n;
  uint16_t* out;
  int64_t ld_out;
  float* lse;
  int Hq, G, tiles, window, split, items;
  float scale_log2;
  float* part_o;      // [row][head][item][D]
  float2* part_ml;    // [row][head][item]
  int* err;
  CacheView cache;
};

// The visible keys of a row, and its pages.
struct Span {
  int lo, n, page0, pages;
  const int32_t* table;
};
// The row's numbers are read by one lane and broadcast: every lane of a warp
// goes through the same pages whatever happens to the arrays meanwhile.
__device__ __forceinline__ Span find_span(const DecodeArgs& a, int row) {
  Span s;
  const int lane = threadIdx.x & 31;
  int seq = 0, n = 0;
  if (lane == 0) {
    seq = a.seq ? a.seq[row] : row;
    n = a.n[row];
    bool bad = false;
    if (seq < 0 || seq >= a.cache.n_seq) {
      bad = true;
      seq = 0;
      n = 0;
    }
    if (n < 0 || n > a.cache.pt_stride * kPageTokens) {
      bad = true;
      n = n < 0 ? 0 : a.cache.pt_stride * kPageTokens;
    }
    if (bad) atomicExch(a.err, kErrBounds);
  }
  seq = __shfl_sync(0xFFFFFFFFu, seq, 0);
  s.n = __shfl_sync(0xFFFFFFFFu, n, 0);
  s.lo = a.window > 0 && s.n > a.window ? s.n - a.window : 0;
  s.page0 = s.lo / kPageTokens;
  s.pages = (s.n + kPageTokens - 1) / kPageTokens - s.page0;
  s.table = a.cache.page_table + static_cast<int64_t>(seq) * a.cache.pt_stride;
  return s;
}

template <bool BF16>
__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                         uint32_t a3, uint32_t b0, uint32_t b1) {
  if constexpr (BF16)
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
        "{%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
        "{%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint4 lds128(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "r"(addr)
               : "memory");
  return v;
}

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Contiguous copy of `bytes` (a multiple of 16) into shared memory.
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes,
                                          uint32_t bar) {
  asm volatile(
      "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
          dst),
      "l"(reinterpret_cast<uint64_t>(src)), "r"(bytes), "r"(bar)
      : "memory");
}

// m = -inf means no weight at all: such a max is taken as 0, so that its
// exponentials are 2^-inf = 0 and not 2^(inf - inf).
__device__ __forceinline__ float finite_max(float m) { return m == -INFINITY ? 0.f : m; }

template <int D>
struct DecodeShape {
  static constexpr int kBlock = kPageTokens * D * 2;    // bytes of one K or V^T block
  static constexpr int kWarps = D == 64 ? 4 : 2;
  static constexpr int kRing = 3;                       // blocks of a warp's ring
  static constexpr int kThreads = kWarps * 32;
  static constexpr int kRingBytes = kWarps * kRing * kBlock;
  static constexpr int kSmem = kRingBytes + 128;        // and the alignment of its start
};

// WIDE: more than 8 query rows (the upper half of the tile is in use).
template <bool BF16, int D, bool WIDE>
__global__ void __launch_bounds__(DecodeShape<D>::kThreads, 2)
decode_attention_kernel(const DecodeArgs a) {
  using S = DecodeShape<D>;
  extern __shared__ uint8_t smem_raw[];
  __shared__ uint64_t bars[S::kWarps * S::kRing];
  __shared__ float2 s_ml[S::kWarps][kRows];
  pdl_trigger();   // the joining kernel may take its place; it waits for this one's end
  const int row = blockIdx.z, head = blockIdx.y / a.tiles, tile = blockIdx.y % a.tiles;
  const int item = blockIdx.x;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
  const Span sp = find_span(a, row);
  const int items = (sp.pages + a.split - 1) / a.split;
  if (item >= items && item > 0) return;
  const int h0 = head * a.G + tile * kRows;              // first query head of the block
  const int rows = min(kRows, a.G - tile * kRows);
  const int p0 = item * a.split;                         // this item's pages, from page0
  const int cnt_all = min(a.split, sp.pages - p0);       // 0 for an empty row
  const int cnt = cnt_all > warp ? (cnt_all - warp + S::kWarps - 1) / S::kWarps : 0;

  uint8_t* smem = reinterpret_cast<uint8_t*>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 127) & ~static_cast<uintptr_t>(127));
  const uint32_t ring = smem_u32(smem) + warp * S::kRing * S::kBlock;
  const uint32_t bar = smem_u32(bars) + warp * S::kRing * 8;
  if (lane == 0) {
    for (int i = 0; i < S::kRing; ++i) mbar_init(bar + 8 * i, 1);
    fence_mbar_init();
    fence_proxy_async_smem();
  }
  __syncwarp();

  // Q in the operand's order: of each 32 dims, dims 8q .. 8q + 7 on lane q.
  uint32_t qa[D / 32][4], qb[D / 32][4];
  const uint16_t* q_row = a.q + row * a.ld_q + static_cast<int64_t>(h0) * D + 8 * q;
#pragma unroll
  for (int c = 0; c < D / 32; ++c) {
    const uint4 z = make_uint4(0, 0, 0, 0);
    const uint4 u = g < rows ? *reinterpret_cast<const uint4*>(q_row + g * D + 32 * c) : z;
    const uint4 v =
        WIDE && g + 8 < rows ? *reinterpret_cast<const uint4*>(q_row + (g + 8) * D + 32 * c) : z;
    qa[c][0] = u.x, qa[c][1] = u.y, qa[c][2] = u.z, qa[c][3] = u.w;
    qb[c][0] = v.x, qb[c][1] = v.y, qb[c][2] = v.z, qb[c][3] = v.w;
  }

  // The warp's j-th page is page p0 + warp + j * kWarps of the row; lane l
  // holds the pool's page of j = 32 i + l.
  int ids = 0;
  auto load_ids = [&](int j0) {
    const int j = j0 + lane;
    if (j < cnt) ids = sp.table[sp.page0 + p0 + warp + j * S::kWarps];
  };
  // Block b of the warp's stream: K of page b / 2, then its V^T.
  auto issue = [&](int b) {
    const int j = b >> 1;
    if (j >= cnt) return;
    if (!(b & 1) && !(j & 31)) load_ids(j);
    int page = __shfl_sync(0xFFFFFFFFu, ids, j & 31);
    if (lane == 0) {
      if (page < 0 || page >= a.cache.n_pages) {
        atomicExch(a.err, kErrBounds);
        page = 0;
      }
      const int st = b % S::kRing;
      // of the last page's keys only the rows that exist
      const int tok = (sp.page0 + p0 + warp + j * S::kWarps) * kPageTokens;
      const uint32_t bytes =
          b & 1 ? S::kBlock : static_cast<uint32_t>(min(kPageTokens, sp.n - tok)) * (D * 2);
      mbar_arrive_expect_tx(bar + 8 * st, bytes);
      bulk_load(ring + st * S::kBlock, a.cache.block(page, b & 1, head, D), bytes, bar + 8 * st);
    }
  };
  // Block b has landed; the same answer in every lane.
  auto arrived = [&](int b) {
    const bool here = mbar_wait(bar + 8 * (b % S::kRing), (b / S::kRing) & 1, a.err);
    return __all_sync(0xFFFFFFFFu, here) != 0;
  };
  for (int b = 0; b < S::kRing; ++b) issue(b);

  float o[D / 8][4];
#pragma unroll
  for (int i = 0; i < D / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
  float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f;
  int b = 0;
  bool ok = true;
  for (int j = 0; j < cnt && ok; ++j) {
    const int tok0 = (sp.page0 + p0 + warp + j * S::kWarps) * kPageTokens;
    const bool edge = tok0 < sp.lo || tok0 + kPageTokens > sp.n;
    // ---- S = Q K^T
    float s[8][4];
#pragma unroll
    for (int i = 0; i < 8; ++i) s[i][0] = s[i][1] = s[i][2] = s[i][3] = 0.f;
    ok = arrived(b);
    if (!ok) break;
    {
      const uint32_t kb = ring + (b % S::kRing) * S::kBlock + q * 16;
#pragma unroll
      for (int i = 0; i < 8; ++i) {      // column n of S tile i: token 32 (i/4) + 8 (n/2) + 2 (i%4) + n%2
        const uint32_t r = kb + (32 * (i >> 2) + 8 * (g >> 1) + 2 * (i & 3) + (g & 1)) * (D * 2);
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
          const uint4 k = lds128(r + 64 * c);
          mma16816<BF16>(s[i], qa[c][0], qb[c][0], qa[c][1], qb[c][1], k.x, k.y);
          mma16816<BF16>(s[i], qa[c][2], qb[c][2], qa[c][3], qb[c][3], k.z, k.w);
        }
      }
    }
    __syncwarp();                        // every lane has read the block
    issue(b + S::kRing);
    ++b;
    // ---- softmax; this lane's columns 2q, 2q + 1 of tile i are tokens
    //      tok0 + 32 (i/4) + 8 q + 2 (i%4) + {0, 1}
    if (edge) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int t = tok0 + 32 * (i >> 2) + 8 * q + 2 * (i & 3);
        if (t < sp.lo || t >= sp.n) s[i][0] = s[i][2] = -INFINITY;
        if (t + 1 < sp.lo || t + 1 >= sp.n) s[i][1] = s[i][3] = -INFINITY;
      }
    }
    float x0 = -INFINITY, x1 = -INFINITY;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x0 = fmaxf(x0, fmaxf(s[i][0], s[i][1]));
      if (WIDE) x1 = fmaxf(x1, fmaxf(s[i][2], s[i][3]));
    }
    x0 = fmaxf(x0, __shfl_xor_sync(0xFFFFFFFFu, x0, 1));
    x0 = fmaxf(x0, __shfl_xor_sync(0xFFFFFFFFu, x0, 2));
    if (WIDE) {
      x1 = fmaxf(x1, __shfl_xor_sync(0xFFFFFFFFu, x1, 1));
      x1 = fmaxf(x1, __shfl_xor_sync(0xFFFFFFFFu, x1, 2));
    }
    const float n0 = fmaxf(m0, x0 * a.scale_log2), n1 = fmaxf(m1, x1 * a.scale_log2);
    const bool rises = n0 != m0 || (WIDE && n1 != m1);
    if (__any_sync(0xFFFFFFFFu, rises)) {
      const float f0 = ex2(m0 - finite_max(n0)), f1 = WIDE ? ex2(m1 - finite_max(n1)) : 1.f;
      l0 *= f0;
      l1 *= f1;
#pragma unroll
      for (int i = 0; i < D / 8; ++i) {
        o[i][0] *= f0;
        o[i][1] *= f0;
        if (WIDE) o[i][2] *= f1, o[i][3] *= f1;
      }
      m0 = n0;
      m1 = n1;
    }
    const float z0 = finite_max(m0), z1 = finite_max(m1);
    uint32_t pa[8], pb[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float u = ex2(fmaf(s[i][0], a.scale_log2, -z0)), v = ex2(fmaf(s[i][1], a.scale_log2, -z0));
      l0 += u + v;
      pa[i] = pack2<BF16>(u, v);
      pb[i] = 0u;
      if (WIDE) {
        const float w = ex2(fmaf(s[i][2], a.scale_log2, -z1)),
                    y = ex2(fmaf(s[i][3], a.scale_log2, -z1));
        l1 += w + y;
        pb[i] = pack2<BF16>(w, y);
      }
    }
    // ---- O += P V
    ok = arrived(b);
    if (!ok) break;
    {
      const uint32_t vb = ring + (b % S::kRing) * S::kBlock + q * 16;
#pragma unroll
      for (int i = 0; i < D / 8; ++i) {
        const uint32_t r = vb + (8 * i + g) * (kPageTokens * 2);
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          uint4 v = lds128(r + 64 * c);
          if (edge) {                    // what lies behind the mask may be anything, NaN too
            uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int t = tok0 + 32 * c + 8 * q + 2 * e;
              if (t < sp.lo || t >= sp.n) w[e] &= 0xFFFF0000u;
              if (t + 1 < sp.lo || t + 1 >= sp.n) w[e] &= 0x0000FFFFu;
            }
            v = make_uint4(w[0], w[1], w[2], w[3]);
          }
          mma16816<BF16>(o[i], pa[4 * c], pb[4 * c], pa[4 * c + 1], pb[4 * c + 1], v.x, v.y);
          mma16816<BF16>(o[i], pa[4 * c + 2], pb[4 * c + 2], pa[4 * c + 3], pb[4 * c + 3], v.z, v.w);
        }
      }
    }
    __syncwarp();
    issue(b + S::kRing);
    ++b;
  }
  if (!ok) {   // a wait gave up: the copies still under way must land before the block ends
    for (int e = b; e < min(2 * cnt, b + S::kRing); ++e) arrived(e);
  }

  // ---- the warps' parts are joined through the ring's memory, in warp order
  l0 += __shfl_xor_sync(0xFFFFFFFFu, l0, 1);
  l0 += __shfl_xor_sync(0xFFFFFFFFu, l0, 2);
  l1 += __shfl_xor_sync(0xFFFFFFFFu, l1, 1);
  l1 += __shfl_xor_sync(0xFFFFFFFFu, l1, 2);
  if (q == 0) {
    s_ml[warp][g] = make_float2(m0, l0);
    s_ml[warp][g + 8] = make_float2(m1, l1);
  }
  __syncthreads();                       // the rings are free from here on
  constexpr int P = D + 8;               // row pitch: 8-byte stores of 8 rows x 4 lanes on distinct banks
  float* so = reinterpret_cast<float*>(smem);
  if (cnt > 0) {
#pragma unroll
    for (int i = 0; i < D / 8; ++i) {
      *reinterpret_cast<float2*>(so + (warp * kRows + g) * P + 8 * i + 2 * q) =
          make_float2(o[i][0], o[i][1]);
      if (WIDE)
        *reinterpret_cast<float2*>(so + (warp * kRows + g + 8) * P + 8 * i + 2 * q) =
            make_float2(o[i][2], o[i][3]);
    }
  }
  __syncthreads();
  const int used = min(S::kWarps, cnt_all);
  for (int e = threadIdx.x; e < rows * (D / 4); e += S::kThreads) {
    const int r = e / (D / 4), d = e % (D / 4) * 4;
    float m = -INFINITY, l = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int w = 0; w < used; ++w) m = fmaxf(m, s_ml[w][r].x);
    const float z = finite_max(m);
    for (int w = 0; w < used; ++w) {
      const float f = ex2(s_ml[w][r].x - z);
      const float4 v = *reinterpret_cast<const float4*>(so + (w * kRows + r) * P + d);
      l = fmaf(f, s_ml[w][r].y, l);
      acc.x = fmaf(f, v.x, acc.x);
      acc.y = fmaf(f, v.y, acc.y);
      acc.z = fmaf(f, v.z, acc.z);
      acc.w = fmaf(f, v.w, acc.w);
    }
    const int64_t at = static_cast<int64_t>(row) * a.Hq + h0 + r;
    if (items > 1) {
      *reinterpret_cast<float4*>(a.part_o + (at * a.items + item) * D + d) = acc;
      if (d == 0) a.part_ml[at * a.items + item] = make_float2(m, l);
    } else {
      const float inv = l != 0.f ? 1.f / l : 0.f;
      *reinterpret_cast<uint2*>(a.out + row * a.ld_out + static_cast<int64_t>(h0 + r) * D + d) =
          make_uint2(pack2<BF16>(acc.x * inv, acc.y * inv), pack2<BF16>(acc.z * inv, acc.w * inv));
      if (d == 0 && a.lse) a.lse[at] = l != 0.f ? (z + log2f(l)) * kLn2 : -INFINITY;
    }
  }
}

// Joins a row's items, one query head per block: the items are dealt to the
// block's thread groups (one thread per four dims) in turn and the groups'
// sums are added in order, so the result depends on the row's items alone.
constexpr int kJoinThreads = 256;

template <bool BF16, int D>
__global__ void __launch_bounds__(kJoinThreads) decode_join_kernel(const DecodeArgs a) {
  constexpr int L = D / 4, NG = kJoinThreads / L;
  __shared__ float s_max[kJoinThreads / 32];
  __shared__ float4 s_acc[NG][L];
  __shared__ float s_l[NG];
  const int h = blockIdx.x, row = blockIdx.y;
  const Span sp = find_span(a, row);     // inputs of the call, not of the first kernel
  const int items = (sp.pages + a.split - 1) / a.split;
  pdl_wait();                            // in every block: the grid ends after the first kernel's
  if (items <= 1) return;
  const int64_t at = static_cast<int64_t>(row) * a.Hq + h;
  const float2* ml = a.part_ml + at * a.items;
  const float4* po = reinterpret_cast<const float4*>(a.part_o + at * a.items * D);
  float m = -INFINITY;
  for (int i = threadIdx.x; i < items; i += kJoinThreads) m = fmaxf(m, ml[i].x);
#pragma unroll
  for (int x = 16; x; x >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, x));
  if ((threadIdx.x & 31) == 0) s_max[threadIdx.x >> 5] = m;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kJoinThreads / 32; ++w) m = fmaxf(m, s_max[w]);
  const float z = finite_max(m);
  const int grp = threadIdx.x / L, d = threadIdx.x % L;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  float l = 0.f;
#pragma unroll 4
  for (int i = grp; i < items; i += NG) {
    const float2 x = ml[i];
    const float4 v = po[static_cast<int64_t>(i) * L + d];
    const float f = ex2(x.x - z);
    l = fmaf(f, x.y, l);
    acc.x = fmaf(f, v.x, acc.x);
    acc.y = fmaf(f, v.y, acc.y);
    acc.z = fmaf(f, v.z, acc.z);
    acc.w = fmaf(f, v.w, acc.w);
  }
  s_acc[grp][d] = acc;
  if (d == 0) s_l[grp] = l;
  __syncthreads();
  if (grp > 0) return;
  for (int k = 1; k < NG; ++k) {
    const float4 v = s_acc[k][d];
    acc.x += v.x;
    acc.y += v.y;
    acc.z += v.z;
    acc.w += v.w;
    l += s_l[k];
  }
  const float inv = l != 0.f ? 1.f / l : 0.f;
  *reinterpret_cast<uint2*>(a.out + row * a.ld_out + static_cast<int64_t>(h) * D + 4 * d) =
      make_uint2(pack2<BF16>(acc.x * inv, acc.y * inv), pack2<BF16>(acc.z * inv, acc.w * inv));
  if (d == 0 && a.lse) a.lse[at] = l != 0.f ? (z + log2f(l)) * kLn2 : -INFINITY;
}

// Pages of an item when the caller leaves it open.  One wave of blocks (two
// per SM) shares the cache of few rows evenly; many rows are cut into items
// of at most kMostPages, so that the last wave's tail is short.
constexpr int64_t kSlots = 2 * kNumSMs;
constexpr int kMostPages = 32;
int auto_split(int pages, int64_t blocks_per_item, int warps) {
  int64_t split = (pages * blocks_per_item + kSlots - 1) / kSlots;
  if (split < warps) split = warps;
  if (split > kMostPages && blocks_per_item >= kSlots) split = kMostPages;
  return static_cast<int>(split < pages ? split : pages);
}

struct Plan {
  int tiles, split, items;
};
Plan plan_decode(const gs_cache& c, int rows, int n_heads, int window, int split_pages) {
  Plan p;
  const int G = n_heads / c.n_kv_heads;
  p.tiles = (G + kRows - 1) / kRows;
  int pages = c.pt_stride;
  if (window > 0 && (window + kPageTokens - 2) / kPageTokens + 1 < pages)
    pages = (window + kPageTokens - 2) / kPageTokens + 1;
  const int warps = c.head_dim == 64 ? DecodeShape<64>::kWarps : DecodeShape<128>::kWarps;
  p.split = split_pages > 0 ? split_pages
                            : auto_split(pages, static_cast<int64_t>(rows) * c.n_kv_heads * p.tiles,
                                         warps);
  p.items = (pages + p.split - 1) / p.split;
  return p;
}

template <bool BF16, int D>
cudaError_t launch_decode(const DecodeArgs& a, int rows, cudaStream_t s) {
  using S = DecodeShape<D>;
  static DeviceOnce once;
  cudaError_t e = once.run([] {
    cudaError_t r = cudaFuncSetAttribute(decode_attention_kernel<BF16, D, true>,
                                         cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem);
    if (r == cudaSuccess)
      r = cudaFuncSetAttribute(decode_attention_kernel<BF16, D, false>,
                               cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem);
    return r;
  });
  if (e != cudaSuccess) return e;
  auto kernel = a.G > 8 ? decode_attention_kernel<BF16, D, true> : decode_attention_kernel<BF16, D, false>;
  e = launch_ex(kernel, dim3(a.items, a.cache.Hkv * a.tiles, rows), dim3(S::kThreads), S::kSmem, s,
                false, dim3(1, 1, 1), a);
  if (e != cudaSuccess || a.items == 1) return e;
  return launch_ex(decode_join_kernel<BF16, D>, dim3(a.Hq, rows), dim3(kJoinThreads), 0, s, true,
                   dim3(1, 1, 1), a);
}

size_t up256(size_t x) { return (x + 255) / 256 * 256; }

struct Scratch {
  size_t o, ml, total;   // offsets of the partial accumulators and of their (max, sum)
};
Scratch scratch_of(const gs_cache& c, int rows, int n_heads, size_t items) {
  const size_t n = static_cast<size_t>(rows) * n_heads * items;
  const size_t ml = kErrBytes + up256(n * c.head_dim * sizeof(float));
  return {kErrBytes, ml, ml + up256(n * sizeof(float2))};
}

bool heads_ok(const gs_cache* c, int rows, int n_heads, int split_pages) {
  return rows >= 0 && n_heads >= 1 && n_heads <= (1 << 16) && n_heads % c->n_kv_heads == 0 &&
         split_pages >= 0;
}

}  // namespace
}  // namespace gs

extern "C" size_t gs_decode_attention_scratch_bytes(const gs_cache* cache, int rows, int n_heads,
                                                    int split_pages) {
  using namespace gs;
  if (check_cache(cache) != GS_OK || !heads_ok(cache, rows, n_heads, split_pages)) return 0;
  const Plan p = plan_decode(*cache, rows, n_heads, 0, split_pages);
  // An open split follows the pages that a window leaves: whatever it is, the
  // items are at most one wave's share, or pages / kMostPages, and the rounding.
  size_t items = p.items;
  if (split_pages == 0) {
    const int64_t blocks = static_cast<int64_t>(rows < 1 ? 1 : rows) * cache->n_kv_heads * p.tiles;
    const size_t wave = static_cast<size_t>(kSlots / blocks), cut = cache->pt_stride / kMostPages;
    items = (wave > cut ? wave : cut) + 2;
    if (items > static_cast<size_t>(cache->pt_stride)) items = cache->pt_stride;
  }
  return scratch_of(*cache, rows, n_heads, items).total;
}

extern "C" int gs_decode_attention(const gs_cache* cache, const void* q, int64_t ld_q,
                                   const int32_t* seq, const int32_t* n, int rows, int n_heads,
                                   float scale, int window, void* out, int64_t ld_out, float* lse,
                                   int split_pages, void* scratch, size_t scratch_bytes,
                                   void* stream) {
  using namespace gs;
  if (const int rc = check_cache(cache)) return rc;
  if (!heads_ok(cache, rows, n_heads, split_pages) || !q || !n || !out || !scratch || window < 0 ||
      !(scale > 0.f) || !std::isfinite(scale))
    return GS_ERR_INVALID_ARG;
  const int D = cache->head_dim;
  const int64_t width = static_cast<int64_t>(n_heads) * D;
  if (ld_q < width || ld_out < width || ld_q % 8 || ld_out % 8 || !aligned16(q) || !aligned16(out) ||
      (reinterpret_cast<uintptr_t>(scratch) & 255))
    return GS_ERR_INVALID_ARG;
  if (rows > 65535) return GS_ERR_UNSUPPORTED;
  if (scratch_bytes < gs_decode_attention_scratch_bytes(cache, rows, n_heads, split_pages))
    return GS_ERR_OOM;
  if (rows == 0) return GS_OK;
  const Plan p = plan_decode(*cache, rows, n_heads, window, split_pages);
  const Scratch sc = scratch_of(*cache, rows, n_heads, p.items);
  uint8_t* base = static_cast<uint8_t*>(scratch);
  DecodeArgs a;
  a.q = static_cast<const uint16_t*>(q);
  a.ld_q = ld_q;
  a.seq = seq;
  a.n = n;
  a.out = static_cast<uint16_t*>(out);
  a.ld_out = ld_out;
  a.lse = lse;
  a.Hq = n_heads;
  a.G = n_heads / cache->n_kv_heads;
  a.tiles = p.tiles;
  a.window = window;
  a.split = p.split;
  a.items = p.items;
  a.scale_log2 = scale * kLog2e;
  a.part_o = reinterpret_cast<float*>(base + sc.o);
  a.part_ml = reinterpret_cast<float2*>(base + sc.ml);
  a.err = static_cast<int*>(scratch);
  a.cache = cache_view(*cache);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e;
  if (cache->dtype == GS_BF16)
    e = D == 64 ? launch_decode<true, 64>(a, rows, s) : launch_decode<true, 128>(a, rows, s);
  else
    e = D == 64 ? launch_decode<false, 64>(a, rows, s) : launch_decode<false, 128>(a, rows, s);
  return e == cudaSuccess ? GS_OK : GS_ERR_CUDA;
}
