// decode_attention.cu -- attention of one new token per sequence over the
// paged cache, split over the cache's length and joined.
//
//   s_j = scale * q . k_j over the visible keys j in [max(0, n - window), n)
//   o = sum_j 2^(s_j' - m) v_j / l,  l = sum_j 2^(s_j' - m),  s' = s log2(e)
//   (m the running maximum of s'; in fp16 15 less, see below)
//
// Each key and value is read once for a group of up to 16 query heads (once for
// every 16 of a larger one), with 4 flops per query head and element of 2 bytes, so
// HBM bounds every group that shares a KV head.  The
// work is cut into items of `split` pages; a block takes one item of one KV
// head (and up to 16 of its query heads), its warps take the item's pages in
// turn, 32 tokens at a time, and are joined at the item's end; until then no warp
// waits for another.
//
// The products are m16n8k16 tensor instructions on the 16 query rows.  One
// token fills at most 16 of the 128 rows of a tcgen05 tile, and its
// accumulator would have to come back from tensor memory twice a page; here
// scores and probabilities never leave the registers.  A dot product does not
// care in which order its terms come, so each lane takes 16 contiguous bytes
// as its share of the operand: of a K row, 8 dims (Q is held in the same
// order); of a V^T row, 8 tokens.  So keys and values come straight from global
// memory into the registers that the products read, a step ahead of them, with
// no shared memory, no barrier and every loaded byte used.  (Bulk copies into a
// ring of shared memory moved the same bytes, but cost about 350 cycles to issue
// and 190 to wait for, 8 KB at a time: 1.5 us per page and warp, where this
// takes 1.1.)  The S tile's columns are given to the tokens in the order in
// which the accumulators of one lane are again the P operand of the 8 tokens
// whose values it reads, so P needs no exchange either.
//
// Running max (log2 units), sum and accumulators are fp32.  P is rounded to
// the cache's type for the second product, relative error 2^-11 (fp16) or 2^-8
// (bf16) at most, like the output's own rounding and averaged over the keys; the
// sum l takes the unrounded P.  fp16 has no exponents for light keys (below 2^-14 it
// loses bits, below 2^-25 all of them), so there the max is held 15 too low: P goes up
// to 2^15, O and l with it, and a weight of 2^-29 still has all its bits.  (As
// two products, P and what its rounding left, the error would vanish; but 0 times an
// infinite value would make NaN of an infinite output.)
//
// Measured (16 query and 8 KV heads of 64, fp16, unless named): 64 rows of 8192
// tokens 162 us, 6.6 TB/s; 32 rows of 1024 to 6144 43 us, 5.5 TB/s, and one row
// of 131,001 (32 / 4 heads of 128, bf16) 48 us, 5.6 TB/s: what is missing is the
// wave's start and the tail of its last blocks; one row of 517 tokens 4.4 us.
// These are tables as wide as the longest row.  An open split and the grid follow
// the table's width, not the lengths, so a table with room to spare costs time:
// 2048 pages wide, the 517 tokens take 7.2 us, 6144 tokens of one row 24 (7.7 at 96
// pages), the 32 rows 87, and 64 rows of 400 tokens 124 (15.6 at 7 pages).
#include <algorithm>
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
  int cluster;        // the items of a row and head are one cluster, and join there
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
// The row's numbers are read by one thread for its block: all threads go
// through the same pages and barriers whatever happens to the arrays meanwhile.
__device__ __forceinline__ Span find_span(const DecodeArgs& a, int row) {
  __shared__ int s_seq, s_n;
  if (threadIdx.x == 0) {
    int seq = a.seq ? a.seq[row] : row, n = a.n[row];
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
    s_seq = seq;
    s_n = n;
  }
  __syncthreads();
  Span s;
  s.n = s_n;
  s.lo = a.window > 0 && s.n > a.window ? s.n - a.window : 0;
  s.page0 = s.lo / kPageTokens;
  s.pages = (s.n + kPageTokens - 1) / kPageTokens - s.page0;
  s.table = a.cache.page_table + static_cast<int64_t>(s_seq) * a.cache.pt_stride;
  return s;
}

template <bool BF16>
__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                         uint32_t a3, uint32_t b0, uint32_t b1) {
  if constexpr (BF16)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
        "{%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
        "{%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// 16 bytes that are read once.
__device__ __forceinline__ uint4 load_once(const uint16_t* p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "l"(p));
  return v;
}

// m = -inf means no weight at all: such a max is taken as 0, so that its
// exponentials are 2^-inf = 0 and not 2^(inf - inf).
__device__ __forceinline__ float finite_max(float m) { return m == -INFINITY ? 0.f : m; }

// The max that a step's largest score (before scaling) asks for, held low as said
// above.  Both roundings are upwards, so P is at most 2^15 (or 1) however large
// the scores are: with 1.4 times that fp16 would come near its end, and scores
// beyond 2^24 could pass it.
template <bool BF16>
constexpr float kHeld = BF16 ? 0.f : 15.f;
template <bool BF16>
__device__ __forceinline__ float held_max(float x, float scale_log2) {
  const float m = __fmul_ru(x, scale_log2);
  return BF16 ? m : __fsub_ru(m, kHeld<BF16>);
}

// Four dims of a head's output, and with the first of them its log-sum-exp.
template <bool BF16, int D>
__device__ __forceinline__ void store_row(const DecodeArgs& a, int row, int head, int d, float m,
                                          float l, const float4& acc) {
  const float inv = l != 0.f ? 1.f / l : 0.f;
  *reinterpret_cast<uint2*>(a.out + row * a.ld_out + static_cast<int64_t>(head) * D + d) =
      make_uint2(pack2<BF16>(acc.x * inv, acc.y * inv), pack2<BF16>(acc.z * inv, acc.w * inv));
  if (d == 0 && a.lse)     // (the 15 go out of m and l first, without a rounding)
    a.lse[static_cast<int64_t>(row) * a.Hq + head] =
        l != 0.f ? (finite_max(m) + kHeld<BF16> + log2f(l * (BF16 ? 1.f : 0x1p-15f))) * kLn2
                 : -INFINITY;
}

constexpr int kMostCluster = 8;

// acc += f v, l += f l_v: products rounded before they are added, so that the
// two ways of joining items give the same bits.
__device__ __forceinline__ void add_scaled(float4& acc, float& l, const float4& v, float l_v, float f) {
  l = __fadd_rn(l, __fmul_rn(f, l_v));
  acc.x = __fadd_rn(acc.x, __fmul_rn(f, v.x));
  acc.y = __fadd_rn(acc.y, __fmul_rn(f, v.y));
  acc.z = __fadd_rn(acc.z, __fmul_rn(f, v.z));
  acc.w = __fadd_rn(acc.w, __fmul_rn(f, v.w));
}

constexpr int kWarps = 4, kThreads = kWarps * 32;
constexpr int kStep = 32;            // tokens of a warp's step: half a page

// WIDE: more than 8 query rows (the upper half of the tile is in use).  Fewer
// leave its exponentials out: 64 rows of 8192 tokens 162 us, with them 163.5;
// one row of 4000 6.2, with them 6.5.
template <bool BF16, int D, bool WIDE>
__global__ void __launch_bounds__(kThreads, D == 64 ? 3 : 2)
decode_attention_kernel(const DecodeArgs a) {
  constexpr int P = D + 8;           // row pitch: 8-byte stores of 8 rows x 4 lanes on distinct banks
  __shared__ alignas(16) float so[kWarps * kRows * P];   // the warps' parts
  __shared__ alignas(16) float s_item[kRows * D];        // in a cluster: this item's part
  __shared__ float2 s_ml[kWarps][kRows], s_item_ml[kRows];
  pdl_trigger();   // the joining kernel may take its place; it waits for this one's end
  const int row = blockIdx.z, head = blockIdx.y / a.tiles, tile = blockIdx.y % a.tiles;
  const int item = blockIdx.x;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
  const Span sp = find_span(a, row);
  const int items = (sp.pages + a.split - 1) / a.split;
  if (item >= items && item > 0) {
    if (a.cluster) {                     // the barriers below want every block
      cluster_sync_all();
      cluster_sync_all();
    }
    return;
  }
  const int h0 = head * a.G + tile * kRows;              // first query head of the block
  const int rows = min(kRows, a.G - tile * kRows);
  // this item's steps: the half pages of its pages that hold visible keys
  const int t0 = (sp.page0 + item * a.split) * 2;
  const int begin = max(t0, sp.lo / kStep);
  const int steps = max(0, min(t0 + 2 * a.split, (sp.n + kStep - 1) / kStep) - begin);
  const int cnt = steps > warp ? (steps - warp + kWarps - 1) / kWarps : 0;

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

  // The warp's j-th step is half page begin + warp + j * kWarps; lane l holds
  // the pool's page of j = 32 i + l.
  int ids = 0;
  const int k_lane = (8 * (g >> 1) + (g & 1)) * D + 8 * q, v_lane = g * kPageTokens + 8 * q;
  const uint16_t *k_at = nullptr, *v_at = nullptr;       // this lane's place in a step's K, V^T
  auto find_step = [&](int j) {
    if (j >= cnt) return;
    if (!(j & 31) && j + lane < cnt) ids = sp.table[(begin + warp + (j + lane) * kWarps) / 2];
    int page = __shfl_sync(0xFFFFFFFFu, ids, j & 31);
    if (page < 0 || page >= a.cache.n_pages) {
      if (lane == 0) atomicExch(a.err, kErrBounds);
      page = 0;
    }
    const int half = (begin + warp + j * kWarps) & 1;
    k_at = a.cache.block(page, 0, head, D) + half * kStep * D + k_lane;
    v_at = a.cache.block(page, 1, head, D) + half * kStep + v_lane;
  };
  constexpr int C = D / 32;          // 32-dim chunks of a K row
  uint4 k[4 * C], v[8];              // S tile i's chunk c; 8 rows of each of 8 V^T tiles
  auto load_k = [&](int j) {
    if (j >= cnt) return;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int c = 0; c < C; ++c) k[i * C + c] = load_once(k_at + 2 * i * D + 32 * c);
  };
  auto load_v = [&](int j) {
    if (j >= cnt) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = load_once(v_at + 8 * i * kPageTokens);
  };
  find_step(0);
  load_k(0);
  load_v(0);

  float o[D / 8][4];
#pragma unroll
  for (int i = 0; i < D / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
  float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f;
  for (int j = 0; j < cnt; ++j) {
    const int tok0 = (begin + warp + j * kWarps) * kStep;
    const bool edge = tok0 < sp.lo || tok0 + kStep > sp.n;
    // ---- S = Q K^T; column n of S tile i is token 8 (n/2) + 2 i + n%2
    float s[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i][0] = s[i][1] = s[i][2] = s[i][3] = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        mma16816<BF16>(s[i], qa[c][0], qb[c][0], qa[c][1], qb[c][1], k[i * C + c].x, k[i * C + c].y);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        mma16816<BF16>(s[i], qa[c][2], qb[c][2], qa[c][3], qb[c][3], k[i * C + c].z, k[i * C + c].w);
    }
    const uint16_t* v_now = v_at;
    find_step(j + 1);
    if constexpr (D == 64) {
      load_k(j + 1);
    } else {   // K's registers take the other dims' values first
#pragma unroll
      for (int i = 0; i < 8; ++i) k[i] = load_once(v_now + 8 * (8 + i) * kPageTokens);
    }
    // ---- softmax; this lane's columns 2q, 2q + 1 of tile i are tokens
    //      tok0 + 8 q + 2 i + {0, 1}
    if (edge) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int t = tok0 + 8 * q + 2 * i;
        if (t < sp.lo || t >= sp.n) s[i][0] = s[i][2] = -INFINITY;
        if (t + 1 < sp.lo || t + 1 >= sp.n) s[i][1] = s[i][3] = -INFINITY;
      }
    }
    float x0 = -INFINITY, x1 = -INFINITY;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x0 = fmaxf(x0, fmaxf(s[i][0], s[i][1]));
      if (WIDE) x1 = fmaxf(x1, fmaxf(s[i][2], s[i][3]));
    }
    x0 = fmaxf(x0, __shfl_xor_sync(0xFFFFFFFFu, x0, 1));
    x0 = fmaxf(x0, __shfl_xor_sync(0xFFFFFFFFu, x0, 2));
    if (WIDE) {
      x1 = fmaxf(x1, __shfl_xor_sync(0xFFFFFFFFu, x1, 1));
      x1 = fmaxf(x1, __shfl_xor_sync(0xFFFFFFFFu, x1, 2));
    }
    const float n0 = fmaxf(m0, held_max<BF16>(x0, a.scale_log2)),
                n1 = fmaxf(m1, held_max<BF16>(x1, a.scale_log2));
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
    uint32_t pa[4], pb[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
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
    auto multiply = [&](float (*acc)[4], uint4* x) {     // 8 tiles of 8 dims
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (edge) {          // what lies behind the mask may be anything, NaN too
          uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int t = tok0 + 8 * q + 2 * e;
            if (t < sp.lo || t >= sp.n) w[e] &= 0xFFFF0000u;
            if (t + 1 < sp.lo || t + 1 >= sp.n) w[e] &= 0x0000FFFFu;
          }
          x[i] = make_uint4(w[0], w[1], w[2], w[3]);
        }
#pragma unroll
      for (int i = 0; i < 8; ++i) mma16816<BF16>(acc[i], pa[0], pb[0], pa[1], pb[1], x[i].x, x[i].y);
#pragma unroll
      for (int i = 0; i < 8; ++i) mma16816<BF16>(acc[i], pa[2], pb[2], pa[3], pb[3], x[i].z, x[i].w);
    };
    multiply(o, v);
    load_v(j + 1);
    if constexpr (D == 128) {
      multiply(o + 8, k);
      load_k(j + 1);
    }
  }

  // ---- the warps' parts are joined, in warp order
  l0 += __shfl_xor_sync(0xFFFFFFFFu, l0, 1);
  l0 += __shfl_xor_sync(0xFFFFFFFFu, l0, 2);
  l1 += __shfl_xor_sync(0xFFFFFFFFu, l1, 1);
  l1 += __shfl_xor_sync(0xFFFFFFFFu, l1, 2);
  if (q == 0) {
    s_ml[warp][g] = make_float2(m0, l0);
    s_ml[warp][g + 8] = make_float2(m1, l1);
  }
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
  const int used = min(kWarps, steps);
  for (int e = threadIdx.x; e < rows * (D / 4); e += kThreads) {
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
    if (items <= 1) {
      store_row<BF16, D>(a, row, h0 + r, d, m, l, acc);
    } else if (a.cluster) {
      *reinterpret_cast<float4*>(s_item + r * D + d) = acc;
      if (d == 0) s_item_ml[r] = make_float2(m, l);
    } else {
      *reinterpret_cast<float4*>(a.part_o + (at * a.items + item) * D + d) = acc;
      if (d == 0) a.part_ml[at * a.items + item] = make_float2(m, l);
    }
  }
  if (!a.cluster) return;
  // ---- the items, in order: the row's values are dealt to the cluster's blocks
  __syncwarp();
  cluster_sync_all();
  if (items > 1) {
    const uint32_t o_at = smem_u32(s_item), ml_at = smem_u32(s_item_ml);
    for (int e = item * kThreads + threadIdx.x; e < rows * (D / 4); e += items * kThreads) {
      const int r = e / (D / 4), d = e % (D / 4) * 4;
      float2 ml[kMostCluster];
      float4 v[kMostCluster];
      float m = -INFINITY;
#pragma unroll
      for (int i = 0; i < kMostCluster; ++i)
        if (i < items) {
          ml[i] = ld_cluster_f32x2(cluster_map(ml_at + r * 8, i));
          v[i] = ld_cluster_f32x4(cluster_map(o_at + (r * D + d) * 4, i));
        }
#pragma unroll
      for (int i = 0; i < kMostCluster; ++i)
        if (i < items) m = fmaxf(m, ml[i].x);
      const float z = finite_max(m);
      float l = 0.f;
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int i = 0; i < kMostCluster; ++i)
        if (i < items) add_scaled(acc, l, v[i], ml[i].y, ex2(ml[i].x - z));
      store_row<BF16, D>(a, row, h0 + r, d, m, l, acc);
    }
  }
  __syncwarp();
  cluster_sync_all();                    // the peers have read this block's part
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
  pdl_wait();      // in every block: the grid ends after the first kernel's
  const Span sp = find_span(a, row);
  const int items = (sp.pages + a.split - 1) / a.split;
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
    add_scaled(acc, l, po[static_cast<int64_t>(i) * L + d], x.y, ex2(x.x - z));
  }
  s_acc[grp][d] = acc;
  if (d == 0) s_l[grp] = l;
  __syncthreads();
  if (grp > 0) return;
  for (int k = 1; k < NG; ++k) add_scaled(acc, l, s_acc[k][d], s_l[k], 1.f);
  store_row<BF16, D>(a, row, h, 4 * d, m, l, acc);
}

// Pages of an item when the caller leaves it open.  Few rows: one wave of blocks
// shares the cache evenly (of the 456 or 304 places that the GPU has for head
// dims 64 and 128, not all: one row of 131,001 tokens takes 48 us on 256 blocks
// and 53 on 304), or eight items that join in a cluster where that is not long.
// (Measured on tables as wide as the row, one shape for each head dim.)
// More than one row, which may differ in length: items of at most kMostPages, so
// that the tail behind the longest is short (32 rows of 1024 to 6144 tokens: 43
// us with 12 pages, 47 with 32, 49 with 4).
constexpr int64_t wave_of(int head_dim) { return head_dim == 64 ? 320 : 256; }
constexpr int kMostPages = 12;
int auto_split(int pages, int rows, int64_t blocks_per_item, int head_dim) {
  const int64_t wave = wave_of(head_dim) / blocks_per_item;
  int64_t items = wave < 1 ? 1 : wave;
  if (items > kMostCluster && pages <= 8 * kMostCluster) items = kMostCluster;
  int64_t split = (pages + items - 1) / items;
  if (split < 2) split = 2;
  if (split > kMostPages && rows > 1) split = kMostPages;
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
  p.split = split_pages > 0 ? std::min(split_pages, c.pt_stride)
                            : auto_split(pages, rows, static_cast<int64_t>(rows < 1 ? 1 : rows) *
                                                          c.n_kv_heads * p.tiles,
                                         c.head_dim);
  p.items = (pages + p.split - 1) / p.split;
  return p;
}

template <bool BF16, int D>
cudaError_t launch_decode(const DecodeArgs& a, int rows, cudaStream_t s) {
  auto kernel = a.G > 8 ? decode_attention_kernel<BF16, D, true> : decode_attention_kernel<BF16, D, false>;
  cudaError_t e = launch_ex(kernel, dim3(a.items, a.cache.Hkv * a.tiles, rows), dim3(kThreads), 0, s,
                            false, dim3(a.cluster ? a.items : 1, 1, 1), a);
  if (e != cudaSuccess || a.items == 1 || a.cluster) return e;
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
  return rows >= 0 && n_heads >= 1 && n_heads < (1 << 16) && n_heads % c->n_kv_heads == 0 &&
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
  // items are at most one wave's share, a cluster, or pages / kMostPages, and
  // the rounding.
  size_t items = p.items;
  if (split_pages == 0) {
    const int64_t blocks = static_cast<int64_t>(rows < 1 ? 1 : rows) * cache->n_kv_heads * p.tiles;
    const size_t wave = static_cast<size_t>(wave_of(cache->head_dim) / blocks),
                 cut = cache->pt_stride / kMostPages, cluster = kMostCluster;
    items = std::max(std::max(wave, cut), cluster) + 2;
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
  if (!aligned4(seq, n, lse)) return GS_ERR_INVALID_ARG;
  if (rows > 65535) return GS_ERR_UNSUPPORTED;
  if (window >= cache->pt_stride * kPageTokens) window = 0;   // no row is longer
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
  // Up to eight items of one wave join within a cluster (one launch, no trip
  // through memory: 517 tokens 4.4 us, through the scratch 5.6; 8 rows of 2000
  // 9.5 and 11.0); more items, or more blocks, through the scratch.
  a.cluster = p.items > 1 && p.items <= kMostCluster &&
              static_cast<int64_t>(p.items) * cache->n_kv_heads * p.tiles * rows <= wave_of(D);
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
