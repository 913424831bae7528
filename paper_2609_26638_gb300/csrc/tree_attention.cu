// tree_attention.cu -- attention of the nodes of a drafted tree over the paged
// cache, split over the cache's length and joined.
//
//   s_ij = scale * q_i . k_j over the keys that node i sees: the cached ones
//          (the window's, where there is one) and the nodes of its mask
//   o_i = sum_j 2^(s'_ij - m_i) v_j / l_i,  l_i = sum_j 2^(s'_ij - m_i)
//
// (s' = s log2(e), m the running maximum, 15 less in fp16; see weights_of.)  A query row is one
// query head of one node.  Up to 16 rows of a KV head, node by node, are one tile of the
// narrow kernel below, more are tiles of 128 for the one in tree_wide.cuh (fp16, 16 / 8
// heads of 64, 32 trees of 1024 to 6144 tokens: 16 rows 50 us here; 32 and 48 rows 77 and
// 104 us with two and three tiles to a warp here, for want of registers, 57 and 62 there).
//
// A narrow block takes one KV head and one item of `split` pages; its warps take
// the item's half pages in turn, straight from global memory into the operand
// registers of m16n8k16 instructions, and are joined at the item's end.  Every byte of
// the cache is read once, and bounds it.
//
// P is rounded to the cache's type for the product with V, as the output is, and the sums are
// not: the reasons, and what that loses, are gs_decode_attention's.
//
// Only steps that reach the tree's nodes, or a window's start, look at masks: a row's
// view of the step's 32 tokens is one word, the cached range or'ed with its
// mask shifted into place.  A masked score is replaced by -inf.  A value that no row
// of the tile sees is cleared; one that some rows see is multiplied as it is, and
// where it is not finite (0 times it would be NaN for the others) by itself, for the rows
// that see it.
#include <algorithm>
#include <cmath>

#include "internal.h"
#include "tree_wide.cuh"

namespace gs {
namespace {

// A tree's numbers, the first key that any of its nodes sees and the first that
// all see, that key's page and the pages from there on.
struct Span {
  int n, keys, count, lo, lo_most, page0, pages;
  const int32_t* table;
};
// They are read by one warp for its block: all threads go through the same pages
// and barriers whatever happens to the arrays meanwhile.
__device__ __forceinline__ Span find_span(const TreeArgs& a, int tree) {
  __shared__ int s_v[6];
  if (threadIdx.x < 32) {
    const TreeNums t = read_tree(a, tree);
    int lo = a.window > 0 ? t.n : 0, lo_most = 0;
    if (a.window > 0) {
      for (int i = threadIdx.x; i < t.count; i += 32) {
        const int x = first_key(a.pos[static_cast<int64_t>(tree) * a.nodes + i], t.n, a.window);
        lo = min(lo, x);
        lo_most = max(lo_most, x);
      }
      lo = __reduce_min_sync(0xFFFFFFFFu, lo);
      lo_most = __reduce_max_sync(0xFFFFFFFFu, lo_most);
    }
    if (threadIdx.x == 0) {
      if (t.bad) atomicExch(a.err, kErrBounds);
      s_v[0] = t.seq, s_v[1] = t.n, s_v[2] = t.keys, s_v[3] = t.count, s_v[4] = lo, s_v[5] = lo_most;
    }
  }
  __syncthreads();
  Span s;
  s.n = s_v[1];
  s.keys = s_v[2];
  s.count = s_v[3];
  s.lo = s_v[4];
  s.lo_most = s_v[5];
  s.page0 = s.lo / kPageTokens;
  s.pages = max(0, (s.keys + kPageTokens - 1) / kPageTokens - s.page0);
  s.table = a.cache.page_table + static_cast<int64_t>(s_v[0]) * a.cache.pt_stride;
  return s;
}

constexpr int kWarps = 4, kThreads = kWarps * 32;
constexpr int kStep = 32;            // tokens of a warp's step: half a page

template <int D>
struct Smem {
  static constexpr int R = 16, P = D + 8;   // row pitch: 8 rows x 4 lanes on distinct banks
  alignas(16) float so[kWarps * 16 * P];         // the warps' parts of 16 rows
  alignas(16) float item[R * D];                 // in a cluster: this item's part
  float2 ml[kWarps][R], item_ml[R];
  uint64_t mask[R];
  int lo[R];
};

template <bool BF16, int D>
__global__ void __launch_bounds__(kThreads, D == 64 ? 3 : 2)
tree_attention_kernel(const TreeArgs a) {
  constexpr int R = Smem<D>::R, P = Smem<D>::P, C = D / 32;
  extern __shared__ __align__(16) uint8_t smem_raw[];
  Smem<D>& sm = *reinterpret_cast<Smem<D>*>(smem_raw);
  pdl_trigger();   // the joining kernel may take its place; it waits for this one's end
  const int tree = blockIdx.z, head = blockIdx.y, item = blockIdx.x;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
  const Span sp = find_span(a, tree);
  const int items = (sp.pages + a.split - 1) / a.split;
  const int rows = sp.count * a.G;       // query rows, at most R
  if (item == 0 && blockIdx.y == 0 && threadIdx.x == 0)
    a.part_n[tree] = TreePart{0, sp.pages, sp.count};
  if (rows <= 0 || (item >= items && item > 0)) {
    if (a.cluster) {                     // the barriers below want every block
      cluster_sync_all();
      cluster_sync_all();
    }
    return;
  }
  const int64_t row0 = static_cast<int64_t>(tree) * a.nodes;   // the tree's first row
  auto node_of = [&](int r) { return r / a.G; };
  auto q_head = [&](int r) { return head * a.G + r % a.G; };
  auto q_at = [&](int r) {
    return a.q + (row0 + node_of(r)) * a.ld_q + static_cast<int64_t>(q_head(r)) * D;
  };
  // this item's steps: the half pages of its pages that hold visible keys
  const int t0 = (sp.page0 + item * a.split) * 2;
  const int begin = max(t0, sp.lo / kStep);
  const int steps = max(0, min(t0 + 2 * a.split, (sp.keys + kStep - 1) / kStep) - begin);
  const int cnt = steps > warp ? (steps - warp + kWarps - 1) / kWarps : 0;

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

  // each row's mask and first key, and Q in the operand's order: of each 32
  // dims, dims 8q .. 8q + 7 on lane q
  if (const int r = threadIdx.x; r < R) {
    uint64_t mask = 0;
    int lo = sp.n;
    if (r < rows) {
      const int node = node_of(r);
      mask = a.mask[row0 + node];
      if (sp.keys - sp.n < 64) mask &= (1ull << (sp.keys - sp.n)) - 1;
      lo = a.window > 0 ? min(max(first_key(a.pos[row0 + node], sp.n, a.window), sp.lo), sp.lo_most)
                        : 0;
    }
    sm.mask[r] = mask;
    sm.lo[r] = lo;
  }
  uint32_t qa[C][4], qb[C][4];
  const uint4 zero4 = make_uint4(0, 0, 0, 0);
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const uint4 u = g < rows ? *reinterpret_cast<const uint4*>(q_at(g) + 8 * q + 32 * c) : zero4;
    const uint4 w =
        g + 8 < rows ? *reinterpret_cast<const uint4*>(q_at(g + 8) + 8 * q + 32 * c) : zero4;
    qa[c][0] = u.x, qa[c][1] = u.y, qa[c][2] = u.z, qa[c][3] = u.w;
    qb[c][0] = w.x, qb[c][1] = w.y, qb[c][2] = w.z, qb[c][3] = w.w;
  }
  __syncthreads();

  float o[D / 8][4];
#pragma unroll
  for (int i = 0; i < D / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
  float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f;
  for (int j = 0; j < cnt; ++j) {
    const int tok0 = (begin + warp + j * kWarps) * kStep;
    const bool edge = tok0 < sp.lo_most || tok0 + kStep > sp.n;
    uint32_t some = 0u, all = 0xFFFFFFFFu;               // tokens that some row, every row sees
    uint32_t pa[4], pb[4];
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
    // ---- softmax; this lane's columns 2q, 2q + 1 of tile i are tokens
    //      tok0 + 8 q + 2 i + {0, 1}
    if (edge) {
      const uint32_t v0 = row_view(sm.mask[g], sm.lo[g], sp.n, tok0),
                     v1 = row_view(sm.mask[g + 8], sm.lo[g + 8], sp.n, tok0);
      if (g < rows) some |= v0, all &= v0;
      if (g + 8 < rows) some |= v1, all &= v1;
      const uint32_t w0 = v0 >> (8 * q), w1 = v1 >> (8 * q);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (!((w0 >> (2 * i)) & 1)) s[i][0] = -INFINITY;
        if (!((w0 >> (2 * i + 1)) & 1)) s[i][1] = -INFINITY;
        if (!((w1 >> (2 * i)) & 1)) s[i][2] = -INFINITY;
        if (!((w1 >> (2 * i + 1)) & 1)) s[i][3] = -INFINITY;
      }
    }
    float x0 = -INFINITY, x1 = -INFINITY;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x0 = fmaxf(x0, fmaxf(s[i][0], s[i][1]));
      x1 = fmaxf(x1, fmaxf(s[i][2], s[i][3]));
    }
    x0 = fmaxf(x0, __shfl_xor_sync(0xFFFFFFFFu, x0, 1));
    x0 = fmaxf(x0, __shfl_xor_sync(0xFFFFFFFFu, x0, 2));
    x1 = fmaxf(x1, __shfl_xor_sync(0xFFFFFFFFu, x1, 1));
    x1 = fmaxf(x1, __shfl_xor_sync(0xFFFFFFFFu, x1, 2));
    const float n0 = fmaxf(m0, x0), n1 = fmaxf(m1, x1);
    if (__any_sync(0xFFFFFFFFu, n0 != m0 || n1 != m1)) {
      const float f0 = moved_max(m0, finite_max(n0), a.scale_log2),
                  f1 = moved_max(m1, finite_max(n1), a.scale_log2);
      l0 *= f0;
      l1 *= f1;
#pragma unroll
      for (int i = 0; i < D / 8; ++i) {
        o[i][0] *= f0;
        o[i][1] *= f0;
        o[i][2] *= f1;
        o[i][3] *= f1;
      }
      m0 = n0;
      m1 = n1;
    }
    const float z0 = finite_max(m0), z1 = finite_max(m1);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 u = weights_of<BF16>(s[i][0], s[i][1], z0, a.scale_log2),
                   w = weights_of<BF16>(s[i][2], s[i][3], z1, a.scale_log2);
      l0 += u.x + u.y;
      l1 += w.x + w.y;
      pa[i] = pack2<BF16>(u.x, u.y);
      pb[i] = pack2<BF16>(w.x, w.y);
    }
    const uint16_t* v_now = v_at;
    find_step(j + 1);
    if constexpr (D == 64) {
      load_k(j + 1);
    } else {   // K's registers take the other dims' values first
#pragma unroll
      for (int i = 0; i < 8; ++i) k[i] = load_once(v_now + 8 * (8 + i) * kPageTokens);
    }
    // ---- O += P V, 8 tiles of 8 dims at a time
    if (edge) {
      some = __reduce_or_sync(0xFFFFFFFFu, some);
      all = __reduce_and_sync(0xFFFFFFFFu, all);
    }
    auto multiply = [&](int i0, uint4* x) {
      uint32_t odd = 0u;         // tokens with a value that is not finite, seen by some rows only
      if (edge) {
        const uint32_t keep = some >> (8 * q), part = (some & ~all) >> (8 * q);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if (!((keep >> (2 * e)) & 1)) w[e] &= 0xFFFF0000u;
            if (!((keep >> (2 * e + 1)) & 1)) w[e] &= 0x0000FFFFu;
            if (not_finite<BF16>(w[e])) odd |= ((part >> (2 * e)) & 3u) << (8 * q + 2 * e);
          }
          x[i] = make_uint4(w[0], w[1], w[2], w[3]);
        }
        odd = __reduce_or_sync(0xFFFFFFFFu, odd);
      }
      for (uint32_t left = odd; left; left &= left - 1) {
        const int tok = __ffs(left) - 1;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
          uint32_t one[4] = {0u, 0u, 0u, 0u};
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (tok >> 1 == 4 * q + e) {
              const uint32_t sel = not_finite<BF16>(w[e]) & (tok & 1 ? 0xFFFF0000u : 0x0000FFFFu);
              one[e] = w[e] & sel;
              w[e] &= ~sel;
            }
          x[i] = make_uint4(w[0], w[1], w[2], w[3]);
          float p[4] = {0.f, 0.f, 0.f, 0.f};
          mma16816<BF16>(p, pa[0], pb[0], pa[1], pb[1], one[0], one[1]);
          mma16816<BF16>(p, pa[2], pb[2], pa[3], pb[3], one[2], one[3]);
          if ((row_view(sm.mask[g], sm.lo[g], sp.n, tok0) >> tok) & 1)
            o[i0 + i][0] += p[0], o[i0 + i][1] += p[1];
          if ((row_view(sm.mask[g + 8], sm.lo[g + 8], sp.n, tok0) >> tok) & 1)
            o[i0 + i][2] += p[2], o[i0 + i][3] += p[3];
        }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i)
        mma16816<BF16>(o[i0 + i], pa[0], pb[0], pa[1], pb[1], x[i].x, x[i].y);
#pragma unroll
      for (int i = 0; i < 8; ++i)
        mma16816<BF16>(o[i0 + i], pa[2], pb[2], pa[3], pb[3], x[i].z, x[i].w);
    };
    multiply(0, v);
    load_v(j + 1);
    if constexpr (D == 128) {
      multiply(8, k);
      load_k(j + 1);
    }
  }

  // ---- the warps' parts are joined, in warp order
  l0 += __shfl_xor_sync(0xFFFFFFFFu, l0, 1);
  l0 += __shfl_xor_sync(0xFFFFFFFFu, l0, 2);
  l1 += __shfl_xor_sync(0xFFFFFFFFu, l1, 1);
  l1 += __shfl_xor_sync(0xFFFFFFFFu, l1, 2);
  if (q == 0) {
    sm.ml[warp][g] = make_float2(m0, l0);
    sm.ml[warp][g + 8] = make_float2(m1, l1);
  }
  const int used = min(kWarps, steps);
  if (cnt > 0) {
#pragma unroll
    for (int i = 0; i < D / 8; ++i) {
      *reinterpret_cast<float2*>(sm.so + (warp * 16 + g) * P + 8 * i + 2 * q) =
          make_float2(o[i][0], o[i][1]);
      *reinterpret_cast<float2*>(sm.so + (warp * 16 + g + 8) * P + 8 * i + 2 * q) =
          make_float2(o[i][2], o[i][3]);
    }
  }
  __syncthreads();
  for (int e = threadIdx.x; e < rows * (D / 4); e += kThreads) {
    const int r = e / (D / 4), d = e % (D / 4) * 4;
    float m = -INFINITY, l = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int w = 0; w < used; ++w) m = fmaxf(m, sm.ml[w][r].x);
    const float z = finite_max(m);
    for (int w = 0; w < used; ++w) {
      const float f = moved_max(sm.ml[w][r].x, z, a.scale_log2);
      const float4 x = *reinterpret_cast<const float4*>(sm.so + (w * 16 + r) * P + d);
      l = fmaf(f, sm.ml[w][r].y, l);
      acc.x = fmaf(f, x.x, acc.x);
      acc.y = fmaf(f, x.y, acc.y);
      acc.z = fmaf(f, x.z, acc.z);
      acc.w = fmaf(f, x.w, acc.w);
    }
    const int64_t row = row0 + node_of(r);
    if (items <= 1) {
      store_row<BF16, D>(a, row, q_head(r), d, m, l, acc);
    } else if (a.cluster) {
      *reinterpret_cast<float4*>(sm.item + r * D + d) = acc;
      if (d == 0) sm.item_ml[r] = make_float2(m, l);
    } else {
      const int64_t at = row * a.Hq + q_head(r);
      *reinterpret_cast<float4*>(a.part_o + (at * a.items + item) * D + d) = acc;
      if (d == 0) a.part_ml[at * a.items + item] = make_float2(m, l);
    }
  }
  if (!a.cluster) return;
  // ---- the items, in order: the tile's values are dealt to the cluster's blocks
  __syncwarp();
  cluster_sync_all();
  if (items > 1) {
    const uint32_t o_at = smem_u32(sm.item), ml_at = smem_u32(sm.item_ml);
    for (int e = item * kThreads + threadIdx.x; e < rows * (D / 4); e += items * kThreads) {
      const int r = e / (D / 4), d = e % (D / 4) * 4;
      float2 ml[kMostCluster];
      float4 x[kMostCluster];
      float m = -INFINITY;
#pragma unroll
      for (int i = 0; i < kMostCluster; ++i)
        if (i < items) {
          ml[i] = ld_cluster_f32x2(cluster_map(ml_at + r * 8, i));
          x[i] = ld_cluster_f32x4(cluster_map(o_at + (r * D + d) * 4, i));
        }
#pragma unroll
      for (int i = 0; i < kMostCluster; ++i)
        if (i < items) m = fmaxf(m, ml[i].x);
      const float z = finite_max(m);
      float l = 0.f;
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int i = 0; i < kMostCluster; ++i)
        if (i < items) add_scaled(acc, l, x[i], ml[i].y, moved_max(ml[i].x, z, a.scale_log2));
      store_row<BF16, D>(a, row0 + node_of(r), q_head(r), d, m, l, acc);
    }
  }
  __syncwarp();
  cluster_sync_all();                    // the peers have read this block's part
}

// Joins the parts of each row and head, a thread per four dims.  Eight parts
// in order make a chunk, the chunks are added in order: however many thread groups
// share a row's chunks, the sums are the same.  (A cluster's items are one chunk.)
constexpr int kJoinThreads = 256;

__device__ __forceinline__ int block_max(int v) {
  __shared__ int s_max;
  if (threadIdx.x == 0) s_max = 0;
  __syncthreads();
  if (v > 0) atomicMax(&s_max, v);
  __syncthreads();
  return s_max;
}

template <bool BF16, int D>
__global__ void __launch_bounds__(kJoinThreads, 4)
tree_join_kernel(const TreeArgs a, int groups, int64_t rows, int team) {
  constexpr int L = D / 4, NG = kJoinThreads / L;
  __shared__ float4 s_acc[NG][L];
  __shared__ float s_l[NG];
  const int grp = threadIdx.x / L, d = threadIdx.x % L, sub = grp % groups;
  const int64_t at = static_cast<int64_t>(blockIdx.x) * (NG / groups) + grp / groups;   // row, head
  const bool in = at < rows * a.Hq;
  const int64_t row = in ? at / a.Hq : 0;
  const int tree = static_cast<int>(row / a.nodes), node = static_cast<int>(row % a.nodes);
  const int head = static_cast<int>(at % a.Hq);
  pdl_wait();      // in every block: the grid ends after the first kernel's
  const TreePart have = a.part_n[tree];
  // part i lies at first + (i > 0 ? more : 0) + i * step
  int parts = 0;
  int64_t first = at * a.items, more = 0, step = 1;
  if (in && node < have.count) {
    if (a.items > 0) {
      parts = (have.pages + a.split - 1) / a.split;
    } else {       // the blocks that share this tile's pages
      const int64_t total = a.part_all[0], blocks = a.part_all[1];
      const int r = node * a.G + head % a.G, tile = r / kWideRows;
      const int tiles = (have.count * a.G + kWideRows - 1) / kWideRows;
      const int64_t u = have.first + static_cast<int64_t>(head / a.G * ((tiles + team - 1) / team) +
                                                          tile / team) * have.pages;
      const int64_t b0 = ((u + 1) * blocks - 1) / total,
                    b1 = ((u + have.pages) * blocks - 1) / total;
      parts = static_cast<int>(b1 - b0) + 1;
      first = ((2 * b0 + 1) * team + tile % team) * kWideRows + r % kWideRows;
      more = -static_cast<int64_t>(team) * kWideRows;
      step = 2ll * team * kWideRows;
    }
  }
  auto part_at = [&](int i) { return first + (i > 0 ? more : 0) + i * step; };
  float m = -INFINITY;
  for (int i = d; i < parts; i += L) m = fmaxf(m, a.part_ml[part_at(i)].x);
#pragma unroll
  for (int x = L / 2; x; x >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, x));
  const float z = finite_max(m), scale_log2 = a.scale_log2;
  const float4* po = reinterpret_cast<const float4*>(a.part_o) + d;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  float l = 0.f;
  // (with several groups to a row, all of the block go through the same rounds)
  const int rounds = groups > 1 ? block_max((parts + 8 * groups - 1) / (8 * groups)) : (parts + 7) / 8;
  for (int round = 0; round < rounds; ++round) {
    const int first_of = (round * groups + sub) * 8;
    float4 part = make_float4(0.f, 0.f, 0.f, 0.f);
    float pl = 0.f;
#pragma unroll
    for (int h = 0; h < 8; h += 4) {
      float4 v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (first_of + h + i < parts) v[i] = po[part_at(first_of + h + i) * L];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (first_of + h + i < parts) {
          const float2 x = a.part_ml[part_at(first_of + h + i)];
          add_scaled(part, pl, v[i], x.y, moved_max(x.x, z, scale_log2));
        }
    }
    if (groups == 1) {
      add_scaled(acc, l, part, pl, 1.f);
      continue;
    }
    s_acc[grp][d] = part;
    if (d == 0) s_l[grp] = pl;
    __syncthreads();
    if (sub == 0)
      for (int i = 0; i < groups && first_of + 8 * i < parts; ++i)
        add_scaled(acc, l, s_acc[grp + i][d], s_l[grp + i], 1.f);
    __syncthreads();
  }
  if (sub == 0 && parts > 1) store_row<BF16, D>(a, row, head, 4 * d, m, l, acc);
}

// Pages of an item of the narrow kernel when the caller leaves it open.  One tree: one
// wave of blocks shares the cache evenly, or eight items that join in a cluster where that is
// not long.  Several trees, which may differ in length: items of at most 16 pages, so
// that the tail behind the longest is short, or 32 where the trees' heads alone fill the
// GPU, as every part of 16 rows is written and read again.  The host does not know the
// lengths, and no cap is the best for all; us by pages of an item, the choice with a star:
//   tokens            nodes, heads            12     16     24     32     48     64
//   32 x 1024-6144    4, 16 / 8 x 64, fp16    45.8   46.7*  47.2   49.3   44.8   51.8
//   the same          8                       49.5   50.1*  49.5   52.1   46.6   53.1
//   16 x 100-6144     5                       30.4   25.9*  26.5   29.7   36.7   42.4
//   4 x 20,000        8                       37.0   39.3*  33.2   33.7   37.0   44.5
//   64 x 8192         8                       191    184    171    170*   172    178
//   48 x 1024-6144    4, 16 / 4 x 128, bf16   84.1   80.8*  76.0   86.6   75.8   83.7
//   16 x 1024-6144    4, 32 / 8 x 128, bf16   61.4   56.4*  62.7   50.8   63.7   76.8
// (up to 18 per cent from the best: a caller who knows the lengths can give a split).
constexpr int64_t wave_of(int head_dim) { return head_dim == 64 ? 320 : 256; }
constexpr int kMostPages = 16;
int auto_split(int pages, int trees, int64_t blocks_per_item, int head_dim) {
  const int64_t wave = wave_of(head_dim) / blocks_per_item;
  int64_t items = wave < 1 ? 1 : wave;
  if (items > kMostCluster && pages <= 8 * kMostCluster) items = kMostCluster;
  int64_t split = (pages + items - 1) / items;
  if (split < 2) split = 2;
  if (trees > 1) split = std::min<int64_t>(split, wave < 1 ? 2 * kMostPages : kMostPages);
  return static_cast<int>(split < pages ? split : pages);
}

constexpr int kNarrowRows = 16;    // of a KV head; more are the wide kernel's

struct Plan {
  bool wide, shared;             // shared: the wide kernel's blocks share all pages
  int tiles, split, items;
};
Plan plan_tree(const gs_cache& c, int trees, int nodes, int n_heads, int window, int split_pages) {
  Plan p;
  const int G = n_heads / c.n_kv_heads;
  p.wide = nodes * G > kNarrowRows;
  p.tiles = p.wide ? (nodes * G + kWideRows - 1) / kWideRows : 1;
  p.shared = p.wide && split_pages == 0 && trees <= kMostShared;
  p.split = p.items = 0;
  if (p.shared) return p;
  int pages = c.pt_stride;
  if (window > 0) {
    const int64_t most = (static_cast<int64_t>(window) - 1 + nodes + kPageTokens - 2) / kPageTokens + 1;
    if (most < pages) pages = static_cast<int>(most);
  }
  const int64_t blocks = static_cast<int64_t>(trees < 1 ? 1 : trees) * c.n_kv_heads;
  p.split = split_pages > 0 ? std::min(split_pages, c.pt_stride)
            : p.wide        ? pages          // (many trees: a block for each tile)
                            : auto_split(pages, trees, blocks, c.head_dim);
  p.items = (pages + p.split - 1) / p.split;
  return p;
}

constexpr int kWideBlocks = 2 * kNumSMs;
constexpr int kMostTeam = 8;

template <bool BF16, int D>
cudaError_t launch_tree(const gs_cache& c, const TreeArgs& a, bool wide, int trees, cudaStream_t s) {
  static DeviceOnce once;
  auto narrow = tree_attention_kernel<BF16, D>;
  auto broad = tree_wide_kernel<BF16, D>;
  constexpr size_t smem = sizeof(Smem<D>), wide_smem = WideSmem<D>::total;
  cudaError_t e = once.run([&] {
    const cudaError_t r = cudaFuncSetAttribute(narrow, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    return r != cudaSuccess ? r
                            : cudaFuncSetAttribute(broad, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                   wide_smem);
  });
  if (e != cudaSuccess) return e;
  const dim3 grid(a.items, a.cache.Hkv * a.tiles, trees);
  // blocks of a team: as even a division of the tiles as kMostTeam allows
  const int teams = (a.tiles + kMostTeam - 1) / kMostTeam, team = (a.tiles + teams - 1) / teams;
  if (wide) {
    CUtensorMap k, v;
    if (!pool_maps(c, &k, &v)) return cudaErrorUnknown;
    e = launch_ex(broad, a.items ? grid : dim3(kWideBlocks / team * team), dim3(kWideThreads), wide_smem,
                  s, false, dim3(1, 1, 1), k, v, a, trees, team);
  } else {
    e = launch_ex(narrow, grid, dim3(kThreads), smem, s, false, dim3(a.cluster ? a.items : 1, 1, 1), a);
  }
  if (e != cudaSuccess || a.items == 1 || a.cluster) return e;
  // a row's chunks are shared by as many groups as the GPU has room for
  constexpr int NG = kJoinThreads / (D / 4);
  const int64_t rows = static_cast<int64_t>(trees) * a.nodes;
  const int64_t most = a.items ? a.items : kWideBlocks / (static_cast<int64_t>(trees) * a.cache.Hkv * teams * team) + 2;
  int groups = 1;
  while (groups < NG && groups * 8 < most && rows * a.Hq * groups < kNumSMs * 4 * NG) groups *= 2;
  const int64_t blocks = (rows * a.Hq * groups + NG - 1) / NG;
  return launch_ex(tree_join_kernel<BF16, D>, dim3(static_cast<unsigned>(blocks)), dim3(kJoinThreads),
                   0, s, true, dim3(1, 1, 1), a, groups, rows, team);
}

size_t up256(size_t x) { return (x + 255) / 256 * 256; }

struct Scratch {         // offsets of the trees' sizes, the partial accumulators, their (max, sum)
  size_t n, o, ml, total;
};
// Parts: one per row, head and item; two tiles per block where the blocks share the pages.
Scratch scratch_of(const gs_cache& c, int trees, int nodes, int n_heads, bool shared, size_t items) {
  const size_t rows = shared ? 2ull * kWideBlocks * kWideRows
                             : static_cast<size_t>(trees) * nodes * n_heads * items;
  Scratch s;
  s.n = kErrBytes;
  s.o = s.n + up256(16 + trees * sizeof(TreePart));
  s.ml = s.o + up256(rows * c.head_dim * sizeof(float));
  s.total = s.ml + up256(rows * sizeof(float2));
  return s;
}

// GS_OK, or what is wrong with the sizes of a call.
int check_sizes(const gs_cache* c, int trees, int nodes, int n_heads, int split_pages) {
  if (const int rc = check_cache(c)) return rc;
  if (trees < 0 || nodes < 1 || n_heads < 1 || n_heads % c->n_kv_heads || split_pages < 0)
    return GS_ERR_INVALID_ARG;
  // trees and heads' tiles are grid dimensions
  if (nodes > kMostNodes || trees > 65535 || n_heads >= (1 << 14)) return GS_ERR_UNSUPPORTED;
  return GS_OK;
}

}  // namespace
}  // namespace gs

extern "C" size_t gs_tree_attention_scratch_bytes(const gs_cache* cache, int trees, int nodes,
                                                  int n_heads, int split_pages) {
  using namespace gs;
  if (check_sizes(cache, trees, nodes, n_heads, split_pages) != GS_OK) return 0;
  const Plan p = plan_tree(*cache, trees, nodes, n_heads, 0, split_pages);
  // An open split of the narrow kernel follows the pages that a window leaves:
  // whatever it is, the items are at most one wave's share, a cluster, or pages /
  // kMostPages, and the rounding.
  size_t items = p.items;
  if (split_pages == 0 && !p.wide) {
    const int64_t blocks = static_cast<int64_t>(trees < 1 ? 1 : trees) * cache->n_kv_heads;
    const size_t wave = static_cast<size_t>(wave_of(cache->head_dim) / blocks),
                 cut = cache->pt_stride / kMostPages, cluster = kMostCluster;
    items = std::max(std::max(wave, cut), cluster) + 2;
    if (items > static_cast<size_t>(cache->pt_stride)) items = cache->pt_stride;
  }
  return scratch_of(*cache, trees, nodes, n_heads, p.shared, items).total;
}

extern "C" int gs_tree_attention(const gs_cache* cache, const void* q, int64_t ld_q,
                                 const int32_t* seq, const int32_t* n, const int32_t* count,
                                 const uint64_t* mask, const int32_t* pos, int trees, int nodes,
                                 int n_heads, float scale, int window, void* out, int64_t ld_out,
                                 float* lse, int split_pages, void* scratch, size_t scratch_bytes,
                                 void* stream) {
  using namespace gs;
  if (const int rc = check_sizes(cache, trees, nodes, n_heads, split_pages)) return rc;
  if (!q || !n || !mask || !out || !scratch || window < 0 || (window > 0 && !pos) ||
      !(scale > 0.f) || !std::isfinite(scale))
    return GS_ERR_INVALID_ARG;
  const int D = cache->head_dim;
  const int64_t width = static_cast<int64_t>(n_heads) * D;
  if (ld_q < width || ld_out < width || ld_q % 8 || ld_out % 8 || !aligned16(q) || !aligned16(out) ||
      (reinterpret_cast<uintptr_t>(scratch) & 255) || (reinterpret_cast<uintptr_t>(mask) & 7))
    return GS_ERR_INVALID_ARG;
  if (!aligned4(seq, n, count, pos, lse)) return GS_ERR_INVALID_ARG;
  if (scratch_bytes < gs_tree_attention_scratch_bytes(cache, trees, nodes, n_heads, split_pages))
    return GS_ERR_OOM;
  if (trees == 0) return GS_OK;
  const Plan p = plan_tree(*cache, trees, nodes, n_heads, window, split_pages);
  const Scratch sc = scratch_of(*cache, trees, nodes, n_heads, p.shared, p.items);
  uint8_t* base = static_cast<uint8_t*>(scratch);
  TreeArgs a;
  a.q = static_cast<const uint16_t*>(q);
  a.ld_q = ld_q;
  a.seq = seq;
  a.n = n;
  a.count = count;
  a.pos = pos;
  a.mask = mask;
  a.out = static_cast<uint16_t*>(out);
  a.ld_out = ld_out;
  a.lse = lse;
  a.Hq = n_heads;
  a.G = n_heads / cache->n_kv_heads;
  a.nodes = nodes;
  a.tiles = p.tiles;
  a.window = window;
  a.split = p.split;
  a.items = p.items;
  a.cluster = !p.wide && p.items > 1 && p.items <= kMostCluster &&
              static_cast<int64_t>(p.items) * cache->n_kv_heads * trees <= wave_of(D);
  a.scale_log2 = scale * kLog2e;
  a.light = std::exp2(-(cache->dtype == GS_BF16 ? 0.f : p.wide ? kSet<false> : kHeld<false>));
  a.part_o = reinterpret_cast<float*>(base + sc.o);
  a.part_ml = reinterpret_cast<float2*>(base + sc.ml);
  a.part_all = reinterpret_cast<int64_t*>(base + sc.n);
  a.part_n = reinterpret_cast<TreePart*>(base + sc.n + 16);
  a.err = static_cast<int*>(scratch);
  a.cache = cache_view(*cache);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e;
  if (cache->dtype == GS_BF16)
    e = D == 64 ? launch_tree<true, 64>(*cache, a, p.wide, trees, s)
                : launch_tree<true, 128>(*cache, a, p.wide, trees, s);
  else
    e = D == 64 ? launch_tree<false, 64>(*cache, a, p.wide, trees, s)
                : launch_tree<false, 128>(*cache, a, p.wide, trees, s);
  return e == cudaSuccess ? GS_OK : GS_ERR_CUDA;
}
