// tree_common.cuh -- the tree attentions' arguments, a tree's numbers and masks,
// and the end of a row.
#pragma once
#include "attend_common.cuh"

namespace gs {
namespace {

constexpr size_t kErrBytes = 256;    // the error word at the scratch's start
constexpr int kMostNodes = 64;       // bits of a mask
constexpr int kMostCluster = 8;

struct TreeArgs {
  const uint16_t* q;
  int64_t ld_q;
  const int32_t *seq, *n, *count, *pos;
  const uint64_t* mask;
  uint16_t* out;
  int64_t ld_out;
  float* lse;
  int Hq, G, nodes, tiles, window, split, items;
  int cluster;        // the items of a tile are one cluster, and join there
  float scale_log2;
  float* part_o;      // [row][head][item][D]
  float2* part_ml;    // [row][head][item]
  int2* part_n;       // [tree]: pages, nodes in use
  int* err;
  CacheView cache;
};

// A tree's numbers: cached keys, keys in all, nodes in use, the first key that
// any node sees, its page and the pages from there on.
struct Span {
  int n, keys, count, lo, lo_most, page0, pages;
  const int32_t* table;
};

// The first cached key that a node at position `pos` sees; positions below n
// count as n.
__device__ __forceinline__ int first_key(int pos, int n, int window) {
  const long long lo = static_cast<long long>(max(pos, n)) + 1 - window;
  return lo < 0 ? 0 : lo > n ? n : static_cast<int>(lo);
}

// The tree's numbers are read by one warp for its block: all threads go through
// the same pages and barriers whatever happens to the arrays meanwhile.
__device__ __forceinline__ Span find_span(const TreeArgs& a, int tree) {
  __shared__ int s_v[6];
  if (threadIdx.x < 32) {
    int seq = a.seq ? a.seq[tree] : tree, n = a.n[tree];
    int count = a.count ? a.count[tree] : a.nodes;
    const int most = a.cache.pt_stride * kPageTokens;
    bool bad = count < 0 || count > a.nodes;
    count = min(max(count, 0), a.nodes);
    if (n < 0 || n > most - count) {
      bad = true;
      n = n < 0 ? 0 : min(n, most);
    }
    int keys = min(n + count, most);
    if (seq < 0 || seq >= a.cache.n_seq) {
      bad = true;
      seq = 0;
      n = keys = 0;
    }
    int lo = a.window > 0 ? n : 0, lo_most = 0;
    if (a.window > 0) {
      for (int i = threadIdx.x; i < count; i += 32) {
        const int x = first_key(a.pos[static_cast<int64_t>(tree) * a.nodes + i], n, a.window);
        lo = min(lo, x);
        lo_most = max(lo_most, x);
      }
      lo = __reduce_min_sync(0xFFFFFFFFu, lo);
      lo_most = __reduce_max_sync(0xFFFFFFFFu, lo_most);
    }
    if (threadIdx.x == 0) {
      if (bad) atomicExch(a.err, kErrBounds);
      s_v[0] = seq, s_v[1] = n, s_v[2] = keys, s_v[3] = count, s_v[4] = lo, s_v[5] = lo_most;
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

__device__ __forceinline__ uint32_t bits_below(int x) {
  return x <= 0 ? 0u : x >= 32 ? 0xFFFFFFFFu : (1u << x) - 1u;
}
// Which of the tokens tok0 .. tok0 + 31 a row sees.  `mask` has no bits at or
// beyond the tree's count.
__device__ __forceinline__ uint32_t row_view(uint64_t mask, int lo, int n, int tok0) {
  const int d = n - tok0;
  uint32_t v = bits_below(d) & ~bits_below(lo - tok0);
  if (d < 32 && d > -64)
    v |= d >= 0 ? static_cast<uint32_t>(mask) << d : static_cast<uint32_t>(mask >> -d);
  return v;
}

// Which of a register's two 16-bit values are infinite or NaN: all bits of their halves.
template <bool BF16>
__device__ __forceinline__ uint32_t not_finite(uint32_t v) {
  constexpr uint32_t E = BF16 ? 0x7F80u : 0x7C00u;
  return ((v & E) == E ? 0x0000FFFFu : 0u) | ((v & (E << 16)) == (E << 16) ? 0xFFFF0000u : 0u);
}

// Four dims of a row's output, and with the first of them its log-sum-exp.
template <bool BF16, int D>
__device__ __forceinline__ void store_row(const TreeArgs& a, int64_t row, int head, int d, float m,
                                          float l, const float4& acc) {
  const float inv = l != 0.f ? 1.f / l : 0.f;
  *reinterpret_cast<uint2*>(a.out + row * a.ld_out + static_cast<int64_t>(head) * D + d) =
      make_uint2(pack2<BF16>(acc.x * inv, acc.y * inv), pack2<BF16>(acc.z * inv, acc.w * inv));
  if (d == 0 && a.lse)     // (the 15 go out of m and l first, without a rounding)
    a.lse[row * a.Hq + head] =
        l != 0.f ? (finite_max(m) + kHeld<BF16> + log2f(l * (BF16 ? 1.f : 0x1p-15f))) * kLn2
                 : -INFINITY;
}

}  // namespace
}  // namespace gs
