// tree_common.cuh -- the tree attentions' arguments, a tree's numbers and masks,
// and the end of a row.
#pragma once
#include "attend_common.cuh"

namespace gs {
namespace {

constexpr size_t kErrBytes = 256;    // the error word at the scratch's start
constexpr int kMostNodes = 64;       // bits of a mask
constexpr int kMostCluster = 8;

// What the joining kernel has to know of a tree.
struct TreePart {
  int64_t first;      // its first page in the order of all work (wide kernel, open split)
  int pages, count;
};

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
  float light;        // 1 over the weight of a row's largest score: 2^-15, 2^-7 or 1
  float* part_o;      // [row][head][item][D]
  float2* part_ml;    // [row][head][item]: the largest score (before scaling), the sum
  TreePart* part_n;   // [tree]
  int64_t* part_all;  // pages of all work, blocks that share it (wide kernel, open split)
  int* err;
  CacheView cache;
};

// The first cached key that a node at position `pos` sees; positions below n
// count as n.
__device__ __forceinline__ int first_key(int pos, int n, int window) {
  const long long lo = static_cast<long long>(max(pos, n)) + 1 - window;
  return lo < 0 ? 0 : lo > n ? n : static_cast<int>(lo);
}

// A tree's numbers as they can be used: sequence, cached keys, keys in all, nodes in use.
struct TreeNums {
  int seq, n, keys, count;
  bool bad;
};
__device__ __forceinline__ TreeNums read_tree(const TreeArgs& a, int tree) {
  TreeNums t;
  const int most = a.cache.pt_stride * kPageTokens;
  t.seq = a.seq ? a.seq[tree] : tree;
  t.n = a.n[tree];
  t.count = a.count ? a.count[tree] : a.nodes;
  t.bad = t.count < 0 || t.count > a.nodes;
  t.count = min(max(t.count, 0), a.nodes);
  if (t.n < 0 || t.n > most - t.count) {
    t.bad = true;
    t.n = t.n < 0 ? 0 : min(t.n, most);
  }
  t.keys = min(t.n + t.count, most);
  if (t.seq < 0 || t.seq >= a.cache.n_seq) {
    t.bad = true;
    t.seq = t.n = t.keys = 0;
  }
  return t;
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

__device__ __forceinline__ float row_lse(const TreeArgs& a, float m, float l) {
  return l != 0.f ? fmaf(finite_max(m), a.scale_log2, log2f(l * a.light)) * kLn2 : -INFINITY;
}

// Four dims of a row's output, and with the first of them its log-sum-exp.
template <bool BF16, int D>
__device__ __forceinline__ void store_row(const TreeArgs& a, int64_t row, int head, int d, float m,
                                          float l, const float4& acc) {
  const float inv = l != 0.f ? 1.f / l : 0.f;
  *reinterpret_cast<uint2*>(a.out + row * a.ld_out + static_cast<int64_t>(head) * D + d) =
      make_uint2(pack2<BF16>(acc.x * inv, acc.y * inv), pack2<BF16>(acc.z * inv, acc.w * inv));
  if (d == 0 && a.lse) a.lse[row * a.Hq + head] = row_lse(a, m, l);
}

}  // namespace
}  // namespace gs
