// qlinear_common.cuh -- what the kernels of gs_qlinear share: the packed layout, the operands
// that a word of eight weights becomes, and the end of a block of rows.
#pragma once
#include "attend_common.cuh"
#include "internal.h"

namespace gs {
namespace {

constexpr int kTileRows = 16;
constexpr int kBlockK = 64;                        // k of one packed block
constexpr int kBlockBytes = kTileRows * kBlockK / 2;
constexpr int kMostSlices = 8;

struct Layout {
  int64_t tiles, blocks, groups;                   // row tiles; 64-k blocks and their groups
  int64_t scale_at, zero_at, total;                // byte offsets
};
inline Layout layout_of(const gs_qweight& w) {
  Layout l;
  const int per = w.gated ? 8 : kTileRows;         // outputs of a tile
  l.tiles = ((w.gated ? w.N / 2 : w.N) + per - 1) / per;
  l.blocks = (w.K + kBlockK - 1) / kBlockK;
  l.groups = (l.blocks * kBlockK + w.group - 1) / w.group;
  l.scale_at = l.tiles * l.blocks * kBlockBytes;
  l.zero_at = l.scale_at + l.tiles * l.groups * kTileRows * 2;
  l.total = l.zero_at + (w.zeros ? l.tiles * l.groups * kTileRows : 0);
  return l;
}

struct LinearArgs {
  const uint4* w;
  const uint32_t* scale;      // [tile][group][8] pairs
  const uint16_t* zero;       // the same, pairs of bytes; NULL: 8
  const uint16_t* x;
  int64_t ld_x;
  void* y;
  int64_t ld_y;
  int64_t tiles, blocks, groups;
  int M, K, outs, slice;        // slice: 64-k blocks of a slice of K
  int rounds;                   // thread blocks' rows; with ON one takes every gridDim.x-th
  int epilogue;
  int* err;
};

// A word's four operand registers.  What is multiplied is, for q of the tile's
// lower and upper rows: fp16: q 2^-24 and q 2^-20; bf16: (16 + q) 2^-4, both.
template <bool BF16>
__device__ __forceinline__ void operands(uint32_t w, uint32_t (&v)[4]) {
  if constexpr (BF16) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      v[j] = ((j ? __funnelshift_r(w, w, 4 * j) : w) & 0x00780078u) | 0x3F803F80u;
  } else {
    v[0] = w & 0x000F000Fu;
    v[1] = w & 0x00F000F0u;
    v[2] = w >> 8 & 0x000F000Fu;
    v[3] = w >> 8 & 0x00F000F0u;
  }
}
template <bool BF16>
constexpr float kUnit0 = BF16 ? 0x1p4f : 0x1p24f;  // what a lower row's sum is multiplied by
template <bool BF16>
constexpr float kUnit1 = BF16 ? 0x1p4f : 0x1p20f;
template <bool BF16>
constexpr float kAdded = BF16 ? 16.f : 0.f;

// The end of a block's rows, which each of a tile's slices holds in `part` as [token][row]: the
// slices' sums in order, the epilogue, the outputs.  The blocks of a cluster share the
// tokens.  `block`: the number of the block of rows.
template <bool BF16, int ROWS, int THREADS, int PITCH>
__device__ __forceinline__ void finish_rows(const LinearArgs& a, const float* part, int m0, int tokens,
                                            int slices, int rank, int64_t block, int tid) {
  const uint32_t part_at = smem_u32(part);
  auto total = [&](int m, int r) {                 // four rows of a token
    if (slices == 1) return *reinterpret_cast<const float4*>(part + m * PITCH + r);
    const uint32_t at = part_at + (m * PITCH + r) * 4;
    float4 u[kMostSlices];
#pragma unroll
    for (int i = 0; i < kMostSlices; ++i)
      if (i < slices) u[i] = ld_cluster_f32x4(cluster_map(at, i));
    float4 v = u[0];
#pragma unroll
    for (int i = 1; i < kMostSlices; ++i)
      if (i < slices) v.x += u[i].x, v.y += u[i].y, v.z += u[i].z, v.w += u[i].w;
    return v;
  };
  const bool gated = a.epilogue == 2;
  const int quads = gated ? ROWS / 8 : ROWS / 4;      // fours of outputs of a token
  const int64_t out0 = block * quads * 4;
  bool range = false;
  for (int e = rank * THREADS + tid; e < tokens * quads; e += slices * THREADS) {
    const int m = e / quads, o = e % quads * 4;
    float r[4];
    if (gated) {
      const int at = o / 8 * kTileRows + o % 8;
      const float4 ga = total(m, at), up = total(m, at + 8);
      r[0] = ga.x / (1.f + expf(-ga.x)) * up.x;
      r[1] = ga.y / (1.f + expf(-ga.y)) * up.y;
      r[2] = ga.z / (1.f + expf(-ga.z)) * up.z;
      r[3] = ga.w / (1.f + expf(-ga.w)) * up.w;
    } else {
      const float4 v = total(m, o);
      r[0] = v.x, r[1] = v.y, r[2] = v.z, r[3] = v.w;
    }
    const int64_t at = (m0 + m) * a.ld_y + out0 + o;
    const int left = static_cast<int>(min(static_cast<int64_t>(4), a.outs - (out0 + o)));
    if (left <= 0) continue;
    if (a.epilogue == 1) {
      float* y = static_cast<float*>(a.y) + at;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (i < left) y[i] += r[i];
    } else {
      uint16_t* y = static_cast<uint16_t*>(a.y) + at;
      const uint32_t lo = pack2<BF16>(r[0], r[1]), hi = pack2<BF16>(r[2], r[3]);
      if (!BF16)
#pragma unroll
        for (int i = 0; i < 4; ++i) range |= i < left && !(fabsf(r[i]) <= 65504.f);
      if (left == 4 && !(reinterpret_cast<uintptr_t>(y) & 7)) {
        *reinterpret_cast<uint2*>(y) = make_uint2(lo, hi);
      } else {
        const uint16_t h[4] = {static_cast<uint16_t>(lo), static_cast<uint16_t>(lo >> 16),
                               static_cast<uint16_t>(hi), static_cast<uint16_t>(hi >> 16)};
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (i < left) y[i] = h[i];
      }
    }
  }
  if (range) atomicExch(a.err, kErrRange);
}

}  // namespace
}  // namespace gs
