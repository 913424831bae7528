// qlinear.cu -- products of a few rows with 4-bit weights and group scales.
//
//   y[m, r] = sum_g s[r, g] * sum_{k in g} (q[r, k] - z[r, g]) x[m, k]
//
// The inner sums are m16n8k16 tensor instructions on the whole numbers q - z,
// exact in either type, accumulated in fp32; a group's sum is then multiplied by
// its scale in fp32.  So a weight is never rounded.  16 weight rows are the
// instruction's rows, 8 tokens its columns.
//
// Weights are laid out once (gs_qweight_pack) in the order in which lanes read
// them: a block of 16 rows and 64 k is 512 bytes, 16 per lane, of which each 32
// bits are the lane's operand of one instruction, two 4-bit values per mask.  A
// dot product does not care in which order its terms come: of each 32 k, lane t
// of a row's four takes 8 neighbouring ones, so that tokens are read from shared
// memory 16 bytes at a time.
//
// A warp takes one tile of 16 rows, a block eight, over one slice of K; the
// slices of a tile are a cluster, and add up in slice order.  The slices follow
// from the weights' shape alone, so a row's result does not depend on the others.
#include <algorithm>

#include "attend_common.cuh"
#include "internal.h"

namespace gs {
namespace {

constexpr int kWarps = 8, kThreads = kWarps * 32;
constexpr int kTileRows = 16, kBlockRows = kWarps * kTileRows;
constexpr int kBlockK = 64;                        // k of one packed block
constexpr int kBlockBytes = kTileRows * kBlockK / 2;
constexpr int kPartPitch = kBlockRows + 4;         // 2-row stores of 8 rows x 4 lanes on distinct banks
constexpr int kMostSlices = 8;

struct Layout {
  int64_t tiles, blocks, groups;                   // row tiles; 64-k blocks and groups of a row
  int64_t scale_at, zero_at, total;                // byte offsets
};
inline Layout layout_of(const gs_qweight& w) {
  Layout l;
  const int per = w.gated ? 8 : kTileRows;         // outputs of a tile
  l.tiles = ((w.gated ? w.N / 2 : w.N) + per - 1) / per;
  l.blocks = (w.K + kBlockK - 1) / kBlockK;
  l.groups = w.K / w.group;
  l.scale_at = l.tiles * l.blocks * kBlockBytes;
  l.zero_at = l.scale_at + l.tiles * l.groups * kTileRows * 2;
  l.total = l.zero_at + (w.zeros ? l.tiles * l.groups * kTileRows : 0);
  return l;
}

inline int check_weight(const gs_qweight* w) {
  if (!w || w->N < 1 || w->K < 32 || (w->dtype != GS_F16 && w->dtype != GS_BF16) || w->zeros < 0 ||
      w->zeros > 1 || w->gated < 0 || w->gated > 1)
    return GS_ERR_INVALID_ARG;
  if (w->group != 32 && w->group != 64 && w->group != 128) return GS_ERR_UNSUPPORTED;
  if (w->K % w->group || (w->gated && w->N % 2)) return GS_ERR_INVALID_ARG;
  if (w->K > (1 << 20) || w->N > (1 << 24)) return GS_ERR_UNSUPPORTED;
  return GS_OK;
}

// Row r of a tile, as a row of the weights; -1 beyond them.
__device__ __forceinline__ int64_t weight_row(int64_t tile, int r, int N, int gated) {
  if (!gated) {
    const int64_t row = tile * kTileRows + r;
    return row < N ? row : -1;
  }
  const int64_t f = tile * 8 + (r & 7);            // rows 0 .. 7 gate, 8 .. 15 up
  return f < N / 2 ? f + (r >= 8 ? N / 2 : 0) : -1;
}

// One 16-byte piece per thread.  Value j of the instruction's four operand
// registers (row g or g + 8, first or second k pair) lies at bits 4 j and 16 + 4 j.
__global__ void __launch_bounds__(256)
pack_weights_kernel(const uint8_t* q, int N, int K, int gated, int64_t pieces, int64_t blocks,
                    uint4* out) {
  const int64_t e = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (e >= pieces) return;
  const int lane = e & 31, g = lane >> 2, t = lane & 3;
  const int64_t block = e >> 5, tile = block / blocks, kb = block % blocks;
  const int64_t row[2] = {weight_row(tile, g, N, gated), weight_row(tile, g + 8, N, gated)};
  uint32_t v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t k = kb * kBlockK + 32 * (i >> 1) + 8 * t + 4 * (i & 1);
    v[i] = 0;
    if (k < K)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (row[h] < 0) continue;
        const uint8_t* p = q + (row[h] * K + k) / 2;
        const uint32_t a = p[0], b = p[1];         // k, k + 1 and k + 2, k + 3, low nibble first
        v[i] |= ((a & 15) | (a >> 4) << 16) << (4 * h) | ((b & 15) | (b >> 4) << 16) << (4 * h + 8);
      }
  }
  out[e] = make_uint4(v[0], v[1], v[2], v[3]);
}

// Scales and zeros as [tile][group][8][2]: rows g and g + 8 side by side.
__global__ void __launch_bounds__(256)
pack_scales_kernel(const uint16_t* scale, const uint8_t* zero, int N, int gated, int64_t total,
                   int64_t groups, uint16_t* scale_out, uint8_t* zero_out) {
  const int64_t e = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (e >= total) return;
  const int r = static_cast<int>(e & 15);
  const int64_t group = (e >> 4) % groups, tile = (e >> 4) / groups;
  const int64_t row = weight_row(tile, (r >> 1) + 8 * (r & 1), N, gated);
  scale_out[e] = row >= 0 ? scale[row * groups + group] : 0;
  if (zero) zero_out[e] = row >= 0 ? zero[row * groups + group] & 15 : 0;
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
  int M, K, outs, group, slice;        // slice: 64-k blocks of a slice of K
  int epilogue;
  int* err;
};

template <bool BF16>
__device__ __forceinline__ uint32_t sub2(uint32_t a, uint32_t b) {
  uint32_t r;
  if constexpr (BF16) {
    __nv_bfloat162 x, y;
    memcpy(&x, &a, 4);
    memcpy(&y, &b, 4);
    x = __hsub2(x, y);
    memcpy(&r, &x, 4);
  } else {
    __half2 x, y;
    memcpy(&x, &a, 4);
    memcpy(&y, &b, 4);
    x = __hsub2(x, y);
    memcpy(&r, &x, 4);
  }
  return r;
}

// 1024 + q in fp16 and 128 + q in bf16 are q in the low bits of a constant.
template <bool BF16>
constexpr uint32_t kBias = BF16 ? 0x43004300u : 0x64006400u;

template <bool BF16, bool SMALL, int NT>
__global__ void __launch_bounds__(kThreads) qlinear_kernel(const LinearArgs a) {
  constexpr int MT = 8 * NT;                       // tokens of a block
  constexpr int KC = NT == 8 ? 512 : 1024;         // k of a chunk of x in shared memory
  constexpr int XP = KC + 32;                      // pitch: 8 lanes of 2 tokens on distinct banks
  constexpr int PF = 4;                            // packed blocks fetched ahead
  extern __shared__ __align__(16) uint8_t smem_raw[];
  uint16_t* sx = reinterpret_cast<uint16_t*>(smem_raw);
  float* part = reinterpret_cast<float*>(smem_raw);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int slices = gridDim.y, m0 = blockIdx.z * MT;
  const int64_t tile = static_cast<int64_t>(blockIdx.x) * kWarps + warp;
  const int b0 = blockIdx.y * a.slice, b1 = min(static_cast<int64_t>(b0) + a.slice, a.blocks);
  const bool live = tile < a.tiles;
  const uint4* w = a.w + (tile * a.blocks) * 32 + lane;
  const uint32_t* sc = a.scale + tile * a.groups * 8 + g;
  const uint16_t* zr = a.zero ? a.zero + tile * a.groups * 8 + g : nullptr;
  constexpr int NS = SMALL ? 2 : 1;                // scales of a block
  uint4 wq[PF];
  uint32_t sq[PF][NS], zq[PF][NS];
  auto fetch = [&](int b, int at) {
    if (!live || b >= b1) return;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
                 : "=r"(wq[at].x), "=r"(wq[at].y), "=r"(wq[at].z), "=r"(wq[at].w)
                 : "l"(w + static_cast<int64_t>(b) * 32));
#pragma unroll
    for (int h = 0; h < NS; ++h) {
      const int64_t grp = SMALL ? min(static_cast<int64_t>(2 * b + h), a.groups - 1)
                                : static_cast<int64_t>(b) * kBlockK / a.group;
      sq[at][h] = sc[grp * 8];
      zq[at][h] = zr ? zr[grp * 8] : 0x0808u;
    }
  };
#pragma unroll
  for (int p = 0; p < PF; ++p) fetch(b0 + p, p);
  float c[NT][4];
#pragma unroll
  for (int i = 0; i < NT; ++i) c[i][0] = c[i][1] = c[i][2] = c[i][3] = 0.f;
  for (int cb = b0; cb < b1; cb += KC / kBlockK) {
    // ---- this chunk's tokens
    if (cb > b0) __syncthreads();
    for (int e = threadIdx.x; e < MT * (KC / 8); e += kThreads) {
      const int m = e / (KC / 8), k = e % (KC / 8) * 8;
      const int64_t kg = static_cast<int64_t>(cb) * kBlockK + k;
      uint4 v = make_uint4(0, 0, 0, 0);
      if (m0 + m < a.M && kg < a.K)
        v = *reinterpret_cast<const uint4*>(a.x + (m0 + m) * a.ld_x + kg);
      *reinterpret_cast<uint4*>(sx + m * XP + k) = v;
    }
    __syncthreads();
    if (!live) continue;
    const int ce = min(cb + KC / kBlockK, b1);
    for (int bb = cb; bb < ce; bb += PF) {
#pragma unroll
      for (int p = 0; p < PF; ++p) {
        const int b = bb + p;
        if (b >= ce) break;
        const uint32_t words[4] = {wq[p].x, wq[p].y, wq[p].z, wq[p].w};
        uint32_t av[4][4];
        float2 s[NS];
#pragma unroll
        for (int h = 0; h < NS; ++h) {
          s[h] = unpack2<BF16>(sq[p][h]);
          const uint32_t z0 = zq[p][h] & 15, z1 = zq[p][h] >> 8 & 15;
          const uint32_t bias0 = kBias<BF16> | z0 | z0 << 16, bias1 = kBias<BF16> | z1 | z1 << 16;
#pragma unroll
          for (int i = 0; i < 4 / NS; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j)
              av[h * 2 + i][j] = sub2<BF16>((words[h * 2 + i] >> (4 * j) & 0x000F000Fu) | kBias<BF16>,
                                            j & 1 ? bias1 : bias0);
        }
        fetch(b + PF, p);
        const uint16_t* xr = sx + (b - cb) * kBlockK + 8 * t;
#pragma unroll
        for (int i = 0; i < NT; ++i) {
          float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint4 v = *reinterpret_cast<const uint4*>(xr + (8 * i + g) * XP + 32 * h);
            mma16816<BF16>(acc, av[2 * h][0], av[2 * h][1], av[2 * h][2], av[2 * h][3], v.x, v.y);
            mma16816<BF16>(acc, av[2 * h + 1][0], av[2 * h + 1][1], av[2 * h + 1][2],
                           av[2 * h + 1][3], v.z, v.w);
            if (SMALL || h == 1) {
              const float2 f = s[SMALL ? h : 0];
              c[i][0] = fmaf(f.x, acc[0], c[i][0]);
              c[i][1] = fmaf(f.x, acc[1], c[i][1]);
              c[i][2] = fmaf(f.y, acc[2], c[i][2]);
              c[i][3] = fmaf(f.y, acc[3], c[i][3]);
              acc[0] = acc[1] = acc[2] = acc[3] = 0.f;
            }
          }
        }
      }
    }
  }
  // ---- the block's rows as [token][row], then the slices are added in order
  __syncthreads();
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    float* p = part + (8 * i + 2 * t) * kPartPitch + warp * kTileRows + g;
    p[0] = c[i][0];
    p[kPartPitch] = c[i][1];
    p[8] = c[i][2];
    p[kPartPitch + 8] = c[i][3];
  }
  __syncwarp();
  if (slices > 1)
    cluster_sync_all();
  else
    __syncthreads();
  const int tokens = min(MT, a.M - m0), rank = blockIdx.y;
  const uint32_t part_at = smem_u32(part);
  auto total = [&](int m, int r) {                 // four rows of a token
    float4 v = *reinterpret_cast<const float4*>(part + m * kPartPitch + r);
    if (slices > 1) {
      const uint32_t at = part_at + (m * kPartPitch + r) * 4;
      float4 u[kMostSlices];
#pragma unroll
      for (int i = 0; i < kMostSlices; ++i)
        if (i < slices) u[i] = ld_cluster_f32x4(cluster_map(at, i));
      v = u[0];
#pragma unroll
      for (int i = 1; i < kMostSlices; ++i)
        if (i < slices) v.x += u[i].x, v.y += u[i].y, v.z += u[i].z, v.w += u[i].w;
    }
    return v;
  };
  const bool gated = a.epilogue == 2;
  const int quads = gated ? kBlockRows / 8 : kBlockRows / 4;      // fours of outputs of a token
  const int64_t out0 = static_cast<int64_t>(blockIdx.x) * quads * 4;
  bool range = false;
  for (int e = rank * kThreads + threadIdx.x; e < tokens * quads; e += slices * kThreads) {
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
  __syncwarp();
  if (slices > 1) cluster_sync_all();              // the peers have read this block's part
}

// Slices of K: two blocks per SM where the rows alone are too few, of at least
// 128 k.  N and K decide, not M.
int slices_of(const Layout& l) {
  const int64_t wide = (l.tiles + kWarps - 1) / kWarps;
  int64_t s = (2 * kNumSMs + wide - 1) / wide;
  s = std::min<int64_t>(s, (l.blocks + 1) / 2);
  return static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(s, kMostSlices)));
}

template <bool BF16, bool SMALL, int NT>
cudaError_t launch_linear(LinearArgs a, int slices, cudaStream_t s) {
  static DeviceOnce once;
  constexpr int MT = 8 * NT, KC = NT == 8 ? 512 : 1024;
  constexpr size_t smem = std::max<size_t>(MT * (KC + 32) * 2, MT * kPartPitch * 4);
  auto kernel = qlinear_kernel<BF16, SMALL, NT>;
  cudaError_t e = once.run([&] {
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  });
  if (e != cudaSuccess) return e;
  const dim3 grid(static_cast<unsigned>((a.tiles + kWarps - 1) / kWarps), slices,
                  (a.M + MT - 1) / MT);
  return launch_ex(kernel, grid, dim3(kThreads), smem, s, false, dim3(1, slices, 1), a);
}

template <bool BF16, bool SMALL>
cudaError_t launch_rows(const LinearArgs& a, int slices, cudaStream_t s) {
  if (a.M <= 8) return launch_linear<BF16, SMALL, 1>(a, slices, s);
  if (a.M <= 16) return launch_linear<BF16, SMALL, 2>(a, slices, s);
  if (a.M <= 32) return launch_linear<BF16, SMALL, 4>(a, slices, s);
  return launch_linear<BF16, SMALL, 8>(a, slices, s);
}

}  // namespace
}  // namespace gs

extern "C" size_t gs_qweight_bytes(const gs_qweight* w) {
  using namespace gs;
  return check_weight(w) == GS_OK ? static_cast<size_t>(layout_of(*w).total) : 0;
}

extern "C" int gs_qweight_pack(const gs_qweight* w, const void* q, const void* scale, const void* zero,
                               void* stream) {
  using namespace gs;
  if (const int rc = check_weight(w)) return rc;
  if (!w->packed || !aligned16(w->packed) || !q || (reinterpret_cast<uintptr_t>(q) & 1) || !scale ||
      (reinterpret_cast<uintptr_t>(scale) & 1) || (w->zeros != 0) != (zero != nullptr))
    return GS_ERR_INVALID_ARG;
  const Layout l = layout_of(*w);
  uint8_t* base = static_cast<uint8_t*>(w->packed);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const int64_t pieces = l.tiles * l.blocks * 32, total = l.tiles * l.groups * kTileRows;
  if (pieces / 256 >= (1ll << 31) - 1) return GS_ERR_UNSUPPORTED;
  pack_weights_kernel<<<static_cast<unsigned>((pieces + 255) / 256), 256, 0, s>>>(
      static_cast<const uint8_t*>(q), w->N, w->K, w->gated, pieces, l.blocks,
      reinterpret_cast<uint4*>(base));
  if (cudaGetLastError() != cudaSuccess) return GS_ERR_CUDA;
  pack_scales_kernel<<<static_cast<unsigned>((total + 255) / 256), 256, 0, s>>>(
      static_cast<const uint16_t*>(scale), static_cast<const uint8_t*>(zero), w->N, w->gated, total,
      l.groups, reinterpret_cast<uint16_t*>(base + l.scale_at), base + l.zero_at);
  return cudaGetLastError() == cudaSuccess ? GS_OK : GS_ERR_CUDA;
}

extern "C" int gs_qlinear(const gs_qweight* w, const void* x, int64_t ld_x, void* y, int64_t ld_y,
                          int M, int epilogue, int32_t* err, void* stream) {
  using namespace gs;
  if (const int rc = check_weight(w)) return rc;
  if (!w->packed || !aligned16(w->packed) || !x || !aligned16(x) || !y || !err || !aligned4(err) || M < 0 ||
      epilogue < 0 || epilogue > 2 || (epilogue == 2) != (w->gated == 1))
    return GS_ERR_INVALID_ARG;
  const int outs = w->gated ? w->N / 2 : w->N;
  if (ld_x < w->K || ld_x % 8 || ld_y < outs ||
      (reinterpret_cast<uintptr_t>(y) & (epilogue == 1 ? 3 : 1)))
    return GS_ERR_INVALID_ARG;
  if (M > (1 << 21)) return GS_ERR_UNSUPPORTED;
  if (M == 0) return GS_OK;
  const Layout l = layout_of(*w);
  const uint8_t* base = static_cast<const uint8_t*>(w->packed);
  const int want = slices_of(l);
  LinearArgs a;
  a.w = reinterpret_cast<const uint4*>(base);
  a.scale = reinterpret_cast<const uint32_t*>(base + l.scale_at);
  a.zero = w->zeros ? reinterpret_cast<const uint16_t*>(base + l.zero_at) : nullptr;
  a.x = static_cast<const uint16_t*>(x);
  a.ld_x = ld_x;
  a.y = y;
  a.ld_y = ld_y;
  a.tiles = l.tiles;
  a.blocks = l.blocks;
  a.groups = l.groups;
  a.M = M;
  a.K = w->K;
  a.outs = outs;
  a.group = w->group;
  a.slice = static_cast<int>((l.blocks + want - 1) / want);
  a.epilogue = epilogue;
  a.err = err;
  const int slices = static_cast<int>((l.blocks + a.slice - 1) / a.slice);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e;
  if (w->dtype == GS_BF16)
    e = w->group == 32 ? launch_rows<true, true>(a, slices, s) : launch_rows<true, false>(a, slices, s);
  else
    e = w->group == 32 ? launch_rows<false, true>(a, slices, s) : launch_rows<false, false>(a, slices, s);
  return e == cudaSuccess ? GS_OK : GS_ERR_CUDA;
}
