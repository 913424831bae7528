// qlinear.cu -- products with 4-bit weights and group scales: few tokens here, more than 32 in
// qlinear_wide.cuh.
//
//   y[m, r] = sum_g s[r, g] * (sum_{k in g} q[r, k] x[m, k] - z[r, g] sum_{k in g} x[m, k])
//
// The inner sums are m16n8k16 tensor instructions: 16 weight rows are the
// instruction's rows, 8 tokens its columns.  Their operand is the whole number q with
// as little work as possible, for the weights are read once and each takes part
// in few products.  In fp16 the four bits as they lie are a number, q 2^-24 (or, four places
// up, q 2^-20, for the tile's upper rows): one mask for two weights.  In bf16 they
// become the upper mantissa bits of 16 + q.  What that adds, and the zero, come off as
// one multiple of the tokens' sum over the group, before the group's scale: all of it is
// fp32, no weight is rounded, and the error is that of fp32 sums of 15 (31 in bf16) s
// |x| a weight.
//
// Weights are laid out once (gs_qweight_pack) in the order in which lanes read
// them: a block of 16 rows and 64 k is 512 bytes, 16 per lane, of which each 32
// bits are the lane's operand of one instruction.  A dot product does not care in
// which order its terms come: of each 32 k, lane t of a row's four takes 8
// neighbouring ones, so that tokens are read from shared memory 16 bytes at a time.
//
// A warp takes one tile of 16 rows over one slice of K; the slices of a tile are a
// cluster, and add up in slice order.  The slices follow from the weights' shape
// alone, so a row's result does not depend on the others.
//
// What bounds it: 28,672 x 8192 and one token 28 us, 4.4 TB/s of weights and near one
// instruction for two weights of a warp's lanes; 8192 x 8192, 11 us for one token, 12 for 8, 15.7
// for 16, 26 for 32: from 16 on the issue of products and of the loads of tokens
// (for 32, the tensor pipes are 35 per cent busy, the issue slots 37); with fewer weights
// the start of a block: a first weight, the tokens and their sums, 4 us in all (1024 x
// 1024 and one token 3.3 us).  Two tiles to a warp read the tokens half as often but leave
// half the warps (28 us for 32).
#include <algorithm>

#include "qlinear_wide.cuh"

namespace gs {
namespace {

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

// Where a word of eight weights has value j (of the instruction's four operand
// registers: row g or g + 8, first or second k pair), for the pair's first and
// second k.  fp16: bits 4 j and 16 + 4 j.  bf16: three bits further up, the last
// value going round the word's end, so that a rotation by 4 j brings it under
// the mantissa's upper bits.
__device__ __forceinline__ uint32_t place_pair(int j, uint32_t first, uint32_t second, bool bf16) {
  const uint32_t v = first | second << 16;
  return bf16 ? __funnelshift_l(v, v, 4 * j + 3) : v << (4 * j);
}

// One 16-byte piece per thread.
__global__ void __launch_bounds__(256)
pack_weights_kernel(const uint8_t* q, int N, int K, int gated, bool bf16, int64_t pieces,
                    int64_t blocks, uint4* out) {
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
        v[i] |= place_pair(h, a & 15, a >> 4, bf16) | place_pair(2 + h, b & 15, b >> 4, bf16);
      }
  }
  out[e] = make_uint4(v[0], v[1], v[2], v[3]);
}

// Scales and zeros as [tile][group][8][2]: rows g and g + 8 side by side.
__global__ void __launch_bounds__(256)
pack_scales_kernel(const uint16_t* scale, const uint8_t* zero, int N, int gated, int64_t total,
                   int64_t groups, int64_t have, uint16_t* scale_out, uint8_t* zero_out) {
  const int64_t e = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (e >= total) return;
  const int r = static_cast<int>(e & 15);
  const int64_t group = (e >> 4) % groups, tile = (e >> 4) / groups;
  const int64_t row = weight_row(tile, (r >> 1) + 8 * (r & 1), N, gated);
  const bool in = row >= 0 && group < have;        // (the last block may be half a block)
  scale_out[e] = in ? scale[row * have + group] : 0;
  if (zero) zero_out[e] = in ? zero[row * have + group] & 15 : 0;
}

// ON: a wave of blocks that keep the tokens in shared memory and go on from tile to tile.
template <int NT, bool ON>
struct Shape {
  static constexpr int tokens = 8 * NT;            // of a block
  static constexpr int warps = NT <= 2 ? 4 : 8;
  static constexpr int threads = 32 * warps, rows = warps * kTileRows;
  static constexpr int resident = warps == 4 ? 4 : 2;    // blocks of an SM
  // k of x in shared memory: twice, or all of them
  static constexpr int chunk = (NT == 1 ? 1024 : 512) * (ON ? 2 : 1);
  static constexpr int pitch = chunk + 32;         // 8 lanes of 2 tokens on distinct banks
  static constexpr int part_pitch = rows + 4;      // 2-row stores of 8 rows x 4 lanes likewise
  static constexpr int x_bytes = tokens * pitch * 2, part_bytes = tokens * part_pitch * 4;
  template <int G>
  static constexpr int ahead = G == 32 ? 4 : 8;          // packed blocks fetched ahead
  template <int G>
  static constexpr int sum_bytes = chunk / G * tokens * 4;
  static constexpr int sum_at = x_bytes * (ON ? 1 : 2);
  template <int G>
  static constexpr int part_at = ON ? sum_at + sum_bytes<G> : 0;
  template <int G>
  static constexpr int smem = std::max(sum_at + sum_bytes<G>, part_at<G> + part_bytes);
};

// A group's scales and zeros as the sums want them: c += f (z u + acc) for the tile's
// lower and upper row, u the tokens' sum.
template <bool BF16>
__device__ __forceinline__ void group_factors(uint32_t scale, uint32_t zero, float2& f, float2& z) {
  f = unpack2<BF16>(scale);
  f.x *= kUnit0<BF16>;
  f.y *= kUnit1<BF16>;
  // a byte as the last one of 2^23 is a number; the products and sums are exact
  const float z0 = __uint_as_float(__byte_perm(zero, 0x4B000000u, 0x7650)),
              z1 = __uint_as_float(__byte_perm(zero, 0x4B000000u, 0x7651));
  z.x = fmaf(z0, -1.f / kUnit0<BF16>, (8388608.f - kAdded<BF16>) / kUnit0<BF16>);
  z.y = fmaf(z1, -1.f / kUnit1<BF16>, (8388608.f - kAdded<BF16>) / kUnit1<BF16>);
}

// G: the group, 32, 64 or 128.
template <bool BF16, int G, int NT, bool ON>
__global__ void __launch_bounds__(Shape<NT, ON>::threads, Shape<NT, ON>::resident)
qlinear_kernel(const LinearArgs a) {
  using S = Shape<NT, ON>;
  constexpr int KC = S::chunk, XP = S::pitch, W = S::warps, PP = S::part_pitch;
  constexpr int PF = S::template ahead<G>, NG = PF * kBlockK / G;   // their groups
  extern __shared__ __align__(16) uint8_t smem_raw[];
  uint16_t* sx = reinterpret_cast<uint16_t*>(smem_raw);                  // [buffer][token][k]
  float* sums = reinterpret_cast<float*>(smem_raw + S::sum_at);          // [group][token]
  float* part = reinterpret_cast<float*>(smem_raw + S::template part_at<G>);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int slices = ON ? 1 : gridDim.y, m0 = blockIdx.z * S::tokens;
  const int tokens = min(S::tokens, a.M - m0);     // (the others' columns hold anything)
  int64_t tile = static_cast<int64_t>(blockIdx.x) * W + warp;
  const int b0 = blockIdx.y * a.slice, b1 = min(static_cast<int64_t>(b0) + a.slice, a.blocks);
  bool live = tile < a.tiles;
  const int64_t of = live ? tile : 0;
  // this lane's place in the block after the one it works on, and its groups' there
  const uint4* w = a.w + (of * a.blocks + b0) * 32 + lane;
  const uint32_t* sc = a.scale + (of * a.groups + static_cast<int64_t>(b0) * kBlockK / G) * 8 + g;
  const uint16_t* zr = a.zero ? a.zero + (sc - a.scale) : nullptr;
  uint4 wq[PF];
  uint32_t sq[NG];
  uint16_t zq[NG];
  auto fetch = [&](int at, int p) {                // the block `at` blocks on, to place p
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
                 : "=r"(wq[p].x), "=r"(wq[p].y), "=r"(wq[p].z), "=r"(wq[p].w)
                 : "l"(w + at * 32));
    if (kBlockK >= G || p % 2 == 0)                // (a group of 128: with its first block)
#pragma unroll
      for (int h = 0; h < (kBlockK >= G ? kBlockK / G : 1); ++h) {
        sq[p * kBlockK / G + h] = sc[(at * kBlockK / G + h) * 8];
        zq[p * kBlockK / G + h] = zr ? zr[(at * kBlockK / G + h) * 8] : 0x0808;
      }
  };
  auto copy = [&](int cb, int to) {                // a chunk's tokens
    const int kn = min(KC, (b1 - cb) * kBlockK);   // a multiple of 64
    const int64_t k0 = static_cast<int64_t>(cb) * kBlockK;
    for (int e = threadIdx.x; e < tokens * (KC / 8); e += S::threads) {
      const int m = e / (KC / 8), k = e % (KC / 8) * 8;
      if (k >= kn) continue;
      const bool in = k0 + k < a.K;                // (else zeros)
      asm volatile("cp.async.ca.shared.global [%0], [%1], 16, %2;" ::"r"(
                       smem_u32(sx + to * (S::x_bytes / 2) + m * XP + k)),
                   "l"(a.x + (m0 + m) * a.ld_x + (in ? k0 + k : 0)), "r"(in ? 16 : 0)
                   : "memory");
    }
  };
  copy(b0, 0);
#pragma unroll
  for (int p = 0; p < PF; ++p)
    if (live && b0 + p < b1) fetch(p, p);
  float c[NT][4], acc[NT][4];
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) c[i][e] = acc[i][e] = 0.f;
  int buf = 0;
  for (int round = blockIdx.x;;) {
    const bool first = !ON || round == static_cast<int>(blockIdx.x);
    const bool again = ON && tile + gridDim.x * W < a.tiles;         // this warp has another tile
    for (int cb = b0; cb < b1; cb += KC / kBlockK, buf ^= ON ? 0 : 1) {
      if (first) {
        asm volatile("cp.async.wait_all;" ::: "memory");
        __syncthreads();                             // the chunk is there, the last one done with
        if (!ON && cb + KC / kBlockK < b1) copy(cb + KC / kBlockK, buf ^ 1);
      }
      const uint16_t* x0 = sx + buf * (S::x_bytes / 2) + g * XP + 8 * t;
      const int ce = min(cb + KC / kBlockK, b1);
      // ---- the tokens' sums over each group: a product with ones, shared by the warps
      constexpr uint32_t one = BF16 ? 0x3F803F80u : 0x3C003C00u;
      const int jobs = first ? ((ce - cb) * kBlockK + G - 1) / G * NT : 0;
      for (int e = warp; e < jobs; e += W) {
        const int i = e % NT, grp = e / NT;
        float u[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int h = 0; h < G / 32; ++h) {
          const uint4 v = *reinterpret_cast<const uint4*>(x0 + 8 * i * XP + grp * G + 32 * h);
          mma16816<BF16>(u, one, one, one, one, v.x, v.y);
          mma16816<BF16>(u, one, one, one, one, v.z, v.w);
        }
        if (g == 0)
          *reinterpret_cast<float2*>(sums + grp * S::tokens + 8 * i + 2 * t) = make_float2(u[0], u[1]);
      }
      if (first) __syncthreads();
      if (!live) continue;
      // one block: its products, and at a group's end its factors
      auto work = [&](int b, int p, bool ahead) {
        const uint32_t words[4] = {wq[p].x, wq[p].y, wq[p].z, wq[p].w};
        const uint16_t* xr = x0 + (b - cb) * kBlockK;
        const float* su = sums + (b - cb) * kBlockK / G * S::tokens + 2 * t;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint32_t v[2][4];
          operands<BF16>(words[2 * h], v[0]);
          operands<BF16>(words[2 * h + 1], v[1]);
#pragma unroll
          for (int i = 0; i < NT; ++i) {
            const uint4 x = *reinterpret_cast<const uint4*>(xr + 8 * i * XP + 32 * h);
            mma16816<BF16>(acc[i], v[0][0], v[0][1], v[0][2], v[0][3], x.x, x.y);
            mma16816<BF16>(acc[i], v[1][0], v[1][1], v[1][2], v[1][3], x.z, x.w);
          }
          if (G == 32 || (h == 1 && (G == 64 || p % 2 == 1))) {
            const int at = p * kBlockK / G + (G == 32 ? h : 0);
            float2 f, z;
            group_factors<BF16>(sq[at], zq[at], f, z);
#pragma unroll
            for (int i = 0; i < NT; ++i) {
              const float2 u = *reinterpret_cast<const float2*>(su + (G == 32 ? h * S::tokens : 0) + 8 * i);
              c[i][0] = fmaf(f.x, fmaf(z.x, u.x, acc[i][0]), c[i][0]);
              c[i][1] = fmaf(f.x, fmaf(z.x, u.y, acc[i][1]), c[i][1]);
              c[i][2] = fmaf(f.y, fmaf(z.y, u.x, acc[i][2]), c[i][2]);
              c[i][3] = fmaf(f.y, fmaf(z.y, u.y, acc[i][3]), c[i][3]);
              acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0.f;
            }
          }
        }
        if (!ahead) return;
        // (a group of two blocks keeps its numbers until its second one is done)
        if (G <= kBlockK) {
          fetch(PF + p, p);
        } else if (p % 2 == 1) {
          fetch(PF + p - 1, p - 1);
          fetch(PF + p, p);
        }
      };
      int b = cb;
      // with PF more blocks to fetch, of the next tile at last
      for (; b + PF <= ce && (b + 2 * PF <= b1 || (again && b + PF == b1)); b += PF) {
        if (ON && b + PF == b1) {
          const int64_t skip = gridDim.x * W - 1;
          w += skip * a.blocks * 32;
          sc += skip * a.groups * 8;
          if (zr) zr += skip * a.groups * 8;
        }
#pragma unroll
        for (int p = 0; p < PF; ++p) work(b + p, p, true);
        w += PF * 32;
        sc += NG * 8;
        if (zr) zr += NG * 8;
      }
      for (; b < ce; b += PF) {
#pragma unroll
        for (int p = 0; p < PF; ++p) {
          if (b + p >= ce) break;
          work(b + p, p, false);
        }
        // the next ones, as many as there are
#pragma unroll
        for (int p = 0; p < PF; ++p)
          if (b + PF + p < b1) fetch(PF + p, p);
        w += PF * 32;
        sc += NG * 8;
        if (zr) zr += NG * 8;
      }
    }
    // ---- the block's rows as [token][row], then the slices are added in order
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      float* p = part + (8 * i + 2 * t) * PP + warp * kTileRows + g;
      p[0] = c[i][0];
      p[PP] = c[i][1];
      p[8] = c[i][2];
      p[PP + 8] = c[i][3];
    }
    __syncwarp();
    if (slices > 1)
      cluster_sync_all();
    else
      __syncthreads();
    finish_rows<BF16, S::rows, S::threads, PP>(a, part, m0, tokens, slices, ON ? 0 : blockIdx.y, round,
                                              threadIdx.x);
    __syncwarp();
    if (slices > 1) cluster_sync_all();            // the peers have read this block's part
    if (!ON) return;
    round += gridDim.x;
    if (round >= a.rounds) return;
    tile += gridDim.x * W;
    live = tile < a.tiles;
#pragma unroll
    for (int i = 0; i < NT; ++i) c[i][0] = c[i][1] = c[i][2] = c[i][3] = 0.f;
  }
}

// Tokens beyond which the kernel of qlinear_wide.cuh takes over: bf16, 8192 x 8192, 32 tokens
// 25.9 us here and 31.1 there, 33 to 64 40.5 to 43.1 and 31.4 to 32.5, 128 83.9 and 34.4;
// 1024 x 1024, fp16, groups of 64, 64 tokens 6.4 and 6.7, 1024 x 4096 11.7 and 9.4.
constexpr int kFewTokens = 32;

// Slices of K, of whole groups and at least 128 k: 16 warps per SM where the rows
// alone are too few.  N and K decide, not M.
int slices_of(const Layout& l) {
  int64_t s = 16 * kNumSMs / l.tiles;
  s = std::min<int64_t>(s, (l.blocks + 1) / 2);
  return static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(s, kMostSlices)));
}

template <bool BF16, int G, int NT, bool ON>
cudaError_t launch_linear(const LinearArgs& args, int slices, cudaStream_t s) {
  using S = Shape<NT, ON>;
  static DeviceOnce once;
  constexpr size_t smem = S::template smem<G>;
  auto kernel = qlinear_kernel<BF16, G, NT, ON>;
  cudaError_t e = once.run([&] {
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  });
  if (e != cudaSuccess) return e;
  LinearArgs a = args;
  a.rounds = static_cast<int>((a.tiles + S::warps - 1) / S::warps);
  const dim3 grid(ON ? std::min(a.rounds, S::resident * kNumSMs) : a.rounds, slices,
                  (a.M + S::tokens - 1) / S::tokens);
  return launch_ex(kernel, grid, dim3(S::threads), smem, s, false, dim3(1, slices, 1), a);
}

// With one slice and few enough k, a wave of blocks goes on from tile to tile: 59,392 rows, K
// 1024, bf16, 5 tokens 11.7 us, 13.0 with a block for each 64 rows, which waits for its first
// weights and tokens every time (K 2048, one token 19.5 and 21.6; 16 tokens 13.9 and 15.9; a
// wave or less, 20,480 rows, 7.0 either way).
template <bool BF16, int G, int NT>
cudaError_t launch_on(const LinearArgs& a, int slices, cudaStream_t s) {
  using S = Shape<NT, true>;
  if (slices == 1 && a.blocks <= S::chunk / kBlockK && a.blocks % S::template ahead<G> == 0)
    return launch_linear<BF16, G, NT, true>(a, slices, s);
  return launch_linear<BF16, G, NT, false>(a, slices, s);
}

// Many tokens: a wave of blocks of 128 rows and a slice of K, by N and K alone.
int wide_slices_of(const Layout& l) {
  const int64_t rows = (l.tiles + kWideTiles - 1) / kWideTiles;
  int64_t s = kNumSMs / rows;
  s = std::min<int64_t>(s, (l.blocks + 1) / 2);
  return static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(s, kMostSlices)));
}

template <bool BF16, int G>
cudaError_t launch_wide(const LinearArgs& a, int slices, cudaStream_t s) {
  static DeviceOnce once;
  auto kernel = qlinear_wide_kernel<BF16, G>;
  cudaError_t e = once.run([&] {
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, WideShape::total);
  });
  if (e != cudaSuccess) return e;
  CUtensorMap x;
  const uint64_t dims[2] = {static_cast<uint64_t>(a.K), static_cast<uint64_t>(a.M)},
                 strides[1] = {static_cast<uint64_t>(a.ld_x) * 2};
  const uint32_t box[2] = {kBlockK, kWideTokens};
  if (!make_map_nd(&x, a.x, 2, dims, strides, box)) return cudaErrorUnknown;
  const dim3 grid(static_cast<unsigned>((a.tiles + kWideTiles - 1) / kWideTiles), slices,
                  (a.M + kWideTokens - 1) / kWideTokens);
  return launch_ex(kernel, grid, dim3(kWideBlockThreads), WideShape::total, s, false, dim3(1, slices, 1), x, a);
}

template <bool BF16, int G>
cudaError_t launch_rows(const LinearArgs& a, int slices, cudaStream_t s) {
  if (a.M > kFewTokens) return launch_wide<BF16, G>(a, slices, s);
  if (a.M <= 8) return launch_on<BF16, G, 1>(a, slices, s);
  if (a.M <= 16) return launch_on<BF16, G, 2>(a, slices, s);
  return launch_linear<BF16, G, 4, false>(a, slices, s);
}

template <bool BF16>
cudaError_t launch_group(const LinearArgs& a, int group, int slices, cudaStream_t s) {
  if (group == 32) return launch_rows<BF16, 32>(a, slices, s);
  if (group == 64) return launch_rows<BF16, 64>(a, slices, s);
  return launch_rows<BF16, 128>(a, slices, s);
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
      static_cast<const uint8_t*>(q), w->N, w->K, w->gated, w->dtype == GS_BF16, pieces, l.blocks,
      reinterpret_cast<uint4*>(base));
  if (cudaGetLastError() != cudaSuccess) return GS_ERR_CUDA;
  pack_scales_kernel<<<static_cast<unsigned>((total + 255) / 256), 256, 0, s>>>(
      static_cast<const uint16_t*>(scale), static_cast<const uint8_t*>(zero), w->N, w->gated, total,
      l.groups, w->K / w->group, reinterpret_cast<uint16_t*>(base + l.scale_at), base + l.zero_at);
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
  const int want = M > kFewTokens ? wide_slices_of(l) : slices_of(l);
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
  a.slice = static_cast<int>(((l.blocks + want - 1) / want + 1) / 2 * 2);   // whole groups
  a.epilogue = epilogue;
  a.err = err;
  const int slices = static_cast<int>((l.blocks + a.slice - 1) / a.slice);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e;
  if (w->dtype == GS_BF16)
    e = launch_group<true>(a, w->group, slices, s);
  else
    e = launch_group<false>(a, w->group, slices, s);
  return e == cudaSuccess ? GS_OK : GS_ERR_CUDA;
}
