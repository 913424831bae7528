// qlinear_wide.cuh -- products with 4-bit weights for many rows: tcgen05.
//
// From some tens of tokens on the products themselves bound the kernel of mma.sync: 8 tokens to an
// instruction, whose operand is loaded from shared memory again for each tile of weights.
// Here 128 weight rows are the rows of a tcgen05 product, 128 tokens its columns, 128 k a
// stage.  Eight warps turn packed blocks into the operand in shared memory, q - z (exact; in
// the other kernel's units), a tile of 16 rows each; the tokens come by TMA; two warps issue
// the products of every other stage (110 cycles each for the issuing thread); a group's products
// add up in tensor memory, and eight more warps, a thread per row and half of the tokens, add
// scale times the sum to the row's sums in registers.
//
// K is sliced over a cluster so that a block for each 128 rows fills the GPU; the slices
// follow from the weights' shape, and no token's sums depend on the others.
//
// Packed weights are copied to shared memory seven stages ahead: two stages ahead in
// registers held the whole to 1.4 TB/s.  What bounds it now is the time that an unpacking
// warp takes for a stage, some 250 instructions one after another with two warps on a scheduler:
// bf16, 8192 x 8192, 128 tokens 34 us, of which the products' own time is a quarter.  Every 128
// tokens unpack the weights again (544 tokens 157 us): beyond 256 tokens gs_linear's 16-bit
// weights are faster (64 to 256 tokens 60 to 64 us, 544 93).
// Unpacking and adding by the same eight warps 36 us; 16 unpacking warps, for want of
// registers, 41.  Groups of 32 are four sums a stage to read from tensor memory and add instead of
// one: fp16, 128 tokens 51 us, 32 with groups of 128.
#pragma once
#include "qlinear_common.cuh"
#include "qlinear_places.h"

namespace gs {
namespace {

constexpr int kWideTokens = 128, kWideRowsOut = 128, kWideTiles = kWideRowsOut / kTileRows;
constexpr int kWideK = 128;                          // k of a stage
// warps: 0 to 7 unpack, 8 to 15 add, then two that issue products and one that fetches tokens
constexpr int kAddWarp = 8, kProductsWarp = 16, kTokensWarp = 18;
constexpr int kAddThreads = 256, kWideBlockThreads = 640;
// Registers of an adding thread and of the others, of 96 at launch.
constexpr int kAddRegs = 128, kOtherRegs = 72;
static_assert(kAddThreads * kAddRegs + (kWideBlockThreads - kAddThreads) * kOtherRegs <= kWideBlockThreads * 96);

struct WideShape {
  static constexpr int stages = 2, ahead = 8;        // of operands; of packed weights
  static constexpr int a_bytes = kWideRowsOut * kWideK * 2, x_bytes = kWideTokens * kWideK * 2;   // halves of 64 k
  static constexpr int sums = 512 / kWideTokens;     // groups' places in tensor memory
  static constexpr int pitch = kWideRowsOut + 4;     // of a token's sums
  static constexpr int x_at = stages * a_bytes;
  static constexpr int w_at = x_at + stages * x_bytes;
  static constexpr int w_bytes = 2 * kBlockBytes, z_bytes = 4 * 16;      // a stage's of a tile
  static constexpr int z_at = w_at + kWideTiles * ahead * w_bytes;
  static constexpr int bars_at = z_at + kWideTiles * ahead * z_bytes;
  static constexpr int total = bars_at + 256 + 1024; // (1024: the start is aligned by hand)
  static constexpr int barriers = 4 * stages + 3 * sums;   // and behind them tensor memory's address
  static_assert(kWideTokens * pitch * 4 <= w_at && total <= 227 * 1024 && 8 * barriers + 4 <= 256);
};

// q - z of a word's pairs, in the operands' units.
template <bool BF16>
__device__ __forceinline__ uint32_t minus(uint32_t v, uint32_t z) {
  uint32_t r;
  if constexpr (BF16) {
    __nv_bfloat162 x, y;
    memcpy(&x, &v, 4);
    memcpy(&y, &z, 4);
    x = __hsub2(x, y);
    memcpy(&r, &x, 4);
  } else {
    __half2 x, y;
    memcpy(&x, &v, 4);
    memcpy(&y, &z, 4);
    x = __hsub2(x, y);
    memcpy(&r, &x, 4);
  }
  return r;
}

__device__ __forceinline__ void copy16(void* to, const void* from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(to)), "l"(from) : "memory");
}

template <bool BF16, int G>
__global__ void __launch_bounds__(kWideBlockThreads, 1)
qlinear_wide_kernel(const __grid_constant__ CUtensorMap map_x, const LinearArgs a) {
  using S = WideShape;
  constexpr int NTOK = kWideTokens, ST = S::stages, NB = S::sums;
  constexpr int PG = kWideK / G;                      // groups of a stage
  constexpr int C = NTOK / 2;                        // tokens of a thread
  constexpr uint32_t idesc = umma_idesc_f16(kWideRowsOut, NTOK) | (BF16 ? (1u << 7) | (1u << 10) : 0u);
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~static_cast<uintptr_t>(1023));
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + S::bars_at);
  const uint32_t a_full = smem_u32(bars), a_empty = a_full + 8 * ST, x_full = a_empty + 8 * ST,
                 x_empty = x_full + 8 * ST, s_full = x_empty + 8 * ST, s_empty = s_full + 8 * NB;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + S::barriers);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int slices = gridDim.y, m0 = blockIdx.z * NTOK, tokens = min(NTOK, a.M - m0);
  const int b0 = blockIdx.y * a.slice;
  const int blocks = static_cast<int>(min(static_cast<int64_t>(a.slice), a.blocks - b0));
  const int n = (blocks + 1) / 2;                    // stages; the last may be half of one
  const int groups = (blocks * kBlockK + G - 1) / G;
  const int64_t tile0 = static_cast<int64_t>(blockIdx.x) * kWideTiles;
  const int64_t group0 = static_cast<int64_t>(b0) * kBlockK / G;
  if (threadIdx.x == 0) {
    for (int i = 0; i < ST; ++i) {
      mbar_init(a_full + 8 * i, kWideTiles);
      mbar_init(a_empty + 8 * i, 1);
      mbar_init(x_full + 8 * i, 1);
      mbar_init(x_empty + 8 * i, 1);
    }
    for (int i = 0; i < NB; ++i) mbar_init(s_full + 8 * i, 1);
    for (int i = 0; i < 2 * NB; ++i) mbar_init(s_empty + 8 * i, kAddThreads / 32);
    fence_mbar_init();
  }
  if (warp == kAddWarp) tmem_alloc(smem_u32(tmem_slot), 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  bool ok = true;
  // waits are warp-uniform; after a failure the warp stops waiting
  auto wait = [&](uint32_t bar, uint32_t phase) {
    if (ok) ok = __all_sync(0xFFFFFFFFu, wait_for(bar, phase, a.err)) != 0;
  };
  if (warp < kAddWarp) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
    // ---- weights: a warp's tile of 16 rows
    const int g = lane >> 2, t = lane & 3;
    const int64_t tile = tile0 + warp;
    const bool live = tile < a.tiles;
    // a lane copies the 16 bytes that it unpacks itself, `ahead` stages before; the first lanes a
    // group's zeros each
    constexpr int AH = S::ahead;
    const uint4* w = a.w + ((live ? tile : 0) * a.blocks + b0) * 32 + lane;
    const uint8_t* zr = reinterpret_cast<const uint8_t*>(a.zero) + ((live ? tile : 0) * a.groups + group0 + lane) * 16;
    uint8_t* wring = smem + S::w_at + warp * AH * S::w_bytes + lane * 16;
    uint8_t* zring = smem + S::z_at + warp * AH * S::z_bytes;
    auto fetch = [&](int s) {
      if (live && s < n) {
#pragma unroll
        for (int b = 0; b < 2; ++b)
          if (2 * s + b < blocks) copy16(wring + s % AH * S::w_bytes + b * kBlockBytes, w + (2 * s + b) * 32);
        if (a.zero && lane < PG && s * PG + lane < groups)
          copy16(zring + s % AH * S::z_bytes + lane * 16, zr + s * PG * 16);
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int s = 0; s < AH - 1; ++s) fetch(s);
    for (int s = 0; s < n; ++s) {
      const int st = s % ST;
      asm volatile("cp.async.wait_group %0;" ::"n"(AH - 2) : "memory");
      __syncwarp();                                  // (all lanes' zeros; and this place's last readers)
      fetch(s + AH - 1);
      if (s >= ST) wait(a_empty + 8 * st, (s / ST + 1) & 1);
      uint8_t* to = smem + st * S::a_bytes + (16 * warp + g) * 128;
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        if (!live || 2 * s + b >= blocks) continue;
        const uint4 x = *reinterpret_cast<const uint4*>(wring + s % AH * S::w_bytes + b * kBlockBytes);
        // halves in turns: rows g and g + 1 write to different banks
        const int odd = g & 1;
        const uint32_t words[2][2] = {{odd ? x.z : x.x, odd ? x.w : x.y}, {odd ? x.x : x.z, odd ? x.y : x.w}};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int group = (b * kBlockK + (h ^ odd) * 32) / G;
          const uint32_t zz = a.zero ? *reinterpret_cast<const uint16_t*>(zring + s % AH * S::z_bytes + group * 16 + g * 2)
                                     : 0x0808u;
          const uint32_t z0 = zz & 15, z1 = zz >> 8 & 15;
          uint32_t zl, zu;
          if constexpr (BF16) {
            zl = 0x3F803F80u | z0 << 3 | z0 << 19;
            zu = 0x3F803F80u | z1 << 3 | z1 << 19;
          } else {
            zl = z0 | z0 << 16;
            zu = z1 << 4 | z1 << 20;
          }
          uint32_t u[4], v[4];
          operands<BF16>(words[h][0], u);
          operands<BF16>(words[h][1], v);
          uint8_t* piece = to + b * kWideRowsOut * 128 + (((4 * (h ^ odd) + t) ^ g) << 4);
          *reinterpret_cast<uint4*>(piece) = make_uint4(minus<BF16>(u[0], zl), minus<BF16>(u[2], zl),
                                                        minus<BF16>(v[0], zl), minus<BF16>(v[2], zl));
          *reinterpret_cast<uint4*>(piece + 8 * 128) =       // rows g and g + 8
              make_uint4(minus<BF16>(u[1], zu), minus<BF16>(u[3], zu), minus<BF16>(v[1], zu),
                         minus<BF16>(v[3], zu));
        }
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(a_full + 8 * st);
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
  } else if (warp >= kProductsWarp) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
    if (warp == kTokensWarp && lane == 0) {
      // ---- tokens
      tma_prefetch_desc(&map_x);
      const uint64_t keep = l2_policy_evict_last();
      int s = 0;
      for (; s < n; ++s) {
        const int st = s % ST, two = 2 * s + 1 < blocks;
        if (s >= ST && !wait_for(x_empty + 8 * st, (s / ST + 1) & 1, a.err)) break;
        const uint32_t dst = smem_u32(smem + S::x_at + st * S::x_bytes);
        mbar_arrive_expect_tx(x_full + 8 * st, S::x_bytes >> (1 - two));
        for (int h = 0; h <= two; ++h)
          tma_load_2d(dst + h * NTOK * 128, &map_x, (b0 + 2 * s + h) * kBlockK, m0, x_full + 8 * st, keep);
      }
      for (int i = max(0, s - ST); i < s; ++i)       // the ring outlives its copies
        wait_for(x_full + 8 * (i % ST), (i / ST) & 1, a.err);
    } else if (warp < kTokensWarp && lane == 0) {
      // ---- products of every other stage
      int last = -1;
      for (int s = warp - kProductsWarp; s < n && ok; s += 2) {
        const int st = s % ST, steps = 2 * s + 1 < blocks ? 8 : 4;
        ok = wait_for(x_full + 8 * st, (s / ST) & 1, a.err) && wait_for(a_full + 8 * st, (s / ST) & 1, a.err);
        if (!ok) break;
        tc_fence_after();
        const uint64_t ad = umma_desc_sw128(smem_u32(smem + st * S::a_bytes));
        const uint64_t xd = umma_desc_sw128(smem_u32(smem + S::x_at + st * S::x_bytes));
#pragma unroll
        for (int k = 0; k < kWideK / 16; ++k) {
          if (k >= steps) break;
          const int q = s * PG + k * 16 / G;         // the group
          const bool first = k * 16 % G == 0, full = (k + 1) * 16 % G == 0;
          if (first && q >= NB && ok) {              // the place's last group is added
            ok = wait_for(s_empty + 8 * place_barrier(q - NB, NB), place_phase(q - NB, NB), a.err);
            tc_fence_after();
          }
          umma_f16(tmem + q % NB * NTOK, ad + (k / 4) * (kWideRowsOut * 128 >> 4) + (k % 4) * 2,
                   xd + (k / 4) * (NTOK * 128 >> 4) + (k % 4) * 2, idesc, !first);
          if (full) umma_commit(s_full + 8 * (q % NB));
        }
        umma_commit(a_empty + 8 * st);
        umma_commit(x_empty + 8 * st);
        last = s;
      }
      if (last >= 0) {                               // the block outlives its arrivals
        wait_for(a_empty + 8 * (last % ST), (last / ST) & 1, a.err);
        wait_for(x_empty + 8 * (last % ST), (last / ST) & 1, a.err);
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kAddRegs));
    // ---- sums: lanes 32 (warp % 4) .. + 31 of tensor memory, half of the columns
    const int rr = lane & 15, rows = warp & 3, half = (warp - kAddWarp) >> 2;
    const int64_t own = tile0 + 2 * rows + (lane >> 4);
    const uint16_t* sc = reinterpret_cast<const uint16_t*>(a.scale) +
                         ((own < a.tiles ? own : 0) * a.groups + group0) * 16 + (rr & 7) * 2 + (rr >> 3);
    const float unit = rr < 8 ? kUnit0<BF16> : kUnit1<BF16>;
    const uint32_t trow = tmem + (static_cast<uint32_t>(rows * 32) << 16) + half * C;
    float c[C];
#pragma unroll
    for (int i = 0; i < C; ++i) c[i] = 0.f;
    uint16_t next[NB];                               // the scales of the next groups
#pragma unroll
    for (int i = 0; i < NB; ++i) next[i] = i < groups ? sc[i * 16] : 0;
    for (int q0 = 0; q0 < groups; q0 += NB) {
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        const int q = q0 + i;
        if (q >= groups) break;
        const float f = unpack2<BF16>(next[i]).x * unit;
        if (q + NB < groups) next[i] = sc[(q + NB) * 16];
        wait(s_full + 8 * i, (q0 / NB) & 1);
        tc_fence_after();
#pragma unroll
        for (int h = 0; h < C; h += 32) {
          uint32_t v[32];
          tmem_ld32_nowait(trow + i * NTOK + h, v);
          tmem_wait_ld();
#pragma unroll
          for (int e = 0; e < 32; ++e) c[h + e] = fmaf(f, __uint_as_float(v[e]), c[h + e]);
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(s_empty + 8 * place_barrier(q, NB));
      }
    }
    // ---- all products are done: the operand's memory takes the rows as [token][row]
    auto barrier = [] { asm volatile("bar.sync 1, 256;" ::: "memory"); };
    float* part = reinterpret_cast<float*>(smem);
    barrier();
    float* to = part + half * C * S::pitch + rows * 32 + lane;
#pragma unroll
    for (int i = 0; i < C; ++i) to[i * S::pitch] = c[i];
    __syncwarp();
    if (warp == kAddWarp) tmem_dealloc(tmem, 512);
    if (slices > 1)
      cluster_sync_all();
    else
      barrier();
    finish_rows<BF16, kWideRowsOut, kAddThreads, S::pitch>(a, part, m0, tokens, slices, blockIdx.y, blockIdx.x,
                                                           threadIdx.x - 32 * kAddWarp);
    __syncwarp();
    if (slices > 1) cluster_sync_all();              // the peers have read this block's part
    return;
  }
  __syncwarp();
  if (slices > 1) {                                  // (both barriers want every thread)
    cluster_sync_all();
    cluster_sync_all();
  }
}

}  // namespace
}  // namespace gs
