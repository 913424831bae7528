// tree_wide.cuh -- tree attention for many query rows of a KV head: tcgen05
// products on tiles of 128 rows.
//
// With R rows per KV head a byte of the cache takes R flops or more, and beyond some
// tens the tensor cores bound it.  A block takes 128 rows, one KV head and one
// item of pages, a page of 64 tokens a step:
//
//   S = Q K^T    [128 rows][64 tokens] in tensor memory; Q and K from shared memory
//   P = 2^(S' - m), by four warps, one thread per row: a row is a lane of
//       tensor memory, so its maximum and sum never leave the thread
//   O += P V     P in tensor memory, over S's place; V^T pages from shared memory
//
// A fifth warp fetches K by TMA and issues the S products, a sixth fetches V^T and
// issues the O products (both lie in the cache as K-major operands): the two
// chains run side by side, as do two blocks per SM.  S has two places, so that
// the products of the next page run during the softmax of this one.
//
// m moves only when a row's maximum rises by more than 2^8 (O is rescaled then; the result
// does not depend on m but for rounding).  In fp16 it is set 7 below the
// maximum, so P stays below 2^15 and a weight of 2^-21 of the largest has all its
// bits, one of 2^-31 some.  P is rounded to the cache's type for the product, the
// sum takes it unrounded, in fp32.
//
// Pages that hold masked tokens clear, in shared memory, the values that no row
// sees.  Values that some rows see and that are not finite are taken out and added to
// those rows' O by hand.
#pragma once
#include "internal.h"
#include "tree_common.cuh"

namespace gs {
namespace {

constexpr int kWideRows = 128;                       // query rows of a block
constexpr int kSoftWarps = 4, kSoftThreads = 128;
constexpr int kScoreWarp = kSoftWarps, kValueWarp = kSoftWarps + 1;
constexpr int kWideThreads = kSoftThreads + 64;      // (with one more warp, registers spill)
constexpr int kTmemCols = 256;                       // S (and P) twice 64, O up to 128
constexpr int kTmemO = 128;
constexpr float kRise = 8.f;                         // log2 units

template <int D>
struct WideSmem {
  static constexpr int H = D / 64;                   // 64-dim halves
  static constexpr int stages = D == 64 ? 4 : 2;
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

__device__ __forceinline__ void soft_barrier() {     // the softmax warps
  asm volatile("bar.sync 1, 128;" ::: "memory");
}

template <bool BF16, int D>
__global__ void __launch_bounds__(kWideThreads, 2)
tree_wide_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                 const TreeArgs a) {
  using L = WideSmem<D>;
  constexpr int H = L::H, ST = L::stages;
  extern __shared__ uint8_t smem_raw[];
  __shared__ uint32_t s_some[2][kSoftWarps], s_all[2][kSoftWarps], s_odd[2];
  __shared__ int64_t s_place[kWideRows];   // of each row: its query, then its output or part
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~static_cast<uintptr_t>(1023));
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + L::bars_at);
  const uint32_t k_full = smem_u32(bars), k_empty = k_full + 8 * ST, v_full = k_empty + 8 * ST,
                 v_empty = v_full + 8 * ST, s_full = v_empty + 8 * ST, p_full = s_full + 16,
                 pv_done = p_full + 16, q_full = pv_done + 16;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 4 * ST + 7);
  pdl_trigger();   // the joining kernel may take its place; it waits for this one's end
  const int tree = blockIdx.z, head = blockIdx.y / a.tiles, tile = blockIdx.y % a.tiles;
  const int item = blockIdx.x;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const Span sp = find_span(a, tree);
  const int items = (sp.pages + a.split - 1) / a.split;
  const int rows = min(kWideRows, sp.count * a.G - tile * kWideRows);
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0)
    a.part_n[tree] = make_int2(sp.pages, sp.count);
  if (rows <= 0 || (item >= items && item > 0)) return;
  const int64_t row0 = static_cast<int64_t>(tree) * a.nodes;
  const int page_begin = sp.page0 + item * a.split;
  const int pages = max(0, min(a.split, sp.pages - item * a.split));

  if (threadIdx.x == 0) {
    tma_prefetch_desc(&map_k);
    tma_prefetch_desc(&map_v);
    for (int i = 0; i < ST; ++i) {
      mbar_init(k_full + 8 * i, 1);
      mbar_init(k_empty + 8 * i, 1);
      mbar_init(v_full + 8 * i, 1);
      mbar_init(v_empty + 8 * i, 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(s_full + 8 * i, 1);
      mbar_init(p_full + 8 * i, kSoftWarps);
      mbar_init(pv_done + 8 * i, 1);
    }
    mbar_init(q_full, kSoftWarps);
    fence_mbar_init();
  }
  if (warp == kScoreWarp) tmem_alloc(smem_u32(tmem_slot), kTmemCols);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  bool ok = true;

  if (warp == kScoreWarp || warp == kValueWarp) {
    // ---- TMA and products.  Lane l holds the number of page 32 i + l.  A page's
    // place in the ring is filled again as soon as its products are done.
    const bool value = warp == kValueWarp;
    const uint32_t full = value ? v_full : k_full, empty = value ? v_empty : k_empty;
    const uint32_t ring = smem_u32(smem + (value ? L::v_at : L::k_at));
    const uint64_t qd = umma_desc_sw128(smem_u32(smem));
    int ids = 0, issued = 0;
    auto fetch = [&](int j) {              // (all lanes)
      if (j >= pages) return;
      if (!(j & 31) && j + lane < pages) {
        ids = sp.table[page_begin + j + lane];
        if (ids < 0 || ids >= a.cache.n_pages) {
          atomicExch(a.err, kErrBounds);
          ids = 0;
        }
      }
      const int page = __shfl_sync(0xFFFFFFFFu, ids, j & 31);
      if (lane == 0 && ok) {
        const int st = j % ST;
        const int block = (2 * page + value) * a.cache.Hkv + head;
        const uint32_t dst = ring + st * L::page_bytes, bar = full + 8 * st;
        if (j >= ST) ok = mbar_wait(empty + 8 * st, (j / ST + 1) & 1, a.err);
        if (ok) {
          mbar_arrive_expect_tx(bar, L::page_bytes);
          if (value) {
            tma_load_3d(dst, &map_v, 0, 0, block, bar);
          } else {
#pragma unroll
            for (int h = 0; h < H; ++h)
              tma_load_4d(dst + h * kPageTokens * 128, &map_k, 0, h, 0, block, bar);
          }
          issued = j + 1;
        }
      }
      __syncwarp();
    };
    for (int j = 0; j < ST; ++j) fetch(j);
    if (lane == 0 && !value && pages > 0) ok = mbar_wait(q_full, 0, a.err);
    for (int j = 0; j < pages; ++j) {
      const int st = j % ST, at = j & 1;
      if (lane == 0 && ok) {
        ok = mbar_wait(full + 8 * st, (j / ST) & 1, a.err);
        if (!value) {      // S of page j, where P of page j - 2 was
          ok = ok && (j < 2 || mbar_wait(pv_done + 8 * at, (j / 2 + 1) & 1, a.err));
          if (ok) {
            tc_fence_after();
            const uint64_t kd = umma_desc_sw128(ring + st * L::page_bytes);
#pragma unroll
            for (int k = 0; k < D / 16; ++k)
              umma_f16(tmem + 64 * at, qd + (k / 4) * (kWideRows * 128 >> 4) + (k % 4) * 2,
                       kd + (k / 4) * (kPageTokens * 128 >> 4) + (k % 4) * 2,
                       wide_idesc<BF16>(kPageTokens), k > 0);
            umma_commit(s_full + 8 * at);
            umma_commit(empty + 8 * st);
          }
        } else {           // O += P V
          ok = ok && mbar_wait(p_full + 8 * at, (j / 2) & 1, a.err);
          if (ok) {
            tc_fence_after();
            const uint64_t vd = umma_desc_sw128(ring + st * L::page_bytes);
#pragma unroll
            for (int k = 0; k < kPageTokens / 16; ++k)
              umma_f16_ta(tmem + kTmemO, tmem + 64 * at + 8 * k, vd + k * 2, wide_idesc<BF16>(D));
            umma_commit(pv_done + 8 * at);
            umma_commit(empty + 8 * st);
          }
        }
      }
      __syncwarp();
      fetch(j + ST);
    }
    // the block's shared memory outlives its copies
    if (lane == 0)
      for (int j = max(0, issued - ST); j < issued; ++j)
        mbar_wait(full + 8 * (j % ST), (j / ST) & 1, a.err);
    __syncwarp();
  } else {
    // ---- softmax: thread = row = lane of tensor memory
    const int r = threadIdx.x;
    const bool live = r < rows, busy = warp * 32 < rows;   // the row, any row of the warp is in use
    const int node = live ? (tile * kWideRows + r) / a.G : 0;
    const int q_head = head * a.G + (live ? (tile * kWideRows + r) % a.G : 0);
    // queries, a row's 16-byte pieces by neighbouring threads (rows not in use
    // hold anything: they meet no other)
    s_place[r] = live ? (row0 + node) * a.ld_q + static_cast<int64_t>(q_head) * D : -1;
    soft_barrier();
#pragma unroll 4
    for (int i = 0; i < D / 8; ++i) {
      const int e = r + i * kSoftThreads, row = e / (D / 8), c = e % (D / 8);
      const uint32_t to = smem_u32(smem) + (c / 8) * kWideRows * 128 + swizzled(row, c % 8);
      if (row < rows)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(a.q + s_place[row] + 8 * c)
                     : "memory");
    }
    const uint32_t trow = tmem + (static_cast<uint32_t>(warp * 32) << 16);
    {
      uint32_t zero[32];
#pragma unroll
      for (int i = 0; i < 32; ++i) zero[i] = 0u;
#pragma unroll
      for (int c = 0; c < D / 32; ++c) tmem_st32(trow + kTmemO + 32 * c, zero);
      tmem_wait_st();
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    fence_proxy_async_smem();
    tc_fence_before();
    __syncwarp();
    if (lane == 0) mbar_arrive(q_full);
    uint64_t mask = 0;
    int lo = sp.n;
    if (live) {
      mask = a.mask[row0 + node];
      if (sp.keys - sp.n < 64) mask &= (1ull << (sp.keys - sp.n)) - 1;
      lo = a.window > 0 ? min(max(first_key(a.pos[row0 + node], sp.n, a.window), sp.lo), sp.lo_most)
                        : 0;
    }
    // waits are warp-uniform; after a failure the warp stops waiting
    auto wait = [&](uint32_t bar, uint32_t phase) {
      if (ok) ok = __all_sync(0xFFFFFFFFu, mbar_wait(bar, phase, a.err)) != 0;
      return ok;
    };
    constexpr float kSet = BF16 ? 0.f : 7.f;         // how far below the maximum m is set
    const F32x2 scale2 = join2(a.scale_log2, a.scale_log2);
    float m = -INFINITY, l = 0.f;
    for (int j = 0; j < pages; ++j) {
      const int at = j & 1, tok0 = (page_begin + j) * kPageTokens;
      const bool edge = tok0 < sp.lo_most || tok0 + kPageTokens > sp.n;
      wait(s_full + 8 * at, (j / 2) & 1);
      tc_fence_after();
      if (busy) {
        uint32_t s[2][32];
        tmem_ld32_nowait(trow + 64 * at, s[0]);
        tmem_ld32_nowait(trow + 64 * at + 32, s[1]);
        tmem_wait_ld();
        if (edge) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint32_t v = row_view(mask, lo, sp.n, tok0 + 32 * h);
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
        const float mx = fmaxf(max3(x[0], x[1], x[2]), x[3]) * a.scale_log2;
        const bool rise = mx - kSet > m + kRise || (m == -INFINITY && mx > m);
        if (__any_sync(0xFFFFFFFFu, rise)) {
          const float set = rise ? mx - kSet : m;
          const float f = rise ? ex2(m - set) : 1.f;   // (m = -inf: 0)
          l *= f;
          m = set;
          if (j > 0 && wait(pv_done + 8 * (at ^ 1), ((j - 1) / 2) & 1)) {
            tc_fence_after();
#pragma unroll
            for (int c = 0; c < D / 32; ++c) {
              uint32_t o[32];
              tmem_ld32_nowait(trow + kTmemO + 32 * c, o);
              tmem_wait_ld();
#pragma unroll
              for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(f * __uint_as_float(o[i]));
              tmem_st32(trow + kTmemO + 32 * c, o);
            }
          }
        }
        const float z = finite_max(m);
        const F32x2 z2 = join2(-z, -z);
        F32x2 sum2[2] = {join2(0.f, 0.f), join2(0.f, 0.f)};
        uint32_t p[32];
#pragma unroll
        for (int i = 0; i < 32; ++i) {
          const float2 e = split2(fma2(join2(__uint_as_float(s[i / 16][2 * (i % 16)]),
                                             __uint_as_float(s[i / 16][2 * (i % 16) + 1])),
                                       scale2, z2));
          const float u = ex2(e.x), w = ex2(e.y);
          sum2[i & 1] = add2(sum2[i & 1], join2(u, w));
          p[i] = pack2<BF16>(u, w);
        }
        tmem_st32(trow + 64 * at, p);
        const float2 sum = split2(add2(sum2[0], sum2[1]));
        l += sum.x + sum.y;
        tmem_wait_st();
      }
      if (edge) {
        // values that no row sees are cleared; those that are not finite and that
        // some rows see go to their O by hand
        const int st = j % ST;
        uint8_t* v = smem + L::v_at + st * L::page_bytes;
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          const uint32_t x = row_view(mask, lo, sp.n, tok0 + 32 * w);
          const uint32_t some = __reduce_or_sync(0xFFFFFFFFu, live ? x : 0u),
                         all = __reduce_and_sync(0xFFFFFFFFu, live ? x : 0xFFFFFFFFu);
          if (lane == 0) s_some[w][warp] = some, s_all[w][warp] = all;
        }
        if (r < 2) s_odd[r] = 0u;
        wait(v_full + 8 * st, (j / ST) & 1);
        soft_barrier();
        // chunk = 8 tokens of a dim
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
          if (j > 0) wait(pv_done + 8 * (at ^ 1), ((j - 1) / 2) & 1);
          tc_fence_after();
          for (int c = 0; c < D / 32; ++c) {
            uint32_t o[32];
            tmem_ld32_nowait(trow + kTmemO + 32 * c, o);
            tmem_wait_ld();
            for (int w = 0; w < 2; ++w)
              for (uint32_t left = s_odd[w] & row_view(mask, lo, sp.n, tok0 + 32 * w); left;
                   left &= left - 1) {
                const int tok = 32 * w + __ffs(left) - 1;
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                  const uint32_t h = *reinterpret_cast<const uint16_t*>(
                      v + swizzled(32 * c + i, tok / 8) + tok % 8 * 2);
                  if (not_finite<BF16>(h))
                    o[i] = __float_as_uint(__uint_as_float(o[i]) + unpack2<BF16>(h).x);
                }
              }
            __syncwarp();
            tmem_st32(trow + kTmemO + 32 * c, o);
          }
          tmem_wait_st();
          soft_barrier();
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
    }
    // ---- the row's end
    if (pages > 0) wait(pv_done + 8 * ((pages - 1) & 1), ((pages - 1) / 2) & 1);
    tc_fence_after();
    // (the last O is done, and so are all products and copies: their shared
    // memory takes the rows, which are then written a row's pieces by neighbours)
    const int64_t row = row0 + node, at = row * a.Hq + q_head;
    constexpr int P = D + 4;
    float* so = reinterpret_cast<float*>(smem);
    const float inv = items > 1 ? 1.f : l != 0.f ? 1.f / l : 0.f;
    if (busy) {
#pragma unroll
      for (int c = 0; c < D / 32; ++c) {
        uint32_t o[32];
        tmem_ld32_nowait(trow + kTmemO + 32 * c, o);
        tmem_wait_ld();
#pragma unroll
        for (int i = 0; i < 32; i += 4)
          *reinterpret_cast<float4*>(so + r * P + 32 * c + i) =
              make_float4(__uint_as_float(o[i]) * inv, __uint_as_float(o[i + 1]) * inv,
                          __uint_as_float(o[i + 2]) * inv, __uint_as_float(o[i + 3]) * inv);
      }
    }
    if (live) {
      if (items > 1)
        a.part_ml[at * a.items + item] = make_float2(m, l);
      else if (a.lse)
        a.lse[at] = l != 0.f ? (finite_max(m) + log2f(l)) * kLn2 : -INFINITY;
      s_place[r] = items > 1 ? (at * a.items + item) * D : row * a.ld_out + static_cast<int64_t>(q_head) * D;
    }
    soft_barrier();
#pragma unroll 4
    for (int e = r; e < rows * (D / 4); e += kSoftThreads) {
      const int i = e / (D / 4), d = e % (D / 4) * 4;
      const float4 v = *reinterpret_cast<const float4*>(so + i * P + d);
      if (items > 1)
        *reinterpret_cast<float4*>(a.part_o + s_place[i] + d) = v;
      else
        *reinterpret_cast<uint2*>(a.out + s_place[i] + d) =
            make_uint2(pack2<BF16>(v.x, v.y), pack2<BF16>(v.z, v.w));
    }
    tc_fence_before();
  }
  __syncthreads();
  tc_fence_after();
  if (warp == kScoreWarp) tmem_dealloc(tmem, kTmemCols);
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
