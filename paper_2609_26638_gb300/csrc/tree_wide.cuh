// tree_wide.cuh -- tree attention for many query rows of a KV head: tcgen05
// products on tiles of 128 rows.
//
// With R rows per KV head a byte of the cache takes R flops or more, and beyond some
// tens the tensor cores bound it.  A block takes 128 rows, one KV head and one
// item of pages, 128 tokens (two pages) a step:
//
//   S = Q K^T    [128 rows][128 tokens] in tensor memory; Q and K from shared memory
//   P = 2^(S' - m), by four warps, one thread per row: a row is a lane of
//       tensor memory, so its maximum and sum never leave the thread
//   O += P V     P in tensor memory, over S's place; V^T pages from shared memory
//
// A fifth warp fetches pages by TMA (K, V^T as they lie in the cache: both are K-major
// operands), a sixth issues the products.  Two blocks per SM: one's softmax
// runs beside the other's products, and each block is a plain chain.
//
// m moves only when a row's maximum rises by more than 2^8 (O is rescaled then; the result
// does not depend on m but for rounding).  In fp16 it is set 7 below the
// maximum, so P stays below 2^15 and a weight of 2^-21 of the largest has all its
// bits, one of 2^-31 some.  P is rounded to the cache's type for the product, the
// sum takes it unrounded, in fp32.
//
// Steps that hold masked tokens clear, in shared memory, the values that no row
// sees.  Values that some rows see and that are not finite are taken out and added to
// those rows' O by hand.
#pragma once
#include "internal.h"
#include "tree_common.cuh"

namespace gs {
namespace {

constexpr int kWideRows = 128, kWideStep = 128;      // query rows of a block, tokens of a step
constexpr int kSoftWarps = 4, kSoftThreads = 128;
constexpr int kWideThreads = kSoftThreads + 64;      // + TMA warp, MMA warp
constexpr int kTmemCols = 256;                       // S (and P) 128, O up to 128
constexpr int kTmemO = 128;
constexpr float kRise = 8.f;                         // log2 units

template <int D>
struct WideSmem {
  static constexpr int H = D / 64;                   // 64-dim halves
  static constexpr int stages = D == 64 ? 2 : 1;
  static constexpr int q_bytes = H * kWideRows * 128;
  static constexpr int k_bytes = H * kWideStep * 128;   // [half][128 tokens][64 dims]
  static constexpr int v_bytes = 2 * D * 128;           // [page][dims][64 tokens]
  static constexpr int k_at = q_bytes, v_at = k_at + stages * k_bytes;
  static constexpr int bars_at = v_at + stages * v_bytes;
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

// 32 lanes x 16 columns into tensor memory.
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
      "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
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
  __shared__ uint32_t s_some[4][kSoftWarps], s_all[4][kSoftWarps], s_odd[4];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~static_cast<uintptr_t>(1023));
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + L::bars_at);
  const uint32_t k_full = smem_u32(bars), k_empty = k_full + 8 * ST, v_full = k_empty + 8 * ST,
                 v_empty = v_full + 8 * ST, q_full = v_empty + 8 * ST, s_full = q_full + 8,
                 p_full = s_full + 8, pv_done = p_full + 8;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 4 * ST + 4);
  pdl_trigger();   // the joining kernel may take its place; it waits for this one's end
  const int tree = blockIdx.z, head = blockIdx.y / a.tiles, tile = blockIdx.y % a.tiles;
  const int item = blockIdx.x;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const Span sp = find_span(a, tree);
  const int items = (sp.pages + a.split - 1) / a.split;
  const int rows = min(kWideRows, sp.count * a.G - tile * kWideRows);
  if (rows <= 0 || (item >= items && item > 0)) return;
  const int64_t row0 = static_cast<int64_t>(tree) * a.nodes;
  const int page_begin = sp.page0 + item * a.split;
  const int pages = max(0, min(a.split, sp.pages - item * a.split));
  const int steps = (pages + 1) / 2;
  const int tok_begin = page_begin * kPageTokens;
  const int limit = min(sp.keys, tok_begin + pages * kPageTokens);   // the item's tokens end here

  if (threadIdx.x == 0) {
    tma_prefetch_desc(&map_k);
    tma_prefetch_desc(&map_v);
    for (int i = 0; i < ST; ++i) {
      mbar_init(k_full + 8 * i, 1);
      mbar_init(k_empty + 8 * i, 1);
      mbar_init(v_full + 8 * i, 1);
      mbar_init(v_empty + 8 * i, 1);
    }
    mbar_init(q_full, kSoftWarps);
    mbar_init(s_full, 1);
    mbar_init(p_full, kSoftWarps);
    mbar_init(pv_done, 1);
    fence_mbar_init();
  }
  if (warp == kSoftWarps + 1) tmem_alloc(smem_u32(tmem_slot), kTmemCols);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  bool ok = true;

  if (warp == kSoftWarps) {
    // ---- TMA: K and V^T of two pages a step; lane l holds the page of place 32 i + l
    int ids = 0, k_issued = 0, v_issued = 0;
    for (int j = 0; j < steps && ok; ++j) {
      if (!((2 * j) & 31) && 2 * j + lane < pages) {
        ids = sp.table[page_begin + 2 * j + lane];
        if (ids < 0 || ids >= a.cache.n_pages) {
          atomicExch(a.err, kErrBounds);
          ids = 0;
        }
      }
      const int st = j % ST, two = 2 * j + 1 < pages;
      const int p0 = __shfl_sync(0xFFFFFFFFu, ids, (2 * j) & 31),
                p1 = __shfl_sync(0xFFFFFFFFu, ids, (2 * j + 1) & 31);
      if (lane == 0) {
        const uint32_t phase = (j / ST + 1) & 1;
        if (j >= ST) ok = mbar_wait(k_empty + 8 * st, phase, a.err);
        if (ok) {
          const uint32_t dst = smem_u32(smem + L::k_at + st * L::k_bytes);
          mbar_arrive_expect_tx(k_full + 8 * st, L::k_bytes >> (1 - two));
          for (int e = 0; e <= two; ++e)
            for (int h = 0; h < H; ++h)
              tma_load_4d(dst + h * kWideStep * 128 + e * kPageTokens * 128, &map_k, 0, h, 0,
                          2 * (e ? p1 : p0) * a.cache.Hkv + head, k_full + 8 * st);
          k_issued = j + 1;
          if (j >= ST) ok = mbar_wait(v_empty + 8 * st, phase, a.err);
        }
        if (ok) {
          const uint32_t dst = smem_u32(smem + L::v_at + st * L::v_bytes);
          mbar_arrive_expect_tx(v_full + 8 * st, L::v_bytes >> (1 - two));
          for (int e = 0; e <= two; ++e)
            tma_load_3d(dst + e * D * 128, &map_v, 0, 0, (2 * (e ? p1 : p0) + 1) * a.cache.Hkv + head,
                        v_full + 8 * st);
          v_issued = j + 1;
        }
      }
      ok = __shfl_sync(0xFFFFFFFFu, ok, 0);
    }
    // the block's shared memory outlives its copies
    if (lane == 0) {
      for (int j = max(0, k_issued - ST); j < k_issued; ++j)
        mbar_wait(k_full + 8 * (j % ST), (j / ST) & 1, a.err);
      for (int j = max(0, v_issued - ST); j < v_issued; ++j)
        mbar_wait(v_full + 8 * (j % ST), (j / ST) & 1, a.err);
    }
    __syncwarp();
  } else if (warp == kSoftWarps + 1) {
    // ---- products: S of step j + 1 follows O += P V of step j, which frees S's place
    if (lane == 0 && steps > 0) {
      const uint64_t qd = umma_desc_sw128(smem_u32(smem));
      auto scores = [&](int j) {
        const int st = j % ST;
        if (!mbar_wait(k_full + 8 * st, (j / ST) & 1, a.err)) return false;
        tc_fence_after();
        const uint64_t kd = umma_desc_sw128(smem_u32(smem + L::k_at + st * L::k_bytes));
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          const uint32_t at = (k / 4) * (kWideRows * 128 >> 4) + (k % 4) * 2;
          umma_f16(tmem, qd + at, kd + at, wide_idesc<BF16>(kWideStep), k > 0);
        }
        umma_commit(k_empty + 8 * st);
        umma_commit(s_full);
        return true;
      };
      ok = mbar_wait(q_full, 0, a.err) && scores(0);
      for (int j = 0; j < steps && ok; ++j) {
        const int st = j % ST;
        ok = mbar_wait(p_full, j & 1, a.err) && mbar_wait(v_full + 8 * st, (j / ST) & 1, a.err);
        if (!ok) break;
        tc_fence_after();
        const uint64_t vd = umma_desc_sw128(smem_u32(smem + L::v_at + st * L::v_bytes));
#pragma unroll
        for (int k = 0; k < kWideStep / 16; ++k)
          umma_f16_ta(tmem + kTmemO, tmem + 8 * k, vd + (k / 4) * (D * 128 >> 4) + (k % 4) * 2,
                      wide_idesc<BF16>(D));
        umma_commit(v_empty + 8 * st);
        umma_commit(pv_done);
        if (j + 1 < steps) ok = scores(j + 1);
      }
    }
    __syncwarp();
  } else {
    // ---- softmax: thread = row = lane of tensor memory
    const int r = threadIdx.x;
    const bool live = r < rows;
    const int node = live ? (tile * kWideRows + r) / a.G : 0;
    const int q_head = head * a.G + (live ? (tile * kWideRows + r) % a.G : 0);
    {
      const uint16_t* q = a.q + (row0 + node) * a.ld_q + static_cast<int64_t>(q_head) * D;
#pragma unroll
      for (int c = 0; c < D / 8; ++c) {
        const uint4 v = live ? *reinterpret_cast<const uint4*>(q + 8 * c) : make_uint4(0, 0, 0, 0);
        *reinterpret_cast<uint4*>(smem + (c / 8) * kWideRows * 128 + swizzled(r, c % 8)) = v;
      }
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
    auto view = [&](int tok) { return row_view(mask, lo, sp.n, tok) & bits_below(limit - tok); };
    // waits are warp-uniform; after a failure the warp stops waiting
    auto wait = [&](uint32_t bar, uint32_t phase) {
      if (ok) ok = __all_sync(0xFFFFFFFFu, mbar_wait(bar, phase, a.err)) != 0;
      return ok;
    };
    constexpr float kSet = BF16 ? 0.f : 7.f;         // how far below the maximum m is set
    float m = -INFINITY, l = 0.f;
    for (int j = 0; j < steps; ++j) {
      const int tok0 = tok_begin + j * kWideStep;
      const bool edge = tok0 < sp.lo_most || tok0 + kWideStep > min(sp.n, limit);
      wait(s_full, j & 1);
      tc_fence_after();
      float mx = -INFINITY;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        uint32_t s[32];
        tmem_ld32_nowait(trow + 32 * c, s);
        tmem_wait_ld();
        if (edge) {
          const uint32_t v = view(tok0 + 32 * c);
#pragma unroll
          for (int i = 0; i < 32; ++i)
            if (!((v >> i) & 1)) s[i] = 0xFF800000u;
        }
        float x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = __uint_as_float(s[e]);
#pragma unroll
        for (int i = 4; i < 28; i += 8)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            x[e] = max3(x[e], __uint_as_float(s[i + e]), __uint_as_float(s[i + 4 + e]));
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = fmaxf(x[e], __uint_as_float(s[28 + e]));
        mx = fmaxf(max3(mx, x[0], x[1]), fmaxf(x[2], x[3]));
      }
      mx *= a.scale_log2;
      const bool rise = mx - kSet > m + kRise || (m == -INFINITY && mx > m);
      if (__any_sync(0xFFFFFFFFu, rise)) {
        const float set = rise ? mx - kSet : m;
        const float f = rise ? ex2(m - set) : 1.f;   // (m = -inf: 0)
        l *= f;
        m = set;
        if (j > 0 && wait(pv_done, (j - 1) & 1)) {
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
          tmem_wait_st();
        }
      }
      const float z = finite_max(m);
      const F32x2 scale2 = join2(a.scale_log2, a.scale_log2), z2 = join2(-z, -z);
      F32x2 sum2 = join2(0.f, 0.f);
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        uint32_t s[32], p[16];
        tmem_ld32_nowait(trow + 32 * c, s);
        tmem_wait_ld();
        if (edge) {
          const uint32_t v = view(tok0 + 32 * c);
#pragma unroll
          for (int i = 0; i < 32; ++i)
            if (!((v >> i) & 1)) s[i] = 0xFF800000u;
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float2 e = split2(fma2(join2(__uint_as_float(s[2 * i]), __uint_as_float(s[2 * i + 1])),
                                       scale2, z2));
          const float x = ex2(e.x), y = ex2(e.y);
          sum2 = add2(sum2, join2(x, y));
          p[i] = pack2<BF16>(x, y);
        }
        tmem_st16(trow + 16 * c, p);
      }
      const float2 sum = split2(sum2);
      l += sum.x + sum.y;
      tmem_wait_st();
      if (edge) {
        // values that no row sees are cleared; those that are not finite and that
        // some rows see go to their O by hand
        const int st = j % ST;
        uint8_t* v = smem + L::v_at + st * L::v_bytes;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const uint32_t x = view(tok0 + 32 * w);
          const uint32_t some = __reduce_or_sync(0xFFFFFFFFu, live ? x : 0u),
                         all = __reduce_and_sync(0xFFFFFFFFu, live ? x : 0xFFFFFFFFu);
          if (lane == 0) s_some[w][warp] = some, s_all[w][warp] = all;
        }
        if (r < 4) s_odd[r] = 0u;
        wait(v_full + 8 * st, (j / ST) & 1);
        soft_barrier();
        // chunk = 8 tokens of a dim; word w of the step's tokens, byte b of the word
        for (int e = r; e < 2 * D * 8; e += kSoftThreads) {
          const int chunk = e % 8, dim = e / 8 % D, page = e / (8 * D);
          const int w = 2 * page + chunk / 4, shift = chunk % 4 * 8;
          uint32_t some = 0u, all = 0xFFFFFFFFu;
#pragma unroll
          for (int k = 0; k < kSoftWarps; ++k) some |= s_some[w][k], all &= s_all[w][k];
          const uint32_t keep = some >> shift, part = (some & ~all) >> shift;
          if ((keep & 0xFF) == 0xFF && !(part & 0xFF)) continue;
          uint4* at = reinterpret_cast<uint4*>(v + page * D * 128 + swizzled(dim, chunk));
          const uint4 x = *at;
          uint32_t word[4] = {x.x, x.y, x.z, x.w}, odd = 0u;
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            if (!((keep >> (2 * k)) & 1)) word[k] &= 0xFFFF0000u;
            if (!((keep >> (2 * k + 1)) & 1)) word[k] &= 0x0000FFFFu;
            const uint32_t nf = not_finite<BF16>(word[k]);
            odd |= ((nf & 1u) | (nf >> 30 & 2u)) << (2 * k) & part;
          }
          *at = make_uint4(word[0], word[1], word[2], word[3]);
          if (odd & 0xFFu) atomicOr(&s_odd[w], (odd & 0xFFu) << shift);
        }
        soft_barrier();
        if (s_odd[0] | s_odd[1] | s_odd[2] | s_odd[3]) {
          if (j > 0) wait(pv_done, (j - 1) & 1);
          tc_fence_after();
          for (int c = 0; c < D / 32; ++c) {
            uint32_t o[32];
            tmem_ld32_nowait(trow + kTmemO + 32 * c, o);
            tmem_wait_ld();
            for (int w = 0; w < 4; ++w)
              for (uint32_t left = s_odd[w] & view(tok0 + 32 * w); left; left &= left - 1) {
                const int tok = 32 * w + __ffs(left) - 1;
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                  const uint32_t h = *reinterpret_cast<const uint16_t*>(
                      v + tok / 64 * D * 128 + swizzled(32 * c + i, tok % 64 / 8) + tok % 8 * 2);
                  if (not_finite<BF16>(h))
                    o[i] = __float_as_uint(__uint_as_float(o[i]) + unpack2<BF16>(h).x);
                }
              }
            __syncwarp();
            tmem_st32(trow + kTmemO + 32 * c, o);
          }
          tmem_wait_st();
          soft_barrier();
          for (int e = r; e < 2 * D * 8; e += kSoftThreads) {
            const int chunk = e % 8, dim = e / 8 % D, page = e / (8 * D);
            const uint32_t odd = s_odd[2 * page + chunk / 4] >> (chunk % 4 * 8);
            if (!(odd & 0xFF)) continue;
            uint4* at = reinterpret_cast<uint4*>(v + page * D * 128 + swizzled(dim, chunk));
            const uint4 x = *at;
            uint32_t word[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const uint32_t sel = ((odd >> (2 * k)) & 1 ? 0x0000FFFFu : 0u) |
                                   ((odd >> (2 * k + 1)) & 1 ? 0xFFFF0000u : 0u);
              word[k] &= ~(not_finite<BF16>(word[k]) & sel);
            }
            *at = make_uint4(word[0], word[1], word[2], word[3]);
          }
        }
        fence_proxy_async_smem();
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(p_full);
    }
    // ---- the row's end
    if (steps > 0) wait(pv_done, (steps - 1) & 1);
    tc_fence_after();
    const int64_t row = row0 + node, at = row * a.Hq + q_head;
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {
      uint32_t o[32];
      tmem_ld32_nowait(trow + kTmemO + 32 * c, o);
      tmem_wait_ld();
      if (live && items <= 1) {
        const float inv = l != 0.f ? 1.f / l : 0.f;
        uint16_t* out = a.out + row * a.ld_out + static_cast<int64_t>(q_head) * D + 32 * c;
#pragma unroll
        for (int i = 0; i < 32; i += 8) {
          uint32_t w[4];
#pragma unroll
          for (int e = 0; e < 4; ++e)
            w[e] = pack2<BF16>(__uint_as_float(o[i + 2 * e]) * inv,
                               __uint_as_float(o[i + 2 * e + 1]) * inv);
          *reinterpret_cast<uint4*>(out + i) = make_uint4(w[0], w[1], w[2], w[3]);
        }
      } else if (live) {
        float* out = a.part_o + (at * a.items + item) * D + 32 * c;
#pragma unroll
        for (int i = 0; i < 32; i += 4)
          *reinterpret_cast<uint4*>(out + i) = make_uint4(o[i], o[i + 1], o[i + 2], o[i + 3]);
      }
      __syncwarp();
    }
    if (live) {
      if (items > 1)
        a.part_ml[at * a.items + item] = make_float2(m, l);
      else if (a.lse)
        a.lse[at] = l != 0.f ? (finite_max(m) + log2f(l)) * kLn2 : -INFINITY;
    }
    tc_fence_before();
  }
  __syncthreads();
  tc_fence_after();
  if (warp == kSoftWarps + 1) tmem_dealloc(tmem, kTmemCols);
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
