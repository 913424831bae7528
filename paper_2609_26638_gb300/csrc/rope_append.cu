// rope_append.cu -- the step between a QKV projection and attention: RMS norm
// of every query and key head, rotary positions, and the write of keys and
// values into their cache pages, in one pass over the projected rows.
//
//   y = x * rsqrt(mean(x^2) + eps) * gain      (per head, over all D dims)
//   (a, b) -> (a cos - b sin, b cos + a sin)    (the pairs of the first R dims)
//
// Each row is read once and written once (queries to q_out, keys and values to
// their pages), so HBM bounds it; everything between is fp32 in registers and
// is rounded once at the store.  cos and sin come from a table that is built
// in 64 bits (gs_rope_table): the fp32 product position * frequency is off by
// up to 2^-25 of the angle, 0.004 rad at position 131,072.
#include <cmath>

#include "internal.h"
#include "step_common.cuh"

namespace gs {
namespace {

constexpr int kAppendThreads = 256;
constexpr int kHeadIters = 4;     // heads one lane group of a warp handles
constexpr int kVRows = 32;        // tokens of one V tile

struct AppendArgs {
  const uint16_t* qkv;
  int64_t ld_qkv;
  uint16_t* q_out;
  int64_t ld_q;
  const float2* table;
  int table_rows, half;
  const __nv_bfloat16 *q_gain, *k_gain;
  float eps;
  const int32_t *seq, *slot, *pos;
  int* err;
  int T, Hq, qk_blocks, chunks;   // chunks of heads per token in the Q/K part
  CacheView cache;
};

// The page and the slot in it that token `t` is written to; page -1 if it is
// not written (slot < 0, or something out of range: the error word is raised).
struct Target {
  int page, at;
};
__device__ __forceinline__ Target find_target(const AppendArgs& a, int t) {
  const int slot = a.slot[t], seq = a.seq[t];
  if (slot < 0) return {-1, 0};
  const int p = slot / kPageTokens;
  if (seq < 0 || seq >= a.cache.n_seq || p >= a.cache.pt_stride) {
    atomicExch(a.err, kErrBounds);
    return {-1, 0};
  }
  const int page = a.cache.page_table[static_cast<int64_t>(seq) * a.cache.pt_stride + p];
  if (page < 0 || page >= a.cache.n_pages) {
    atomicExch(a.err, kErrBounds);
    return {-1, 0};
  }
  return {page, slot % kPageTokens};
}

// Queries and keys.  A head's D dims lie on D / 8 neighbouring lanes, 16 bytes
// each, so a warp holds 32 / (D / 8) heads of one token at once and goes
// through kHeadIters such groups: its loads are issued together, and the
// lane's cos and sin are read once for all of them.  A half-layout pair sits
// on two lanes R / 16 apart: the partner's raw 16-bit values come by shuffle.
template <bool BF16, int D, bool HALF>
__device__ void rotate_heads(const AppendArgs& a) {
  constexpr int LPH = D / 8, HPW = 32 / LPH;
  const int lane = threadIdx.x & 31, sub = lane % LPH;
  const int warp = blockIdx.x * (kAppendThreads / 32) + (threadIdx.x >> 5);
  const int t = warp / a.chunks;
  if (t >= a.T) return;
  const int heads = a.Hq + a.cache.Hkv;
  const int h0 = (warp % a.chunks) * (HPW * kHeadIters) + lane / LPH;
  const uint16_t* row = a.qkv + t * a.ld_qkv + sub * 8;
  uint4 x[kHeadIters];
#pragma unroll
  for (int i = 0; i < kHeadIters; ++i) {
    const int h = h0 + i * HPW;
    x[i] = h < heads ? *reinterpret_cast<const uint4*>(row + h * D) : make_uint4(0, 0, 0, 0);
  }
  int pos = a.pos[t];
  if (pos < 0 || pos >= a.table_rows) {
    if (lane == 0) atomicExch(a.err, kErrBounds);
    pos = pos < 0 ? 0 : a.table_rows - 1;
  }
  const bool turns = sub * 8 < 2 * a.half;
  const bool second = HALF && sub * 8 >= a.half;
  const int partner = HALF && turns ? (second ? sub - a.half / 8 : sub + a.half / 8) : sub;
  float2 cs[HALF ? 8 : 4];
  if (turns) {
    const float2* r = a.table + static_cast<int64_t>(pos) * a.half +
                      (HALF ? sub * 8 - (second ? a.half : 0) : sub * 4);
#pragma unroll
    for (int e = 0; e < (HALF ? 8 : 4); e += 2) {
      const float4 v = *reinterpret_cast<const float4*>(r + e);
      cs[e] = make_float2(v.x, v.y);
      cs[e + 1] = make_float2(v.z, v.w);
    }
  }
  const Target to = find_target(a, t);
#pragma unroll
  for (int i = 0; i < kHeadIters; ++i) {
    const int h = h0 + i * HPW;
    const uint32_t raw[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
    float y[8];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float2 f = unpack2<BF16>(raw[e]);
      y[2 * e] = f.x;
      y[2 * e + 1] = f.y;
    }
    float z[8];   // the partner's values (half layout)
    if constexpr (HALF) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float2 f =
            unpack2<BF16>(__shfl_sync(0xFFFFFFFFu, raw[e], lane - sub + partner));
        z[2 * e] = f.x;
        z[2 * e + 1] = f.y;
      }
    }
    const __nv_bfloat16* gain = h < a.Hq ? a.q_gain : a.k_gain;
    if (a.q_gain) {
      float ss = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) ss = fmaf(y[e], y[e], ss);
#pragma unroll
      for (int m = 1; m < LPH; m *= 2) ss += __shfl_xor_sync(0xFFFFFFFFu, ss, m);
      const float r = rsqrtf(ss * (1.f / D) + a.eps);
      const uint4 g = *reinterpret_cast<const uint4*>(gain + sub * 8);
      const uint32_t gw[4] = {g.x, g.y, g.z, g.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float2 f = unpack2<true>(gw[e]);
        y[2 * e] *= r * f.x;
        y[2 * e + 1] *= r * f.y;
      }
      if constexpr (HALF) {
        const uint4 p = *reinterpret_cast<const uint4*>(gain + partner * 8);
        const uint32_t pw[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 f = unpack2<true>(pw[e]);
          z[2 * e] *= r * f.x;
          z[2 * e + 1] *= r * f.y;
        }
      }
    }
    if (turns) {
      if constexpr (HALF) {
        const float sign = second ? 1.f : -1.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = fmaf(y[e], cs[e].x, sign * z[e] * cs[e].y);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float p = y[2 * e], q = y[2 * e + 1];
          y[2 * e] = fmaf(p, cs[e].x, -q * cs[e].y);
          y[2 * e + 1] = fmaf(q, cs[e].x, p * cs[e].y);
        }
      }
    }
    if (h >= heads) continue;
    const uint4 o = make_uint4(pack2<BF16>(y[0], y[1]), pack2<BF16>(y[2], y[3]),
                               pack2<BF16>(y[4], y[5]), pack2<BF16>(y[6], y[7]));
    if (h < a.Hq) {
      *reinterpret_cast<uint4*>(a.q_out + t * a.ld_q + h * D + sub * 8) = o;
    } else if (to.page >= 0) {
      *reinterpret_cast<uint4*>(a.cache.block(to.page, 0, h - a.Hq, D) + to.at * D + sub * 8) = o;
    }
  }
}

// Values: a tile of 32 tokens of one KV head goes through shared memory and is
// written transposed.  Eight tokens that fill an aligned run of slots (same
// page, consecutive rows and slots, the first slot a multiple of 8) are one
// 16-byte store per dim, by the tile in which the run starts (it reads up to 7
// rows of the next tile); what is in no such run (single decode tokens, ragged
// ends) is stored element by element.  The row pitch D + 2 keeps the
// transposed reads off each other's banks.
template <int D>
__device__ void write_values(const AppendArgs& a) {
  constexpr int P = D + 2, kBack = 8, kSpan = kBack + kVRows + 8;
  __shared__ uint16_t tile[(kVRows + 8) * P];
  __shared__ Target to[kSpan];          // rows t0 - 8 .. t0 + 39
  __shared__ bool starts[kSpan];        // a full aligned run starts at this row
  __shared__ uint8_t run[kVRows], single[kVRows];
  __shared__ int n_run, n_single;
  const int block = blockIdx.x - a.qk_blocks;
  const int head = block % a.cache.Hkv, t0 = (block / a.cache.Hkv) * kVRows;
  const int rows = min(kVRows, a.T - t0);
  const uint16_t* src = a.qkv + (a.Hq + a.cache.Hkv + head) * D;
  auto load_rows = [&](int r0, int r1) {
    for (int v = r0 * (D / 8) + threadIdx.x; v < r1 * (D / 8); v += kAppendThreads) {
      const int r = v / (D / 8), c = v % (D / 8) * 8;
      const uint4 x = *reinterpret_cast<const uint4*>(src + (t0 + r) * a.ld_qkv + c);
      uint32_t* s = reinterpret_cast<uint32_t*>(tile + r * P + c);
      s[0] = x.x;
      s[1] = x.y;
      s[2] = x.z;
      s[3] = x.w;
    }
  };
  load_rows(0, rows);
  if (threadIdx.x < kSpan) {
    const int t = t0 - kBack + static_cast<int>(threadIdx.x);
    to[threadIdx.x] = t >= 0 && t < a.T ? find_target(a, t) : Target{-1, 0};
  }
  __syncthreads();
  if (threadIdx.x < kSpan) {
    const int i = threadIdx.x;
    bool ok = i + 8 <= kSpan && to[i].page >= 0 && to[i].at % 8 == 0;
    for (int j = 1; ok && j < 8; ++j)
      ok = to[i + j].page == to[i].page && to[i + j].at == to[i].at + j;
    starts[i] = ok;
  }
  __syncthreads();
  if (threadIdx.x < kVRows) {
    const int i = kBack + threadIdx.x, first = i - to[i].at % 8;
    const bool written = static_cast<int>(threadIdx.x) < rows && to[i].page >= 0;
    // row `first` starts the run that this row's slot lies in, if it is one
    const bool in_run = written && starts[first] && to[first].page == to[i].page &&
                        to[first].at == to[i].at - (i - first);
    const uint32_t below = (1u << threadIdx.x) - 1u;
    const uint32_t r = __ballot_sync(0xFFFFFFFFu, written && starts[i]);
    const uint32_t s = __ballot_sync(0xFFFFFFFFu, written && !in_run);
    if (r >> threadIdx.x & 1) run[__popc(r & below)] = threadIdx.x;
    if (s >> threadIdx.x & 1) single[__popc(s & below)] = threadIdx.x;
    if (threadIdx.x == 0) {
      n_run = __popc(r);
      n_single = __popc(s);
    }
  }
  __syncthreads();
  const int last = n_run ? run[n_run - 1] + 8 : 0;
  if (last > kVRows) {                  // a run that ends in the next tile
    load_rows(kVRows, last);
    __syncthreads();
  }
  for (int w = threadIdx.x; w < D * n_run; w += kAppendThreads) {
    const int d = w / n_run, r = run[w % n_run];
    uint32_t p[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      p[i] = tile[(r + 2 * i) * P + d] | static_cast<uint32_t>(tile[(r + 2 * i + 1) * P + d]) << 16;
    const Target at = to[kBack + r];
    *reinterpret_cast<uint4*>(a.cache.block(at.page, 1, head, D) + d * kPageTokens + at.at) =
        make_uint4(p[0], p[1], p[2], p[3]);
  }
  for (int w = threadIdx.x; w < n_single * D; w += kAppendThreads) {
    const int r = single[w / D], d = w % D;
    const Target at = to[kBack + r];
    a.cache.block(at.page, 1, head, D)[d * kPageTokens + at.at] = tile[r * P + d];
  }
}

template <bool BF16, int D, bool HALF>
__global__ void __launch_bounds__(kAppendThreads) rope_append_kernel(const AppendArgs a) {
  if (static_cast<int>(blockIdx.x) < a.qk_blocks)
    rotate_heads<BF16, D, HALF>(a);
  else
    write_values<D>(a);
}

template <bool BF16, int D>
void launch_append(const AppendArgs& a, bool half, int blocks, cudaStream_t s) {
  if (half)
    rope_append_kernel<BF16, D, true><<<blocks, kAppendThreads, 0, s>>>(a);
  else
    rope_append_kernel<BF16, D, false><<<blocks, kAppendThreads, 0, s>>>(a);
}

struct Frequencies {
  double inv[64];
};

// One (cos, sin) pair per thread, in 64 bits; rounded once.
__global__ void rope_table_kernel(Frequencies f, double magnitude, int rows, int half, float2* table) {
  const int64_t i = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x;
  if (i >= static_cast<int64_t>(rows) * half) return;
  double s, c;
  sincos(static_cast<double>(i / half) * f.inv[i % half], &s, &c);
  table[i] = make_float2(static_cast<float>(c * magnitude), static_cast<float>(s * magnitude));
}

}  // namespace
}  // namespace gs

extern "C" int gs_rope_table(const gs_rope_scaling* sc, int rotary_dim, int rows, void* table,
                             void* stream) {
  using namespace gs;
  if (!sc || !table || !aligned16(table) || rows < 1 || rotary_dim < 16 || rotary_dim > 128 ||
      rotary_dim % 16 || !(sc->theta > 1.f) || !std::isfinite(sc->theta))
    return GS_ERR_INVALID_ARG;
  if (sc->kind < GS_ROPE_PLAIN || sc->kind > GS_ROPE_YARN) return GS_ERR_INVALID_ARG;
  if (sc->kind != GS_ROPE_PLAIN && (!(sc->factor >= 1.f) || !std::isfinite(sc->factor)))
    return GS_ERR_INVALID_ARG;
  if (sc->kind == GS_ROPE_YARN &&
      (sc->original_ctx < 1 || !(sc->beta_fast > sc->beta_slow) || !(sc->beta_slow > 0.f) ||
       !std::isfinite(sc->beta_fast) || !(sc->magnitude >= 0.f) || !std::isfinite(sc->magnitude)))
    return GS_ERR_INVALID_ARG;
  const int half = rotary_dim / 2;
  const double R = rotary_dim, factor = sc->kind == GS_ROPE_PLAIN ? 1.0 : sc->factor;
  double theta = sc->theta, magnitude = 1.0;
  if (sc->kind == GS_ROPE_NTK) theta *= std::pow(factor, R / (R - 2.0));
  // YaRN: the (real-valued) pair whose wave makes `turns` turns in the original context
  const double two_pi = 6.283185307179586476925;
  auto pair_of = [&](double turns) {
    return R * std::log(sc->original_ctx / (turns * two_pi)) / (2.0 * std::log(theta));
  };
  double lo = 0.0, hi = 0.0;
  if (sc->kind == GS_ROPE_YARN) {
    lo = std::fmax(std::floor(pair_of(sc->beta_fast)), 0.0);
    hi = std::fmin(std::ceil(pair_of(sc->beta_slow)), R - 1.0);
    if (hi <= lo) hi = lo + 0.001;
    magnitude = sc->magnitude > 0.f ? sc->magnitude : 0.1 * std::log(factor) + 1.0;
  }
  Frequencies f;
  for (int i = 0; i < half; ++i) {
    const double plain = std::pow(theta, -2.0 * i / R);
    double stretched = 0.0;   // the share of the frequency that is divided by the factor
    if (sc->kind == GS_ROPE_LINEAR) stretched = 1.0;
    if (sc->kind == GS_ROPE_YARN) stretched = std::fmin(std::fmax((i - lo) / (hi - lo), 0.0), 1.0);
    f.inv[i] = plain * (1.0 - stretched) + plain / factor * stretched;
  }
  const int64_t n = static_cast<int64_t>(rows) * half;
  rope_table_kernel<<<static_cast<unsigned>((n + 255) / 256), 256, 0,
                      static_cast<cudaStream_t>(stream)>>>(f, magnitude, rows, half,
                                                           static_cast<float2*>(table));
  return cudaGetLastError() == cudaSuccess ? GS_OK : GS_ERR_CUDA;
}

extern "C" int gs_rope_append(const gs_cache* cache, const gs_rope* rope, const void* qkv,
                              int64_t ld_qkv, int T, int n_heads, const void* q_gain,
                              const void* k_gain, float eps, const int32_t* seq,
                              const int32_t* slot, const int32_t* pos, void* q_out, int64_t ld_q,
                              int32_t* err, void* stream) {
  using namespace gs;
  if (const int rc = check_cache(cache)) return rc;
  if (!rope || !rope->table || !aligned16(rope->table) || rope->table_rows < 1 ||
      (rope->layout != GS_ROPE_HALF && rope->layout != GS_ROPE_INTERLEAVED))
    return GS_ERR_INVALID_ARG;
  const int D = cache->head_dim, Hkv = cache->n_kv_heads;
  if (rope->rotary_dim < 16 || rope->rotary_dim > D || rope->rotary_dim % 16)
    return GS_ERR_INVALID_ARG;
  if (!qkv || !seq || !slot || !pos || !q_out || !err || T < 0 || n_heads < 1 || n_heads % Hkv)
    return GS_ERR_INVALID_ARG;
  if (!q_gain != !k_gain || !(eps >= 0.f)) return GS_ERR_INVALID_ARG;
  const int64_t width = (static_cast<int64_t>(n_heads) + 2 * Hkv) * D;
  if (width > (1 << 24)) return GS_ERR_UNSUPPORTED;
  if (ld_qkv < width || ld_q < static_cast<int64_t>(n_heads) * D || ld_qkv % 8 || ld_q % 8 ||
      !aligned16(qkv) || !aligned16(q_out) || !aligned16(q_gain) || !aligned16(k_gain) ||
      (q_out == qkv && ld_q != ld_qkv))
    return GS_ERR_INVALID_ARG;
  if (T == 0) return GS_OK;
  const int per_warp = 32 / (D / 8) * kHeadIters;
  AppendArgs a;
  a.qkv = static_cast<const uint16_t*>(qkv);
  a.ld_qkv = ld_qkv;
  a.q_out = static_cast<uint16_t*>(q_out);
  a.ld_q = ld_q;
  a.table = static_cast<const float2*>(rope->table);
  a.table_rows = rope->table_rows;
  a.half = rope->rotary_dim / 2;
  a.q_gain = static_cast<const __nv_bfloat16*>(q_gain);
  a.k_gain = static_cast<const __nv_bfloat16*>(k_gain);
  a.eps = eps;
  a.seq = seq;
  a.slot = slot;
  a.pos = pos;
  a.err = err;
  a.T = T;
  a.Hq = n_heads;
  a.chunks = (n_heads + Hkv + per_warp - 1) / per_warp;
  a.cache = cache_view(*cache);
  constexpr int warps = kAppendThreads / 32;
  const int64_t qk_blocks = (static_cast<int64_t>(T) * a.chunks + warps - 1) / warps;
  const int64_t blocks = qk_blocks + static_cast<int64_t>((T + kVRows - 1) / kVRows) * Hkv;
  if (static_cast<int64_t>(T) * a.chunks + warps >= (1ll << 31) || blocks >= (1ll << 31))
    return GS_ERR_UNSUPPORTED;
  a.qk_blocks = static_cast<int>(qk_blocks);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const bool half = rope->layout == GS_ROPE_HALF;
  const int n = static_cast<int>(blocks);
  if (cache->dtype == GS_BF16)
    D == 64 ? launch_append<true, 64>(a, half, n, s) : launch_append<true, 128>(a, half, n, s);
  else
    D == 64 ? launch_append<false, 64>(a, half, n, s) : launch_append<false, 128>(a, half, n, s);
  return cudaGetLastError() == cudaSuccess ? GS_OK : GS_ERR_CUDA;
}
