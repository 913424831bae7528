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
//
// Measured: 8191 prompt tokens (32 query and 8 KV heads of 128, bf16, norm, full
// rotation) 37 us, 5.5 TB/s, with issue slots 58% busy and the loads' latency the
// largest stall (45 us with blocks of 256 threads, whose warps end together; 38
// with 16 instead of 8 heads a lane group); a batch of 256 single tokens 4.3 us;
// one token 2.7 us, the launch.
#include <cmath>

#include "internal.h"
#include "step_common.cuh"

namespace gs {
namespace {

constexpr int kAppendThreads = 128;
constexpr int kAhead = 4;         // heads of a lane group that are loaded together
constexpr int kVRows = 32;        // tokens of one V tile at most

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
  int T, Hq, v_blocks, iters;
  int v_rows, v_heads;            // tokens of a V tile, KV heads that its block takes in turn
  int q_chunks, chunks;           // a token's chunks of query heads, and of all heads, in the Q/K part
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

// Queries and keys.  A head's D dims lie on D / 8 neighbouring lanes, so a warp
// holds 32 / (D / 8) heads of one token at once and goes through `iters` such
// groups, all of queries or all of keys, four at a time.  A lane's eight dims are
// two fours a and b: neighbours, or in the half layout dims i and i + R / 2, so
// that pairs never lie on two lanes.  Gain and rotation are the same for all
// heads; they are made into two factors per element once, and two elements go
// through each instruction:
//   out_a = rsqrt(...) * (a * A_a + b * B_a),  A = gain cos, B = -+ partner's gain sin
template <bool BF16, int D, bool HALF>
__device__ void rotate_heads(const AppendArgs& a) {
  constexpr int LPH = D / 8, HPW = 32 / LPH;
  const int lane = threadIdx.x & 31, sub = lane % LPH;
  const int warp = (blockIdx.x - a.v_blocks) * (kAppendThreads / 32) + (threadIdx.x >> 5);
  const int t = warp / a.chunks, chunk = warp % a.chunks;
  if (t >= a.T) return;
  const bool keys = chunk >= a.q_chunks;
  // heads h0, h0 + HPW, ... below `heads`, of the queries or of the keys
  const int first = (keys ? chunk - a.q_chunks : chunk) * HPW * a.iters;
  const int h0 = first + lane / LPH;
  const int heads = keys ? a.cache.Hkv : a.Hq;
  const int iters = min(a.iters, (heads - first + HPW - 1) / HPW);
  const int mine = min(iters, (heads - h0 + HPW - 1) / HPW);   // of them, with a head for this lane
  const bool turns = sub * 8 < 2 * a.half;
  const int da = HALF && turns ? sub * 4 : sub * 8, db = HALF && turns ? a.half + sub * 4 : da + 4;
  const uint16_t* src = a.qkv + t * a.ld_qkv + ((keys ? a.Hq : 0) + h0) * D + da;
  uint2 xa[kAhead], xb[kAhead];
  auto load = [&](int i0) {   // the next kAhead heads
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      xa[i] = xb[i] = make_uint2(0, 0);
      if (i0 + i < mine) {
        xa[i] = *reinterpret_cast<const uint2*>(src + i * HPW * D);
        xb[i] = *reinterpret_cast<const uint2*>(src + i * HPW * D + (db - da));
      }
    }
    src += kAhead * HPW * D;
  };
  load(0);
  int pos = a.pos[t];
  if (pos < 0 || pos >= a.table_rows) {
    if (lane == 0) atomicExch(a.err, kErrBounds);
    pos = pos < 0 ? 0 : a.table_rows - 1;
  }
  const __nv_bfloat16* gain = keys ? a.k_gain : a.q_gain;
  float A[8], B[8];   // of a's four elements, then of b's
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    A[e] = 1.f;
    B[e] = 0.f;
  }
  if (turns) {
    const float4* r = reinterpret_cast<const float4*>(a.table + static_cast<int64_t>(pos) * a.half +
                                                      sub * 4);
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const float4 v = r[e];   // cos, sin of the lane's pairs 2e and 2e + 1
      if constexpr (HALF) {
        A[2 * e] = A[4 + 2 * e] = v.x;
        A[2 * e + 1] = A[5 + 2 * e] = v.z;
        B[2 * e] = -v.y;
        B[2 * e + 1] = -v.w;
        B[4 + 2 * e] = v.y;
        B[5 + 2 * e] = v.w;
      } else {
        A[4 * e] = A[4 * e + 1] = v.x;
        A[4 * e + 2] = A[4 * e + 3] = v.z;
        B[4 * e] = -v.y;
        B[4 * e + 1] = v.y;
        B[4 * e + 2] = -v.w;
        B[4 * e + 3] = v.w;
      }
    }
  }
  if (gain) {
    const uint2 ga = *reinterpret_cast<const uint2*>(gain + da);
    const uint2 gb = *reinterpret_cast<const uint2*>(gain + db);
    const float2 g[4] = {unpack2<true>(ga.x), unpack2<true>(ga.y), unpack2<true>(gb.x),
                         unpack2<true>(gb.y)};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float2 q = HALF ? g[e ^ 2] : make_float2(g[e].y, g[e].x);   // the partners'
      A[2 * e] *= g[e].x;
      A[2 * e + 1] *= g[e].y;
      B[2 * e] *= q.x;
      B[2 * e + 1] *= q.y;
    }
  }
  F32x2 A2[4], B2[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    A2[e] = join2(A[2 * e], A[2 * e + 1]);
    B2[e] = join2(B[2 * e], B[2 * e + 1]);
  }
  // where the lane's first head goes, and from there the next one; how many go
  uint16_t* out;
  int64_t step = HPW * D;
  int stored = mine;
  if (!keys) {
    out = a.q_out + t * a.ld_q + h0 * D + da;
  } else {
    const Target to = find_target(a, t);
    if (to.page < 0) stored = 0;
    out = a.cache.block(max(to.page, 0), 0, h0, D) + to.at * D + da;
    step = HPW * (kPageTokens * D);
  }
#pragma unroll 1
  for (int i0 = 0; i0 < iters; i0 += kAhead) {
    if (i0) load(i0);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const float2 f[4] = {unpack2<BF16>(xa[i].x), unpack2<BF16>(xa[i].y), unpack2<BF16>(xb[i].x),
                           unpack2<BF16>(xb[i].y)};
      F32x2 y[4], ss = join2(0.f, 0.f);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        y[e] = join2(f[e].x, f[e].y);
        ss = fma2(y[e], y[e], ss);
      }
      float r = 1.f;
      if (gain) {
        const float2 s2 = split2(ss);
        float s = s2.x + s2.y;
#pragma unroll
        for (int m = 1; m < LPH; m *= 2) s += __shfl_xor_sync(0xFFFFFFFFu, s, m);
        r = rsqrtf(s * (1.f / D) + a.eps);
      }
      const F32x2 r2 = join2(r, r);
      F32x2 v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = mul2(y[e], A2[e]);
      if (turns) {   // (else B is 0, but the partner may be infinite)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          v[e] = fma2(HALF ? y[e ^ 2] : join2(f[e].y, f[e].x), B2[e], v[e]);
      }
      uint32_t o[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float2 w = split2(mul2(v[e], r2));
        o[e] = pack2<BF16>(w.x, w.y);
      }
      if (i0 + i < stored) {
        *reinterpret_cast<uint2*>(out) = make_uint2(o[0], o[1]);
        *reinterpret_cast<uint2*>(out + (db - da)) = make_uint2(o[2], o[3]);
      }
      out += step;
    }
  }
}

// Values: a tile of up to 32 tokens of one KV head goes through shared memory and is
// written transposed.  Eight tokens that fill an aligned run of slots (same
// page, consecutive rows and slots, the first slot a multiple of 8) are one
// 16-byte store per dim, by the tile in which the run starts (it reads up to 7
// rows of the next tile); what is in no such run (single decode tokens, ragged
// ends) is stored element by element.  The row pitch D + 2 keeps the
// transposed reads off each other's banks.
template <int D>
__device__ void write_values(const AppendArgs& a) {
  constexpr int P = D + 2, kBack = 8, kSpan = kBack + kVRows + 8;
  __shared__ alignas(16) uint16_t tile[(kVRows + 8) * P];
  __shared__ Target to[kSpan];          // rows t0 - 8 .. t0 + 39
  __shared__ bool starts[kSpan];        // a full aligned run starts at this row
  __shared__ uint8_t run[kVRows], single[kVRows];
  __shared__ int n_run, n_single;
  const int block = blockIdx.x, groups = (a.cache.Hkv + a.v_heads - 1) / a.v_heads;
  const int head0 = block % groups * a.v_heads, t0 = (block / groups) * a.v_rows;
  const int rows = min(a.v_rows, a.T - t0);
  auto load_rows = [&](int head, int r0, int r1) {
    const uint16_t* src = a.qkv + (a.Hq + a.cache.Hkv + head) * D;
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
  load_rows(head0, 0, rows);
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
  const int last = n_run ? run[n_run - 1] + 8 : 0;   // past v_rows: a run that ends in the next tile
  for (int head = head0; head < min(head0 + a.v_heads, a.cache.Hkv); ++head) {
    if (head > head0) {
      __syncthreads();                 // the tile has been read
      load_rows(head, 0, max(rows, last));
      __syncthreads();
    } else if (last > a.v_rows) {
      load_rows(head, a.v_rows, last);
      __syncthreads();
    }
    // at most four runs of eight rows start in a tile; two dims at a time
    for (int w = threadIdx.x; w < D / 2 * 4; w += kAppendThreads) {
      if ((w & 3) >= n_run) continue;
      const int d = w >> 2, r = run[w & 3];
      const uint32_t* s = reinterpret_cast<const uint32_t*>(tile) + r * (P / 2) + d;
      uint32_t lo[4], hi[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t u = s[2 * i * (P / 2)], v = s[(2 * i + 1) * (P / 2)];
        lo[i] = __byte_perm(u, v, 0x5410);
        hi[i] = __byte_perm(u, v, 0x7632);
      }
      const Target at = to[kBack + r];
      uint16_t* out = a.cache.block(at.page, 1, head, D) + 2 * d * kPageTokens + at.at;
      *reinterpret_cast<uint4*>(out) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
      *reinterpret_cast<uint4*>(out + kPageTokens) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
    }
    for (int w = threadIdx.x; w < n_single * D; w += kAppendThreads) {
      const int r = single[w / D], d = w % D;
      const Target at = to[kBack + r];
      a.cache.block(at.page, 1, head, D)[d * kPageTokens + at.at] = tile[r * P + d];
    }
  }
}

template <bool BF16, int D, bool HALF>
__global__ void __launch_bounds__(kAppendThreads, 8) rope_append_kernel(const AppendArgs a) {
  // the values' blocks take longest: they come first
  if (static_cast<int>(blockIdx.x) < a.v_blocks)
    write_values<D>(a);
  else
    rotate_heads<BF16, D, HALF>(a);
}

template <bool BF16, int D>
cudaError_t launch_append(const AppendArgs& a, bool half, int blocks, cudaStream_t s) {
  return launch_ex(half ? rope_append_kernel<BF16, D, true> : rope_append_kernel<BF16, D, false>,
                   dim3(blocks), dim3(kAppendThreads), 0, s, false, dim3(1, 1, 1), a);
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
  if (!q_gain != !k_gain || !(eps >= 0.f) || !aligned4(seq, slot, pos, err))
    return GS_ERR_INVALID_ARG;
  const int64_t width = (static_cast<int64_t>(n_heads) + 2 * Hkv) * D;
  if (width > (1 << 24)) return GS_ERR_UNSUPPORTED;
  if (ld_qkv < width || ld_q < static_cast<int64_t>(n_heads) * D || ld_qkv % 8 || ld_q % 8 ||
      !aligned16(qkv) || !aligned16(q_out) || !aligned16(q_gain) || !aligned16(k_gain) ||
      (q_out == qkv && ld_q != ld_qkv))
    return GS_ERR_INVALID_ARG;
  if (T == 0) return GS_OK;
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
  // A warp takes twice as many heads where that still leaves two waves of warps
  // (32 an SM): what it sets up for a token then serves more of them.
  const int hpw = 32 / (D / 8);
  for (a.iters = 2 * kAhead;; a.iters /= 2) {
    a.q_chunks = (n_heads + hpw * a.iters - 1) / (hpw * a.iters);
    a.chunks = a.q_chunks + (Hkv + hpw * a.iters - 1) / (hpw * a.iters);
    if (a.iters == kAhead || static_cast<int64_t>(T) * a.chunks >= 2 * 32 * kNumSMs) break;
  }
  // a decode batch's values are scattered 2-byte stores: small tiles on many SMs
  a.v_rows = static_cast<int64_t>(T) * Hkv >= kVRows * kNumSMs ? kVRows : 8;
  a.v_heads = static_cast<int64_t>((T + kVRows - 1) / kVRows) * Hkv >= 8 * kNumSMs ? 4 : 1;
  a.cache = cache_view(*cache);
  constexpr int warps = kAppendThreads / 32;
  const int64_t qk_blocks = (static_cast<int64_t>(T) * a.chunks + warps - 1) / warps;
  const int64_t v_blocks =
      static_cast<int64_t>((T + a.v_rows - 1) / a.v_rows) * ((Hkv + a.v_heads - 1) / a.v_heads);
  const int64_t blocks = qk_blocks + v_blocks;
  if (static_cast<int64_t>(T) * a.chunks + warps >= (1ll << 31) || blocks >= (1ll << 31))
    return GS_ERR_UNSUPPORTED;
  a.v_blocks = static_cast<int>(v_blocks);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const bool half = rope->layout == GS_ROPE_HALF;
  const int n = static_cast<int>(blocks);
  cudaError_t e;
  if (cache->dtype == GS_BF16)
    e = D == 64 ? launch_append<true, 64>(a, half, n, s) : launch_append<true, 128>(a, half, n, s);
  else
    e = D == 64 ? launch_append<false, 64>(a, half, n, s) : launch_append<false, 128>(a, half, n, s);
  return e == cudaSuccess ? GS_OK : GS_ERR_CUDA;
}
