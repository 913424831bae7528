// step_common.cuh -- what the single-token step operators share: 16-bit
// element types, the paged cache as kernels see it, and host-side checks.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <mutex>

#include "ptx.cuh"
#include "../../include/gs.h"

namespace gs {

constexpr int kPageTokens = 64;

// Packed pairs of 16-bit elements <-> fp32.
template <bool BF16>
__device__ __forceinline__ float2 unpack2(uint32_t v) {
  if constexpr (BF16) {
    return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xFFFF0000u));
  } else {
    __half2 h;
    memcpy(&h, &v, 4);
    return __half22float2(h);
  }
}

template <bool BF16>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  uint32_t r;
  if constexpr (BF16) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    memcpy(&r, &h, 4);
  } else {
    const __half2 h = __floats2half2_rn(a, b);
    memcpy(&r, &h, 4);
  }
  return r;
}

// Two fp32 values in a 64-bit register pair: one instruction for both.
typedef unsigned long long F32x2;
__device__ __forceinline__ F32x2 join2(float a, float b) {
  F32x2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float2 split2(F32x2 v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}
__device__ __forceinline__ F32x2 mul2(F32x2 a, F32x2 b) {
  F32x2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ F32x2 fma2(F32x2 a, F32x2 b, F32x2 c) {
  F32x2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}

__device__ __forceinline__ F32x2 add2(F32x2 a, F32x2 b) {
  F32x2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
// rounded toward zero
__device__ __forceinline__ F32x2 add2_rz(F32x2 a, F32x2 b) {
  F32x2 r;
  asm("add.rz.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

// One layer of the paged cache.  A page holds [2][Hkv][64 * D] elements: keys
// as [64 tokens][D], values transposed as [D][64 tokens].
struct CacheView {
  uint16_t* kv;
  const int32_t* page_table;
  int n_pages, n_seq, pt_stride, Hkv;

  // First element of a page's K (which = 0) or V^T (which = 1) of one KV head.
  __device__ __forceinline__ uint16_t* block(int page, int which, int head, int D) const {
    return kv + ((static_cast<int64_t>(page) * 2 + which) * Hkv + head) * (kPageTokens * D);
  }
};

inline CacheView cache_view(const gs_cache& c) {
  return {static_cast<uint16_t*>(c.kv), c.page_table, c.n_pages, c.n_seq, c.pt_stride,
          c.n_kv_heads};
}

// Runs a kernel's set-up once per device, under a lock (framework calls may
// come from several host threads); a failed run is tried again by the next call.
class DeviceOnce {
 public:
  template <class F>
  cudaError_t run(F setup) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    std::lock_guard<std::mutex> lock(mu_);
    if (dev < 64 && ((done_ >> dev) & 1)) return cudaSuccess;
    e = setup();
    if (e == cudaSuccess && dev < 64) done_ |= 1ull << dev;
    return e;
  }

 private:
  std::mutex mu_;
  uint64_t done_ = 0;
};

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
// All of them aligned for 32-bit elements (NULL is).
template <class... P>
inline bool aligned4(const P*... p) {
  return ((reinterpret_cast<uintptr_t>(p) | ...) & 3) == 0;
}

// GS_OK, or what is wrong with a cache descriptor.
inline int check_cache(const gs_cache* c) {
  if (!c || !c->kv || !c->page_table || !aligned16(c->kv) || !aligned4(c->page_table) || c->n_pages < 1 || c->n_kv_heads < 1 ||
      c->n_seq < 1 || c->pt_stride < 1 || c->pt_stride > (1 << 24))
    return GS_ERR_INVALID_ARG;
  if (c->dtype != GS_F16 && c->dtype != GS_BF16) return GS_ERR_INVALID_ARG;
  if (c->head_dim != 64 && c->head_dim != 128) return GS_ERR_UNSUPPORTED;
  return GS_OK;
}

}  // namespace gs
