// attend_common.cuh -- what the attentions over the paged cache share: the
// tensor instruction on 16 rows, exponentials, the held maximum, sums of parts.
#pragma once
#include <cmath>

#include "step_common.cuh"

namespace gs {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

template <bool BF16>
__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                         uint32_t a3, uint32_t b0, uint32_t b1) {
  if constexpr (BF16)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
        "{%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
        "{%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// 16 bytes that are read once.
__device__ __forceinline__ uint4 load_once(const uint16_t* p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "l"(p));
  return v;
}

// m = -inf means no weight at all: such a max is taken as 0, so that its
// exponentials are 2^-inf = 0 and not 2^(inf - inf).
__device__ __forceinline__ float finite_max(float m) { return m == -INFINITY ? 0.f : m; }

// How far below the largest exponent the max is held: in fp16 15, so that light keys keep
// their bits.
template <bool BF16>
constexpr float kHeld = BF16 ? 0.f : 15.f;

// The weights of two scores against the running maximum m (finite_max of it), 2^(scale (s - m)),
// and as much more as m is held low.  Maxima are kept as they come from the products, before
// scaling: the difference of two scores is exact where they are near each other, however
// large they are, while scale * s is rounded by more than a weight's range from 2^27 on.  P is
// at most 2^15 (or 1).
template <bool BF16>
__device__ __forceinline__ float2 weights_of(float s0, float s1, float m, float scale_log2) {
  const float2 e = split2(fma2(add2(join2(s0, s1), join2(-m, -m)), join2(scale_log2, scale_log2),
                               join2(kHeld<BF16>, kHeld<BF16>)));
  return make_float2(ex2(e.x), ex2(e.y));
}
// What sums against maximum `from` are multiplied by against one no less, of which z is the
// finite_max (found outside of loops: within the joining kernel's, one of 131,001 tokens took 0.9 us more).
__device__ __forceinline__ float moved_max(float from, float z, float scale_log2) {
  return ex2((from - z) * scale_log2);
}

// acc += f v, l += f l_v: products rounded before they are added, so that the
// two ways of joining items give the same bits.
__device__ __forceinline__ void add_scaled(float4& acc, float& l, const float4& v, float l_v, float f) {
  l = __fadd_rn(l, __fmul_rn(f, l_v));
  acc.x = __fadd_rn(acc.x, __fmul_rn(f, v.x));
  acc.y = __fadd_rn(acc.y, __fmul_rn(f, v.y));
  acc.z = __fadd_rn(acc.z, __fmul_rn(f, v.z));
  acc.w = __fadd_rn(acc.w, __fmul_rn(f, v.w));
}

}  // namespace gs
