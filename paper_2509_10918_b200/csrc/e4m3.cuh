// Rows in 8 bits (1 sign, 4 exponent, 3 mantissa bits) with a scale for each: q = e4m3(448 p / max|p|).
#pragma once

#include <cuda_fp8.h>

#include "common.cuh"
#include "tc.cuh"

namespace toma {

constexpr float kE4m3Max = 448.f;
// A row whose largest magnitude is below this comes out as zeros with scale 0 (448 / max|p| would leave fp32).
constexpr float kE4m3Tiny = 7.88860905e-31f;  // 2^-100

// Where 448 p / top lies next to a border between two e4m3 values the side is decided exactly.  A border m has at most 5 significant
// bits and v is within 2^-20 of 448 p / top, so only a v within 8 units of the last place of a number of 5 bits is in question; with p of at
// most 16 bits (a product of two bf16) times 7 and m times top are exact in fp32, and 448 p / top >< m is 7 p / 64 >< m top / 4096.
__device__ __forceinline__ float e4m3_decided(float v, float p, float top) {
  const uint32_t b = __float_as_uint(fabsf(v)) + 8u;
  if ((b & 0x7FFFFu) > 16u || b >= 0x7F800000u) return v;  // (the latter: no number)
  const float m = __uint_as_float(b & ~0x7FFFFu), d = fabsf(p) * 0.109375f - m * (top * 2.44140625e-4f);
  const uint32_t side = __float_as_uint(m) + (d > 0.f ? 1u : d < 0.f && m > 0.f ? 0xFFFFFFFFu : 0u);
  return copysignf(__uint_as_float(side), v);
}
__device__ __forceinline__ uint32_t e4m3_pair(float lo, float hi) { return __nv_cvt_float2_to_fp8x2(make_float2(lo, hi), __NV_SATFINITE, __NV_E4M3); }

// A row whose largest |p| is `top`.
struct E4m3Row {
  float top, t, below, above;  // t ~ 448 / top, and t 2^-21 less and more
  bool none, zero;
  __device__ __forceinline__ explicit E4m3Row(float top_) : top(top_) {
    // a row with an infinity or none-number in it has none-numbers in its place and as its scale
    none = !(top < INFINITY), zero = top < kE4m3Tiny;
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(top * 0.001953125f));  // (1 / top of a large top would leave the normal numbers)
    t = none ? __uint_as_float(0x7FC00000u) : zero ? 0.f : r * 0.875f;
    below = t * (1.f - 4.76837158e-7f), above = t * (1.f + 4.76837158e-7f);
  }
  // The scale is this over the root mean square.
  __device__ __forceinline__ float scale() const { return none ? t : zero ? 0.f : top * (1.f / kE4m3Max); }
  // Eight of its elements.  t is within 2^-22 of 448 / top (reciprocal 1 unit of the last place, product half a unit), so 448 p / top lies
  // between p below and p above, and where both come out as the same value so does it; elsewhere (one element in some 10^5, ties
  // among them) it is decided exactly.
  __device__ __forceinline__ uint2 packet(const float (&p)[8]) const {
    uint32_t lo[4], hi[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint64_t x = tc::pack2(p[2 * e], p[2 * e + 1]);
      float a, b;
      tc::unpack2(tc::mul2(x, tc::pack2(below, below)), a, b);
      lo[e] = e4m3_pair(a, b);
      tc::unpack2(tc::mul2(x, tc::pack2(above, above)), a, b);
      hi[e] = e4m3_pair(a, b);
    }
    uint2 q = make_uint2(lo[0] | lo[1] << 16, lo[2] | lo[3] << 16);
    if (q.x != (hi[0] | hi[1] << 16) || q.y != (hi[2] | hi[3] << 16)) {
#pragma unroll
      for (int e = 0; e < 4; ++e) lo[e] = e4m3_pair(e4m3_decided(p[2 * e] * t, p[2 * e], top), e4m3_decided(p[2 * e + 1] * t, p[2 * e + 1], top));
      q = make_uint2(lo[0] | lo[1] << 16, lo[2] | lo[3] << 16);
    }
    return q;
  }
};
__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }  // ordered, NaN above infinity

// Eight consecutive elements (16 bytes of bf16, 32 of fp32 in store8), aligned to 16 bytes.
__device__ __forceinline__ void load8(const __nv_bfloat16* p, float (&v)[8]) {
  const uint4 q = *reinterpret_cast<const uint4*>(p);
  const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    v[2 * e] = __uint_as_float(w[e] << 16);
    v[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&v)[8]) {
  __align__(16) __nv_bfloat162 h[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) h[e] = __floats2bfloat162_rn(v[2 * e], v[2 * e + 1]);
  *reinterpret_cast<uint4*>(p) = *reinterpret_cast<const uint4*>(h);
}
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}

}  // namespace toma
