// Rows in 8 bits (1 sign, 4 exponent, 3 mantissa bits) with a scale for each: q = e4m3(448 p / max|p|).
#pragma once

#include <cuda_fp8.h>

#include "common.cuh"

namespace toma {

constexpr float kE4m3Max = 448.f;
// A row whose largest magnitude is below this comes out as zeros with scale 0 (448 / max|p| would leave fp32).
constexpr float kE4m3Tiny = 7.88860905e-31f;  // 2^-100

// v = p t with t = fp32(448 / top) is within 2 units in the last place of 448 p / top.  The borders between neighbouring e4m3
// values have at most 5 significant bits, so only where v is within 3 units of a number of 5 bits can v lie on the wrong
// side of one, or look like a tie that is none.
__device__ __forceinline__ uint32_t e4m3_distance(float v) { return (__float_as_uint(v) + 3u) & 0x7FFFFu; }  // <= 6: near one
// There the side is decided exactly: p of at most 16 bits (a product of two bf16) times 7 and m of 5 bits times top are exact in
// fp32, and 448 p / top >< m is 7 p / 64 >< m top / 4096.
__device__ __forceinline__ float e4m3_decided(float v, float p, float top) {
  const uint32_t b = __float_as_uint(fabsf(v)) + 3u;
  if ((b & 0x7FFFFu) > 6u || b >= 0x7F800000u) return v;  // (the latter: no number)
  const float m = __uint_as_float(b & ~0x7FFFFu), d = fabsf(p) * 0.109375f - m * (top * 2.44140625e-4f);
  const uint32_t side = __float_as_uint(m) + (d > 0.f ? 1u : d < 0.f && m > 0.f ? 0xFFFFFFFFu : 0u);
  return copysignf(__uint_as_float(side), v);
}
// Eight of them, v[i] = p[i] t, in two words.
__device__ __forceinline__ uint2 e4m3_packet(const float (&p)[8], float t, float top) {
  float v[8];
  uint32_t near = 0xFFFFFFFFu;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    v[e] = p[e] * t;
    near = min(near, e4m3_distance(v[e]));
  }
  if (near <= 6u) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e4m3_decided(v[e], p[e], top);
  }
  uint32_t h[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) h[e] = __nv_cvt_float2_to_fp8x2(make_float2(v[2 * e], v[2 * e + 1]), __NV_SATFINITE, __NV_E4M3);
  return make_uint2(h[0] | h[1] << 16, h[2] | h[3] << 16);
}
__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }  // ordered, NaN above infinity

// Eight consecutive elements (16 bytes of bf16, 32 of fp32), aligned to 16 bytes.
__device__ __forceinline__ void load8(const __nv_bfloat16* p, float (&v)[8]) {
  const uint4 q = *reinterpret_cast<const uint4*>(p);
  const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    v[2 * e] = __uint_as_float(w[e] << 16);
    v[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
  const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
  v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
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
