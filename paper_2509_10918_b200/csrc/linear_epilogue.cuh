// The epilogue of the tensor-core projections: scales, bias, activation, residual.
#pragma once

#include "common.cuh"
#include "tc.cuh"

namespace toma {

// What a kernel multiplies and what it does with the sums.  kPlain: bf16, up to three matrices, an activation.  kPlus: bf16, one
// matrix, bias, activation and residual.  kPlus8: the same of e4m3 operands with scales.  A row of a stage is 128 bytes of either
// type, so e4m3 takes the same slabs, boxes and cycles with twice the contraction elements; W is K-major there, [n][k] as stored.
constexpr int kPlain = 0, kPlus = 1, kPlus8 = 2;

// The epilogue of kPlus and kPlus8.  bias, a_scale, w_scale: [n], [m], [n], residual: [m][n], each or none.
struct LinearPlus {
  const __nv_bfloat16 *bias, *residual;
  const float *a_scale, *w_scale;
  __nv_bfloat16* c;
  int ldc, ldr;
};

namespace epi {
using namespace tc;

// GELU(v) = v Phi(v) = max(v, 0) - |v| Phi(-|v|) of two values, for results that are rounded to bf16.
// Phi(-a) = erfcx(a / sqrt 2) / 2 * 2^(-a^2 log2(e) / 2), and erfcx(x) / 2 = t (c0 + c1 t + ... + c7 t^7) with
// t = 1 / (1 + 0.33 x): the coefficients are the minimax fit of the relative error on x in [0, 10] (9.4e-8; with fp32
// arithmetic the result is within 5e-7 of the exact one for v > -1 and 8e-6 down to -13, where v (1 + erff) loses all
// digits).  Eleven issue slots and two MUFU operations per value against about 45 slots with erff, which made the first
// layer of an MLP of 4096 x 2560 x 640 a matter of its epilogue (34 us of which 13 us the activation).
__device__ __forceinline__ float rcp_mufu(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float min_nan(float a, float b) {  // a number that is none stays one
  float d;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
  return d;
}
__device__ __forceinline__ uint64_t both(float v) { return pack2(v, v); }
__device__ __forceinline__ void gelu2(uint32_t& v0, uint32_t& v1) {
  const float x0 = __uint_as_float(v0), x1 = __uint_as_float(v1);
  const uint64_t a = pack2(min_nan(fabsf(x0), 30.f), min_nan(fabsf(x1), 30.f));
  float d0, d1, e0, e1;
  unpack2(fma2(a, both(0.233345238f), both(1.f)), d0, d1);
  const uint64_t t = pack2(rcp_mufu(d0), rcp_mufu(d1));
  uint64_t q = fma2(both(-0.0676728131f), t, both(0.230118425f));
  q = fma2(q, t, both(-0.175574611f));
  q = fma2(q, t, both(0.204249755f));
  q = fma2(q, t, both(0.0236104601f));
  q = fma2(q, t, both(0.100611901f));
  q = fma2(q, t, both(0.0914779779f));
  q = fma2(q, t, both(0.0931789011f));
  unpack2(mul2(mul2(a, both(-0.72134752f)), a), e0, e1);
  q = mul2(mul2(mul2(q, t), a), pack2(ex2_mufu(e0), ex2_mufu(e1)));
  float g0, g1;
  unpack2(sub2(pack2(fmaxf(x0, 0.f), fmaxf(x1, 0.f)), q), g0, g1);
  v0 = __float_as_uint(g0);
  v1 = __float_as_uint(g1);
}
// v sigmoid(z) = v / (1 + 2^(-z log2(e))) of two values, with z = v (SiLU) or z = 2 sqrt(2 / pi) (v + 0.044715 v^3) (GELU by tanh:
// (1 + tanh u) / 2 = sigmoid(2 u)).  The exponent's argument is rounded to fp32, so that the result's relative error grows with it: 2^-21
// for |z| < 5, 2^-18 for SiLU and 2^-16 for GELU at z = -85, by evaluation of the argument alone, to which the approximate
// exponential and reciprocal add 2^-22 each.  The rounding to bf16 is up to 2^-8, and everything below z = -5 is
// less than 2^-7 of its argument.  Below z = -87 the reciprocal leaves the normal numbers and the result is 0, 10^-36 off.  (A
// none-number in v stays one through the product with v.)
template <int kAct>
__device__ __forceinline__ void by_sigmoid2(uint32_t& v0, uint32_t& v1) {
  const uint64_t v = pack2(__uint_as_float(v0), __uint_as_float(v1));
  uint64_t z;
  if constexpr (kAct == kActSilu) z = mul2(v, both(-1.44269504f));
  else z = mul2(v, fma2(mul2(v, v), both(-0.102943240f), both(-2.30220819f)));
  float z0, z1, d0, d1;
  unpack2(z, z0, z1);
  unpack2(add2(pack2(ex2_mufu(z0), ex2_mufu(z1)), both(1.f)), d0, d1);
  float y0, y1;
  unpack2(mul2(v, pack2(rcp_mufu(d0), rcp_mufu(d1))), y0, y1);
  v0 = __float_as_uint(y0);
  v1 = __float_as_uint(y1);
}
// To full precision: fp32 mode is what bf16 runs are checked against.
__device__ __forceinline__ float activate_f32(float x, int act) {
  if (act == kActNone) return x;
  if (act == kActGelu) return 0.5f * x * erfcf(-0.70710678118654752f * x);
  return x / (1.f + expf(-(act == kActSilu ? x : x * fmaf(0.0713548162f, x * x, 1.59576912f))));
}
// r[e] += the eight bf16 of a packet.
__device__ __forceinline__ void add_packet(uint32_t* r, const uint4& b) {
  const uint32_t bb[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    float lo, hi;
    unpack2(add2(pack2(__uint_as_float(r[2 * u]), __uint_as_float(r[2 * u + 1])), pack2(__uint_as_float(bb[u] << 16), __uint_as_float(bb[u] & 0xFFFF0000u))),
            lo, hi);
    r[2 * u] = __float_as_uint(lo);
    r[2 * u + 1] = __float_as_uint(hi);
  }
}

// The epilogue of eight columns of one row, into global memory.
template <int kKind>
struct Finish8 {
  float4 s0, s1;
  uint4 bias, res;
  float row_scale;
  __device__ __forceinline__ void fetch(const LinearPlus& p, int row, int n) {
    if constexpr (kKind == kPlus8) {
      s0 = *reinterpret_cast<const float4*>(p.w_scale + n), s1 = *reinterpret_cast<const float4*>(p.w_scale + n + 4);
      row_scale = p.a_scale[row];
    }
    if (p.bias) bias = *reinterpret_cast<const uint4*>(p.bias + n);
    if (p.residual) res = *reinterpret_cast<const uint4*>(p.residual + (size_t)row * p.ldr + n);
  }
  __device__ __forceinline__ void out(float (&v)[8], const LinearPlus& p, int act, __nv_bfloat16* c) const {
    uint32_t r[8];
    if constexpr (kKind == kPlus8) {
      const float s[8] = {s0.x, s0.y, s0.z, s0.w, s1.x, s1.y, s1.z, s1.w};
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = v[e] * row_scale * s[e];
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = __float_as_uint(v[e]);
    if (p.bias) add_packet(r, bias);
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      if (act == kActGelu) gelu2(r[e], r[e + 1]);
      else if (act == kActSilu) by_sigmoid2<kActSilu>(r[e], r[e + 1]);
      else if (act == kActGeluTanh) by_sigmoid2<kActGeluTanh>(r[e], r[e + 1]);
    }
    if (p.residual) add_packet(r, res);
    __align__(16) __nv_bfloat162 q[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) q[u] = __floats2bfloat162_rn(__uint_as_float(r[2 * u]), __uint_as_float(r[2 * u + 1]));
    *reinterpret_cast<uint4*>(c) = *reinterpret_cast<const uint4*>(q);
  }
};
template <int kKind>
__device__ __forceinline__ void finish8(float (&v)[8], float row_scale, const LinearPlus& p, int act, const uint4& res, int n, __nv_bfloat16* c) {
  Finish8<kKind> f;
  if constexpr (kKind == kPlus8) {
    f.s0 = *reinterpret_cast<const float4*>(p.w_scale + n), f.s1 = *reinterpret_cast<const float4*>(p.w_scale + n + 4);
    f.row_scale = row_scale;
  }
  if (p.bias) f.bias = *reinterpret_cast<const uint4*>(p.bias + n);
  f.res = res;
  f.out(v, p, act, c);
}

}  // namespace epi
}  // namespace toma
