// The norm between two blocks: h = x + delta rounded to the tensors' type (the residual stream taken on by a block's output),
// y = h / sqrt(mean(h^2) + eps) * weight, in the tensors' type or in e4m3 with a scale for each row.
//
// One pass: a row's elements stay in the registers of the threads that loaded them, between the loads and the stores there is
// the sum of their squares (fp32: two chains of at most 20 terms a thread, then a tree) and for 8 bits the maximum of |h weight|.
// 8 bits: q = e4m3(448 p / max|p|) with p = h weight, which bf16 factors give exactly; 1 / rms is in the row's scale alone.
//
// HBM bounds it: 65536 x 640 in bf16 with the addition 53 us (6.3 TB/s), 32767 x 1280 without 27.7 (6.0), to 8 bits 23.7 (5.3, with
// the instructions of the conversion close behind).  As many threads as hold a row in a few packets each, and the rows of a CTA one behind
// the other with the next one's loads under way: with one row per CTA of 128 threads 32767 x 1280 to 8 bits took 55 us, with rows of
// a warp 33, and 24 with the next row on its way and an element's value decided by two products (e4m3.cuh).
#include "e4m3.cuh"
#include "tc.cuh"

namespace toma {

namespace {

template <int kLanes>
__device__ __forceinline__ float sum_row(float v, float* red, int t) {
#pragma unroll
  for (int o = kLanes < 32 ? kLanes / 2 : 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if constexpr (kLanes > 32) {
    if ((t & 31) == 0) red[t >> 5] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int w = 0; w < kLanes / 32; ++w) v += red[w];
  }
  return v;
}
__device__ __forceinline__ float max_nan(float a, float b) {  // a number that is none stays one
  float d;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
  return d;
}
template <int kLanes>
__device__ __forceinline__ float max_row(float v, float* red, int t) {
#pragma unroll
  for (int o = kLanes < 32 ? kLanes / 2 : 16; o > 0; o >>= 1) v = max_nan(v, __shfl_xor_sync(0xffffffffu, v, o));
  if constexpr (kLanes > 32) {
    if ((t & 31) == 0) red[t >> 5] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int w = 0; w < kLanes / 32; ++w) v = max_nan(v, red[w]);
  }
  return v;
}

// Blocks of an SM at once: as many as the registers of a thread allow.  It holds kVec packets of x, delta and weight as they lie in memory
// and of h as floats, and some 30 besides; 64 registers make four blocks of 256 threads, 84 three, 128 two.
template <typename T, bool kAdd, int kVec>
constexpr int kNormRegs = kVec * (8 + (int)sizeof(T) * (kAdd ? 6 : 4)) + 30;
template <typename T, bool kAdd, int kLanes, int kVec>
constexpr int kNormCtas = kLanes > 256 ? (kVec * sizeof(T) <= 4 ? 2 : 1)  // (of 512 threads)
                          : kNormRegs<T, kAdd, kVec> <= 64  ? 4
                          : kNormRegs<T, kAdd, kVec> <= 84  ? 3
                          : kNormRegs<T, kAdd, kVec> <= 128 ? 2
                                                            : 1;

// Packets of eight elements as they lie in memory.
template <typename T> struct Raw;
template <> struct Raw<__nv_bfloat16> { uint4 q; };
template <> struct Raw<float> { float4 q[2]; };
__device__ __forceinline__ void load_raw(const __nv_bfloat16* p, Raw<__nv_bfloat16>& r) { r.q = *reinterpret_cast<const uint4*>(p); }
__device__ __forceinline__ void load_raw(const float* p, Raw<float>& r) {
  r.q[0] = reinterpret_cast<const float4*>(p)[0];
  r.q[1] = reinterpret_cast<const float4*>(p)[1];
}
__device__ __forceinline__ void widen(const Raw<__nv_bfloat16>& r, float (&v)[8]) {
  const uint32_t w[4] = {r.q.x, r.q.y, r.q.z, r.q.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    v[2 * e] = __uint_as_float(w[e] << 16);
    v[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ void widen(const Raw<float>& r, float (&v)[8]) {
  v[0] = r.q[0].x, v[1] = r.q[0].y, v[2] = r.q[0].z, v[3] = r.q[0].w, v[4] = r.q[1].x, v[5] = r.q[1].y, v[6] = r.q[1].z, v[7] = r.q[1].w;
}
__device__ __forceinline__ float max3_abs(float top, float a, float b) {  // a number that is none stays one
  float d;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(top), "f"(fabsf(a)), "f"(fabsf(b)));
  return d;
}

// kLanes threads per row, kVec packets of 8 elements in each.  A row's threads go on to further rows, the next one's elements on
// their way while this one's are worked on; the weight stays in registers.
template <typename T, bool kQ8, bool kAdd, int kLanes, int kVec>
__global__ void __launch_bounds__(kLanes < 256 ? 256 : kLanes, kNormCtas<T, kAdd, kLanes, kVec>) rms_norm_kernel(const NormOp o) {
  constexpr int kRows = kLanes < 256 ? 256 / kLanes : 1;
  __shared__ float red_s[2][kRows][(kLanes + 31) / 32], red_m[2][kRows][(kLanes + 31) / 32];
  const int group = threadIdx.x / kLanes, t = threadIdx.x % kLanes;
  tc::dependency_wait();  // launched with programmatic stream serialisation
  if (threadIdx.x == 0) tc::release_dependents();
  const bool weighted = o.weight != nullptr;
  const float inv_dim = 1.f / (float)o.dim;
  bool in[kVec];
  Raw<T> w[kVec], x[kVec], d[kAdd ? kVec : 1];
#pragma unroll
  for (int v = 0; v < kVec; ++v) {
    in[v] = (v * kLanes + t) * 8 < o.dim;
    w[v] = x[v] = Raw<T>{};
    if constexpr (kAdd) d[v] = Raw<T>{};
    if (in[v] && weighted) load_raw((const T*)o.weight + (v * kLanes + t) * 8, w[v]);
  }
  const auto fetch = [&](int row) {
#pragma unroll
    for (int v = 0; v < kVec; ++v)
      if (in[v]) {
        load_raw((const T*)o.x + (size_t)row * o.ldx + (v * kLanes + t) * 8, x[v]);
        if constexpr (kAdd) load_raw((const T*)o.delta + (size_t)row * o.ldd + (v * kLanes + t) * 8, d[v]);
      }
  };
  // (all threads of a block take the same number of turns: there are barriers in them where a row is several warps')
  int row = blockIdx.x * kRows + group;
  if (row < o.rows) fetch(row);
  for (int base = blockIdx.x * kRows, turn = 0; base < o.rows; base += gridDim.x * kRows, ++turn) {
    const bool live = row < o.rows;
    float h[kVec][8];
#pragma unroll
    for (int v = 0; v < kVec; ++v) {
      widen(x[v], h[v]);
      if constexpr (kAdd) {
        float e[8];
        widen(d[v], e);
#pragma unroll
        for (int u = 0; u < 8; ++u) h[v][u] += e[u];
        if constexpr (sizeof(T) == 2) {  // rounded to the stream's type
          __align__(16) __nv_bfloat162 q[4];
#pragma unroll
          for (int u = 0; u < 4; ++u) q[u] = __floats2bfloat162_rn(h[v][2 * u], h[v][2 * u + 1]);
          const Raw<T> r{*reinterpret_cast<const uint4*>(q)};
          if (o.sum && live && in[v]) *reinterpret_cast<uint4*>((T*)o.sum + (size_t)row * o.lds + (v * kLanes + t) * 8) = r.q;
          widen(r, h[v]);
        } else {
          if (o.sum && live && in[v]) store8((T*)o.sum + (size_t)row * o.lds + (v * kLanes + t) * 8, h[v]);
        }
      }
    }
    const int next = row + (int)gridDim.x * kRows;
    if (next < o.rows) fetch(next);
    uint64_t ss2 = 0;
#pragma unroll
    for (int v = 0; v < kVec; ++v)
#pragma unroll
      for (int u = 0; u < 8; u += 2) {
        const uint64_t p = tc::pack2(h[v][u], h[v][u + 1]);
        ss2 = tc::fma2(p, p, ss2);
      }
    float s0, s1;
    tc::unpack2(ss2, s0, s1);
    const float ss = sum_row<kLanes>(s0 + s1, red_s[turn & 1][group], t);
    // (2 units of the last place of rsqrtf: enough for y in 16 bits.  A row's scale in fp32 has them too: 7.3e-8 off, root mean square, where
    // one rounding of 64 bits is 5.1e-8; below the 2^-4 of the e4m3 that it multiplies in any case.)
    const float r = sizeof(T) == 4 ? 1.f / sqrtf(ss / (float)o.dim + o.eps) : rsqrtf(fmaf(ss, inv_dim, o.eps));
    if constexpr (!kQ8) {
#pragma unroll
      for (int v = 0; v < kVec; ++v) {
        float f[8];
        widen(w[v], f);
#pragma unroll
        for (int u = 0; u < 8; ++u) f[u] = weighted ? h[v][u] * r * f[u] : h[v][u] * r;
        if (live && in[v]) store8((T*)o.y + (size_t)row * o.ldy + (v * kLanes + t) * 8, f);
      }
    } else {
      float top = 0.f;
#pragma unroll
      for (int v = 0; v < kVec; ++v) {
        if (weighted) {
          float f[8];
          widen(w[v], f);
#pragma unroll
          for (int u = 0; u < 8; u += 2) tc::unpack2(tc::mul2(tc::pack2(h[v][u], h[v][u + 1]), tc::pack2(f[u], f[u + 1])), h[v][u], h[v][u + 1]);
        }
#pragma unroll
        for (int u = 0; u < 8; u += 2) top = max3_abs(top, h[v][u], h[v][u + 1]);
      }
      top = max_row<kLanes>(top, red_m[turn & 1][group], t);
      const E4m3Row q8(top);
#pragma unroll
      for (int v = 0; v < kVec; ++v) {
        const uint2 q = q8.packet(h[v]);
        if (live && in[v]) *reinterpret_cast<uint2*>((uint8_t*)o.y + (size_t)row * o.ldy + (v * kLanes + t) * 8) = q;
      }
      if (live && t == 0) o.scale[row] = r * q8.scale();
    }
    row = next;
  }
}

template <typename T, bool kQ8, bool kAdd, int kLanes, int kVec>
cudaError_t run_norm(const NormOp& o, cudaStream_t s) {
  constexpr int kRows = kLanes < 256 ? 256 / kLanes : 1;
  const int blocks = (o.rows + kRows - 1) / kRows, most = sm_count() * kNormCtas<T, kAdd, kLanes, kVec>;
  count_launch();
  return launch_dependent(rms_norm_kernel<T, kQ8, kAdd, kLanes, kVec>, dim3(blocks < most ? blocks : most), dim3(kRows * kLanes), 0, s, o);
}

template <typename T, bool kQ8, bool kAdd>
cudaError_t norm_form(const NormOp& o, cudaStream_t s) {
  const int packets = (o.dim + 7) / 8;
  if (packets <= 8) return run_norm<T, kQ8, kAdd, 8, 1>(o, s);
  if (packets <= 16) return run_norm<T, kQ8, kAdd, 16, 1>(o, s);
  if (packets <= 32) return run_norm<T, kQ8, kAdd, 32, 1>(o, s);
  if (packets <= 64) return run_norm<T, kQ8, kAdd, 32, 2>(o, s);
  if (packets <= 96) return run_norm<T, kQ8, kAdd, 32, 3>(o, s);
  if (packets <= 128) return run_norm<T, kQ8, kAdd, 32, 4>(o, s);
  if (packets <= 160) return run_norm<T, kQ8, kAdd, 32, 5>(o, s);
  if (packets <= 256) return run_norm<T, kQ8, kAdd, 128, 2>(o, s);
  if (packets <= 384) return run_norm<T, kQ8, kAdd, 128, 3>(o, s);
  if (packets <= 512) return run_norm<T, kQ8, kAdd, 128, 4>(o, s);
  if (packets <= 1024) return run_norm<T, kQ8, kAdd, 512, 2>(o, s);
  return run_norm<T, kQ8, kAdd, 512, 4>(o, s);
}

// A CTA's 32 columns of w [K][N]: their maxima, then the columns as rows of q.  (Once per model: two reads, the second from L2.)
constexpr int kQwRows = 128;
__global__ void __launch_bounds__(256) quantise_weight_kernel(int K, int N, const __nv_bfloat16* __restrict__ w, uint8_t* __restrict__ q, int ldq,
                                                              float* __restrict__ scale) {
  __shared__ uint32_t red[64][33];
  __shared__ float tile[kQwRows][33];
  __shared__ float top_of[32];
  const int n0 = blockIdx.x * 32, t = threadIdx.x, c = t % 4 * 8, line = t / 4;  // 8 columns of every 64th row
  tc::dependency_wait();
  if (t == 0) tc::release_dependents();
  const bool there = n0 + c < N;
  uint32_t top[8] = {};
  for (int k = line; k < K; k += 64) {
    float v[8] = {};
    if (there) load8(w + (size_t)k * N + n0 + c, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) top[e] = max(top[e], abs_bits(v[e]));
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) red[line][c + e] = top[e];
  __syncthreads();
  if (t < 32) {
    uint32_t m = 0;
    for (int l = 0; l < 64; ++l) m = max(m, red[l][t]);
    top_of[t] = __uint_as_float(m);
    if (n0 + t < N) scale[n0 + t] = E4m3Row(top_of[t]).scale();
  }
  for (int k0 = 0; k0 < K; k0 += kQwRows) {
    __syncthreads();
    for (int k = line; k < kQwRows; k += 64) {
      float v[8] = {};
      if (there && k0 + k < K) load8(w + (size_t)(k0 + k) * N + n0 + c, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) tile[k][c + e] = v[e];
    }
    __syncthreads();
    for (int e = t; e < 32 * kQwRows / 8; e += 256) {  // packet of 8 k of a column
      const int col = e / (kQwRows / 8), k = e % (kQwRows / 8) * 8;
      if (n0 + col >= N || k0 + k >= K) continue;
      float p[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) p[u] = tile[k + u][col];
      *reinterpret_cast<uint2*>(q + (size_t)(n0 + col) * ldq + k0 + k) = E4m3Row(top_of[col]).packet(p);
    }
  }
}

}  // namespace

cudaError_t launch_rms_norm(const NormOp& o, cudaStream_t s) {
  const bool add = o.delta != nullptr;
  const cudaError_t e = o.scale ? (add ? norm_form<__nv_bfloat16, true, true>(o, s) : norm_form<__nv_bfloat16, true, false>(o, s))
                        : o.f32 ? (add ? norm_form<float, false, true>(o, s) : norm_form<float, false, false>(o, s))
                                : (add ? norm_form<__nv_bfloat16, false, true>(o, s) : norm_form<__nv_bfloat16, false, false>(o, s));
  return e != cudaSuccess ? e : cudaGetLastError();
}

cudaError_t launch_quantise_weight(int K, int N, const void* w, void* q, int ldq, float* scale, cudaStream_t s) {
  count_launch();
  const cudaError_t e = launch_dependent(quantise_weight_kernel, dim3((N + 31) / 32), dim3(256), 0, s, K, N, (const __nv_bfloat16*)w, (uint8_t*)q, ldq, scale);
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace toma
