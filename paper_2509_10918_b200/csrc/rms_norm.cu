// The norm between two blocks: h = x + delta rounded to the tensors' type (the residual stream taken on by a block's output),
// y = h / sqrt(mean(h^2) + eps) * weight, in the tensors' type or in e4m3 with a scale for each row.
//
// One pass: a row's elements stay in the registers of the threads that loaded them, between the loads and the stores there is
// the sum of their squares (fp32: chains of at most 40 terms, then a tree) and for 8 bits the maximum of |h weight|.
// 8 bits: q = e4m3(448 p / max|p|) with p = h weight, which bf16 factors give exactly; 1 / rms is in the row's scale alone.
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
template <int kLanes>
__device__ __forceinline__ uint32_t max_row(uint32_t v, uint32_t* red, int t) {
#pragma unroll
  for (int o = kLanes < 32 ? kLanes / 2 : 16; o > 0; o >>= 1) v = max(v, __shfl_xor_sync(0xffffffffu, v, o));
  if constexpr (kLanes > 32) {
    if ((t & 31) == 0) red[t >> 5] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int w = 0; w < kLanes / 32; ++w) v = max(v, red[w]);
  }
  return v;
}

// kLanes threads per row, kVec packets of 8 elements in each.
template <typename T, bool kQ8, int kLanes, int kVec>
__global__ void __launch_bounds__(kLanes < 256 ? 256 : kLanes) rms_norm_kernel(const NormOp o) {
  constexpr int kRows = kLanes < 256 ? 256 / kLanes : 1;
  __shared__ float red_s[kRows][kLanes / 32];
  __shared__ uint32_t red_m[kRows][kLanes / 32];
  const int group = threadIdx.x / kLanes, t = threadIdx.x % kLanes;
  const int row = blockIdx.x * kRows + group;
  const bool live = row < o.rows;
  tc::dependency_wait();  // launched with programmatic stream serialisation
  if (threadIdx.x == 0) tc::release_dependents();
  const T* x = (const T*)o.x + (size_t)row * o.ldx;
  const T* delta = (const T*)o.delta + (size_t)row * o.ldd;
  const T* weight = (const T*)o.weight;
  float h[kVec][8];
#pragma unroll
  for (int v = 0; v < kVec; ++v) {
    const int e = (v * kLanes + t) * 8;
    if (live && e < o.dim) load8(x + e, h[v]);
    else
#pragma unroll
      for (int u = 0; u < 8; ++u) h[v][u] = 0.f;
  }
  if (o.delta) {
#pragma unroll
    for (int v = 0; v < kVec; ++v) {
      const int e = (v * kLanes + t) * 8;
      if (live && e < o.dim) {
        float d[8];
        load8(delta + e, d);
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          T r;
          from_f32(r, h[v][u] + d[u]);
          h[v][u] = to_f32(r);
        }
        if (o.sum) store8((T*)o.sum + (size_t)row * o.lds + e, h[v]);
      }
    }
  }
  float ss = 0.f;
#pragma unroll
  for (int v = 0; v < kVec; ++v)
#pragma unroll
    for (int u = 0; u < 8; ++u) ss = fmaf(h[v][u], h[v][u], ss);
  ss = sum_row<kLanes>(ss, red_s[group], t);
  const float r = 1.f / sqrtf(ss / (float)o.dim + o.eps);
  if constexpr (!kQ8) {
#pragma unroll
    for (int v = 0; v < kVec; ++v) {
      const int e = (v * kLanes + t) * 8;
      if (live && e < o.dim) {
        float w[8];
        if (weight) load8(weight + e, w);
#pragma unroll
        for (int u = 0; u < 8; ++u) w[u] = weight ? h[v][u] * r * w[u] : h[v][u] * r;
        store8((T*)o.y + (size_t)row * o.ldy + e, w);
      }
    }
  } else {
    uint32_t top_bits = 0;
#pragma unroll
    for (int v = 0; v < kVec; ++v) {
      const int e = (v * kLanes + t) * 8;
      if (weight && live && e < o.dim) {
        float w[8];
        load8(weight + e, w);
#pragma unroll
        for (int u = 0; u < 8; ++u) h[v][u] *= w[u];
      }
#pragma unroll
      for (int u = 0; u < 8; ++u) top_bits = max(top_bits, abs_bits(h[v][u]));
    }
    top_bits = max_row<kLanes>(top_bits, red_m[group], t);
    const float top = __uint_as_float(top_bits);
    // a row with an infinity or none-number in it has none-numbers in its place and as its scale
    const bool none = top_bits >= 0x7F800000u, zero = top < kE4m3Tiny;
    const float f = none ? __uint_as_float(0x7FC00000u) : zero ? 0.f : kE4m3Max / top;
#pragma unroll
    for (int v = 0; v < kVec; ++v) {
      const int e = (v * kLanes + t) * 8;
      if (live && e < o.dim) *reinterpret_cast<uint2*>((uint8_t*)o.y + (size_t)row * o.ldy + e) = e4m3_packet(h[v], f, top);
    }
    if (live && t == 0) o.scale[row] = none ? __uint_as_float(0x7FC00000u) : zero ? 0.f : r * top * (1.f / kE4m3Max);
  }
}

template <typename T, bool kQ8, int kLanes, int kVec>
cudaError_t run_norm(const NormOp& o, cudaStream_t s) {
  constexpr int kRows = kLanes < 256 ? 256 / kLanes : 1;
  count_launch();
  return launch_dependent(rms_norm_kernel<T, kQ8, kLanes, kVec>, dim3((o.rows + kRows - 1) / kRows), dim3(kRows * kLanes), 0, s, o);
}

template <typename T, bool kQ8>
cudaError_t norm_form(const NormOp& o, cudaStream_t s) {
  const int packets = (o.dim + 7) / 8;
  if (packets <= 32) return run_norm<T, kQ8, 32, 1>(o, s);
  if (packets <= 64) return run_norm<T, kQ8, 32, 2>(o, s);
  if (packets <= 96) return run_norm<T, kQ8, 32, 3>(o, s);
  if (packets <= 128) return run_norm<T, kQ8, 32, 4>(o, s);
  if (packets <= 256) return run_norm<T, kQ8, 128, 2>(o, s);
  if (packets <= 512) return run_norm<T, kQ8, 128, 4>(o, s);
  if (packets <= 1024) return run_norm<T, kQ8, 512, 2>(o, s);
  return run_norm<T, kQ8, 512, 4>(o, s);
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
    const float f = __uint_as_float(m);
    top_of[t] = f;
    if (n0 + t < N) scale[n0 + t] = m >= 0x7F800000u ? __uint_as_float(0x7FC00000u) : f < kE4m3Tiny ? 0.f : f * (1.f / kE4m3Max);
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
      const float m = top_of[col], f = abs_bits(m) >= 0x7F800000u ? __uint_as_float(0x7FC00000u) : m < kE4m3Tiny ? 0.f : kE4m3Max / m;
      *reinterpret_cast<uint2*>(q + (size_t)(n0 + col) * ldq + k0 + k) = e4m3_packet(p, f, m);
    }
  }
}

}  // namespace

cudaError_t launch_rms_norm(const NormOp& o, cudaStream_t s) {
  const cudaError_t e = o.scale ? norm_form<__nv_bfloat16, true>(o, s) : o.f32 ? norm_form<float, false>(o, s) : norm_form<__nv_bfloat16, false>(o, s);
  return e != cudaSuccess ? e : cudaGetLastError();
}

cudaError_t launch_quantise_weight(int K, int N, const void* w, void* q, int ldq, float* scale, cudaStream_t s) {
  count_launch();
  const cudaError_t e = launch_dependent(quantise_weight_kernel, dim3((N + 31) / 32), dim3(256), 0, s, K, N, (const __nv_bfloat16*)w, (uint8_t*)q, ldq, scale);
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace toma
