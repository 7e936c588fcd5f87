// c = act(a w + bias) + residual in fp32 on the tensor cores, for more than 16 rows.
//
// A float is the sum of three bf16 numbers, exactly: x = x0 + x1 + x2 with x0 = bf16(x), x1 = bf16(x - x0), x2 = x - x0 - x1 (8 bits
// each of the 24).  Of the nine products of two such sums the three smallest are below 2^-25 of the whole, the other six are
// multiplied by tcgen05, whose products are exact and whose sums are in fp32.  A long chain of such sums is not as exact as one of
// fused multiply-adds (they are cut off, not rounded), so a chain ends with its stage of 64 contraction elements, the small
// products first, and the stages' sums are added up by the threads, rounded: 1003 x 2560 x 640 is TODO off 64 bits, the FFMA form
// 5.1e-7.  Six bf16 products run at some 375 TFLOP/s, FFMA at 75.
//
// A CTA has a tile of 128 x 128 or 128 x 64.  Sixteen warps take a stage's floats from global memory (the next stage's are on their way in
// registers meanwhile), cut them into three planes in shared memory (two stages) and add up the sums of the stage before, 32
// or 16 columns of a row a thread; a seventeenth issues the MMAs.  Where there are few tiles a cluster of 2, 4 or 8 CTAs splits the
// contraction and exchanges its parts through distributed shared memory.
#include <climits>

#include "clusters.cuh"
#include "common.cuh"
#include "tc.cuh"

namespace toma {

using namespace tc;

namespace {

constexpr int kStep = 64;                     // contraction elements of a stage
constexpr int kPlaneA = 128 * 128, kSlab = kStep * 128;
constexpr int kWarps = 16;                    // that cut and add
template <int NT> constexpr int kStageBytes = 3 * (kPlaneA + NT / 64 * kSlab);
template <int NT> constexpr int kSmem = 1024 + 2 * kStageBytes<NT> + 256;

struct F32Bars {
  uint64_t full[2], done[2], taken[2];  // planes are there; products are through; sums have been taken
  uint32_t tmem_base;
  int abort_flag;
};

struct F32Op {
  const float *a, *w, *bias, *residual;
  float* c;
  int lda, ldr, ldc, M, N, K, act;
};

__device__ __forceinline__ float activate(float x, int act) {
  if (act == kActGelu) return 0.5f * x * erfcf(-0.70710678118654752f * x);
  if (act == kActNone) return x;
  return x / (1.f + expf(-(act == kActSilu ? x : x * fmaf(0.0713548162f, x * x, 1.59576912f))));
}

// Eight floats as three packets of bf16.
__device__ __forceinline__ void cut(const float4& lo, const float4& hi, uint8_t* at, int plane) {
  float v[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
  for (int p = 0; p < 3; ++p) {
    uint32_t q[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * e], v[2 * e + 1]);
      q[e] = *reinterpret_cast<const uint32_t*>(&b);
      if (p < 2) unpack2(sub2(pack2(v[2 * e], v[2 * e + 1]), pack2(__uint_as_float(q[e] << 16), __uint_as_float(q[e] & 0xFFFF0000u))), v[2 * e], v[2 * e + 1]);
    }
    *reinterpret_cast<uint4*>(at + p * plane) = make_uint4(q[0], q[1], q[2], q[3]);
  }
}

template <int NT, int S>
__global__ void __launch_bounds__((kWarps + 1) * 32, 1) linear_f32_kernel(const F32Op o, uint32_t* dev_status) {
  constexpr int kCols = NT / 4, kItemsW = NT / 64;  // columns of a thread; packets of w of a thread (two of a)
  constexpr int kPart = kCols / S;                  // columns that a CTA finishes in a thread
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  F32Bars* bar = reinterpret_cast<F32Bars*>(smem + 2 * kStageBytes<NT>);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = S > 1 ? (int)cluster_rank() : 0, tile = blockIdx.x / S;
  const int nk = (o.K + kStep - 1) / kStep, first = rank * nk / S, steps = (rank + 1) * nk / S - first;  // (nk >= S: one at least)
  const int mb = (o.M + 127) / 128, m0 = tile % mb * 128, n0 = tile / mb * NT;

  if (tid == 0) {
    for (int s = 0; s < 2; ++s) {
      mbar_init(&bar->full[s], kWarps);
      mbar_init(&bar->done[s], 1);
      mbar_init(&bar->taken[s], kWarps);
    }
    bar->abort_flag = 0;
    mbar_fence_init();
  }
  dependency_wait();
  if (tid == 0) release_dependents();
  if (warp == kWarps) tmem_alloc(&bar->tmem_base, 2 * NT);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = bar->tmem_base;
  volatile int* abort_flag = &bar->abort_flag;
  bool ok = true;

  float acc[kCols] = {};
  const int quarter = warp & 3, group = warp >> 2, m = m0 + quarter * 32 + lane;
  if (warp == kWarps) {
    if (elect_one()) {
      constexpr uint32_t idesc = idesc_f16(kFmtBF16, kFmtBF16, false, true, 128, NT);
      for (int i = 0; i < steps; ++i) {
        const int s = i & 1;
        if (!mbar_wait(&bar->full[s], (i >> 1) & 1, dev_status, abort_flag)) break;
        if (i >= 2 && !mbar_wait(&bar->taken[s], ((i >> 1) - 1) & 1, dev_status, abort_flag)) break;
        tc_fence_after();
        const uint32_t aa = smem_u32(smem + s * kStageBytes<NT>), wa = aa + 3 * kPlaneA;
        constexpr int pa[6] = {2, 0, 1, 1, 0, 0}, pw[6] = {0, 2, 1, 0, 1, 0};  // the smallest first
#pragma unroll
        for (int p = 0; p < 6; ++p)
#pragma unroll
          for (int kk = 0; kk < kStep / 16; ++kk)
            mma_ss(tmem + s * NT, smem_desc_sw128(aa + pa[p] * kPlaneA + kk * 32, 16, 1024),
                   smem_desc_sw128(wa + pw[p] * (NT / 64 * kSlab) + kk * 2048, kSlab, 1024), idesc, p > 0 || kk > 0);
        mma_commit(&bar->done[s]);
      }
    }
  } else {
    float4 xa[2][2], xw[kItemsW][2];
    const float4 none = make_float4(0.f, 0.f, 0.f, 0.f);
    const auto fetch = [&](int step) {
      const int k0 = (first + step) * kStep;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int i = tid + j * 512, r = m0 + (i >> 3), k = k0 + (i & 7) * 8;
        const float* at = o.a + (size_t)r * o.lda + k;
        xa[j][0] = r < o.M && k < o.K ? *reinterpret_cast<const float4*>(at) : none;
        xa[j][1] = r < o.M && k + 4 < o.K ? *reinterpret_cast<const float4*>(at + 4) : none;
      }
#pragma unroll
      for (int j = 0; j < kItemsW; ++j) {
        const int i = tid + j * 512, k = k0 + i / (NT / 8), n = n0 + i % (NT / 8) * 8;
        const float* at = o.w + (size_t)k * o.N + n;
        xw[j][0] = k < o.K && n < o.N ? *reinterpret_cast<const float4*>(at) : none;
        xw[j][1] = k < o.K && n + 4 < o.N ? *reinterpret_cast<const float4*>(at + 4) : none;
      }
    };
    const auto take = [&](int step) {  // the sums of a stage
      const int s = step & 1;
      if (!mbar_wait_warp(&bar->done[s], (step >> 1) & 1, dev_status, abort_flag)) return false;
      tc_fence_after();
      uint32_t r[kCols];
      const uint32_t at = tmem + s * NT + group * kCols + ((uint32_t)(quarter * 32) << 16);
      if constexpr (kCols == 32) tmem_ld32(at, r);
      else tmem_ld16(at, r);
      tmem_wait_ld();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&bar->taken[s]);
#pragma unroll
      for (int e = 0; e < kCols; ++e) acc[e] += __uint_as_float(r[e]);
      return true;
    };
    fetch(0);
    for (int i = 0; i < steps; ++i) {
      // (the slot's last products were waited for when their sums were taken)
      uint8_t* sa = smem + (i & 1) * kStageBytes<NT>;
      uint8_t* sw = sa + 3 * kPlaneA;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int e = tid + j * 512;
        cut(xa[j][0], xa[j][1], sa + sw128_offset(e >> 3, e & 7), kPlaneA);
      }
#pragma unroll
      for (int j = 0; j < kItemsW; ++j) {
        const int e = tid + j * 512, k = e / (NT / 8), p = e % (NT / 8);
        cut(xw[j][0], xw[j][1], sw + (p >> 3) * kSlab + sw128_offset(k, p & 7), NT / 64 * kSlab);
      }
      fence_proxy_async();
      __syncwarp();
      if (lane == 0) mbar_arrive(&bar->full[i & 1]);
      if (i + 1 < steps) fetch(i + 1);
      if (i > 0 && !take(i - 1)) { ok = false; break; }
    }
    if (ok) ok = take(steps - 1);
  }

  if constexpr (S > 1) {
    cluster_arrive();
    cluster_wait();  // nobody's products read the stages any more: they take the parts, [other rank][column / 4][thread]
    if (warp < kWarps) {
#pragma unroll
      for (int q = 0; q < S; ++q) {
        if (q == rank) continue;
#pragma unroll
        for (int e = 0; e < kPart; e += 4) {
          const uint32_t at = peer_addr(smem_u32(smem + (((rank < q ? rank : rank - 1) * (kPart / 4) + e / 4) * 512 + tid) * 16), (uint32_t)q);
          const uint32_t v[4] = {__float_as_uint(acc[q * kPart + e]), __float_as_uint(acc[q * kPart + e + 1]), __float_as_uint(acc[q * kPart + e + 2]),
                                 __float_as_uint(acc[q * kPart + e + 3])};
          st_peer_v4(at, v);
        }
      }
    }
    cluster_arrive();
    cluster_wait();  // the parts of all are there; nobody writes any more
  }
  if (warp < kWarps && ok && m < o.M) {
    float own[kPart];
#pragma unroll
    for (int q = 0; q < S; ++q)
      if (q == rank)
#pragma unroll
        for (int e = 0; e < kPart; ++e) own[e] = acc[q * kPart + e];
    float v[kPart] = {};
#pragma unroll
    for (int r = 0; r < S; ++r)
#pragma unroll
      for (int e = 0; e < kPart; e += 4) {
        float4 p;
        if (r == rank) p = make_float4(own[e], own[e + 1], own[e + 2], own[e + 3]);
        else p = *reinterpret_cast<const float4*>(smem + (((r < rank ? r : r - 1) * (kPart / 4) + e / 4) * 512 + tid) * 16);
        v[e] += p.x, v[e + 1] += p.y, v[e + 2] += p.z, v[e + 3] += p.w;
      }
    const int n_first = n0 + group * kCols + rank * kPart;
    // An infinity is no sum of three numbers: where one or a none-number has come in, the sums are taken as they are defined.  (A
    // row with a none-number in it has nothing else, so that rows of padding do not cost their length times the columns.)
    bool odd = false;
#pragma unroll
    for (int e = 0; e < kPart; ++e) odd |= n_first + e < o.N && !(fabsf(v[e]) < INFINITY);
    if (odd) {
      const float* row = o.a + (size_t)m * o.lda;
      bool none = false;
      for (int k = 0; k < o.K; k += 4) {
        const float4 q = *reinterpret_cast<const float4*>(row + k);
        none |= q.x != q.x || q.y != q.y || q.z != q.z || q.w != q.w;
      }
#pragma unroll
      for (int e = 0; e < kPart; ++e)
        if (n_first + e < o.N && !(fabsf(v[e]) < INFINITY)) {
          v[e] = none ? __uint_as_float(0x7FC00000u) : 0.f;
          for (int k = none ? o.K : 0; k < o.K; ++k) v[e] = fmaf(row[k], o.w[(size_t)k * o.N + n_first + e], v[e]);
        }
    }
#pragma unroll
    for (int e = 0; e < kPart; e += 4) {
      const int n = n_first + e;
      if (n >= o.N) continue;
      if (o.bias) {
        const float4 b = *reinterpret_cast<const float4*>(o.bias + n);
        v[e] += b.x, v[e + 1] += b.y, v[e + 2] += b.z, v[e + 3] += b.w;
      }
      if (o.act != kActNone) {
#pragma unroll
        for (int u = 0; u < 4; ++u) v[e + u] = activate(v[e + u], o.act);
      }
      if (o.residual) {
        const float4 r = *reinterpret_cast<const float4*>(o.residual + (size_t)m * o.ldr + n);
        v[e] += r.x, v[e + 1] += r.y, v[e + 2] += r.z, v[e + 3] += r.w;
      }
      *reinterpret_cast<float4*>(o.c + (size_t)m * o.ldc + n) = make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]);
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == kWarps) {
    tc_fence_after();
    tmem_dealloc(tmem, 2 * NT);
  }
}

template <int NT, int S>
int f32_at_once() {
  static ClusterState st;
  return clusters_at_once(linear_f32_kernel<NT, S>, st, S, (kWarps + 1) * 32, kSmem<NT>);
}
template <int NT, int S>
cudaError_t run_f32(const F32Op& o, uint32_t* dev_status, cudaStream_t s) {
  const long long ctas = (long long)((o.M + 127) / 128) * ((o.N + NT - 1) / NT) * S;
  if (ctas > INT32_MAX) return cudaErrorInvalidValue;
  return launch_dependent_cluster(linear_f32_kernel<NT, S>, dim3((unsigned)ctas), dim3((kWarps + 1) * 32), (size_t)kSmem<NT>, S, s, o, dev_status);
}

}  // namespace

// Rows of 16-byte packets: what the kernel loads and stores.
bool linear_f32_tc_ok(const LinearPlusOp& o) {
  return o.M > 16 && o.N % 4 == 0 && o.K % 4 == 0 && o.lda % 4 == 0 && o.ldc % 4 == 0 && (!o.residual || o.ldr % 4 == 0);
}

cudaError_t launch_linear_f32_tc(const LinearPlusOp& l, uint32_t* dev_status, cudaStream_t s) {
  const F32Op o{(const float*)l.a, (const float*)l.w, (const float*)l.bias, (const float*)l.residual, (float*)l.c, l.lda, l.ldr, l.ldc, l.M, l.N, l.K, l.act};
  const int steps = (l.K + kStep - 1) / kStep;
  struct Form {
    int cols, parts, at_once, launch, step;
    cudaError_t (*run)(const F32Op&, uint32_t*, cudaStream_t);
  };
  const Form forms[] = {{128, 1, f32_at_once<128, 1>(), 5000, 900, run_f32<128, 1>}, {64, 1, f32_at_once<64, 1>(), 5000, 600, run_f32<64, 1>},
                        {128, 2, f32_at_once<128, 2>(), 7000, 900, run_f32<128, 2>}, {128, 4, f32_at_once<128, 4>(), 7000, 900, run_f32<128, 4>},
                        {64, 2, f32_at_once<64, 2>(), 7000, 600, run_f32<64, 2>},    {64, 4, f32_at_once<64, 4>(), 7000, 600, run_f32<64, 4>}};
  int best = -1;
  long long least = LLONG_MAX;
  const int tune = g_tune_linear_tile.load(std::memory_order_relaxed);  // test-only
  for (int i = 0; i < 6; ++i) {
    const Form& f = forms[i];
    if (f.at_once < 1 || steps < f.parts) continue;
    const long long tiles = (long long)((l.M + 127) / 128) * ((l.N + f.cols - 1) / f.cols);
    const long long cost = (tiles + f.at_once - 1) / f.at_once * (f.launch + (long long)((steps + f.parts - 1) / f.parts) * f.step);
    if (cost < least || tune == i + 1) least = tune == i + 1 ? -1 : cost, best = i;
  }
  if (best < 0) return cudaErrorInvalidValue;
  const cudaError_t e = forms[best].run(o, dev_status, s);
  count_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace toma
