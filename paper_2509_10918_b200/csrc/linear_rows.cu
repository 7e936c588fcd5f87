// c = act(a w + bias) + residual for at most 16 rows of a: a modulation vector out of a time embedding, a single token.
//
// What there is to do is to read w once: 2 m <= 32 multiply-adds per weight are far below what the SMs have, and tiles of 128
// rows leave most SMs without a tile.  So 64 columns of w are a cluster's, its CTAs split the contraction between them and their
// eight warps split it further, with no staging in shared memory: a weight goes from global memory into the operand registers of
// an mma.sync (the legacy tensor path, whose rate does not matter here: 32 columns of 16 padded rows take 16 instructions per 2 KB
// of weights).  The order of the contraction elements inside an instruction is free as long as both operands use the same, and is
// chosen so that a thread's elements are consecutive in memory:
//   bf16, w [k][n]: 32 elements at a time, thread t of four has elements 8 t .. 8 t + 7, each as 16 bytes of a row of w (eight columns,
//   one of each of eight instructions: columns 8 g + j form instruction j), paired by byte permutations; of a it has 16 bytes.
//   e4m3, w [n][k]: 64 elements at a time, thread t has elements 16 t .. 16 t + 15, 16 bytes of a column, and of a row of a.
// The warps' sums are added up through shared memory, the CTAs' through distributed shared memory, in a fixed order.
// 2 x 5120 x 1280 in bf16 (13 MB of weights, out of L2) 7.1 us, 1 x 640 x 640 3.7, 8-bit 2 x 1280 x 5120 6.0; tiles of 128 rows took 9.5,
// 6.5 and 14.6.  A norm of one row of 608, all latency, takes 1.8.
#include "clusters.cuh"
#include "linear_epilogue.cuh"

namespace toma {

using namespace tc;
using namespace epi;

namespace {

constexpr int kWarps = 8, kBlock = 64, kPitch = kBlock + 4;

__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_e4m3(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint4 load16(const void* p) { return *reinterpret_cast<const uint4*>(p); }
__device__ __forceinline__ uint4 none16() { return make_uint4(0, 0, 0, 0); }
// 16 bytes of a row of e4m3, `left` (a multiple of 8) of them real; nothing behind them is read.
__device__ __forceinline__ uint4 load16_e4m3(const uint8_t* p, int left) {
  if (left >= 16) return load16(p);
  if (left < 8) return none16();
  const uint2 q = *reinterpret_cast<const uint2*>(p);
  return make_uint4(q.x, q.y, 0, 0);
}
__device__ __forceinline__ uint32_t word(const uint4& q, int i) { return i == 0 ? q.x : i == 1 ? q.y : i == 2 ? q.z : q.w; }

// An eight of columns of a row: the sums of the warps, and of all CTAs of the cluster where `mine`.
template <int kRows>
__device__ __forceinline__ void add_up(const float (&part)[kWarps][kRows][kPitch], float (&sums)[8][kRows][8], int split, int rank, int row, int oct,
                                       bool mine, float (&v)[8]) {
  const int per = 8 / split;
  __syncthreads();
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = 0.f;
  if (row < kRows) {
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const float4 x = *reinterpret_cast<const float4*>(&part[w][row][oct * 8]), y = *reinterpret_cast<const float4*>(&part[w][row][oct * 8 + 4]);
      v[0] += x.x, v[1] += x.y, v[2] += x.z, v[3] += x.w, v[4] += y.x, v[5] += y.y, v[6] += y.z, v[7] += y.w;
    }
  }
  if (split > 1) {
    cluster_wait();  // all CTAs have begun
    if (row < kRows) {
      // to who finishes this eight, which has per of them a row
      const uint32_t at = peer_addr(smem_u32(&sums[0][0][0]) + (uint32_t)(((rank * kRows + row) * per + oct % per) * 32), (uint32_t)(oct / per));
      uint32_t b[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) b[e] = __float_as_uint(v[e]);
      st_peer_v4(at, b);
      st_peer_v4(at + 16, b + 4);
    }
    cluster_arrive();
    cluster_wait();  // all sums are there, and nobody writes into another's any more
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = 0.f;
    if (mine) {
      for (int r = 0; r < split; ++r) {
        const float* at = &sums[0][0][0] + ((r * kRows + row) * per + oct % per) * 8;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += at[e];
      }
    }
  }
}

struct RowsOp {
  const void *a, *w;
  int lda, ldw, M, N, K, act, split;
};

// The operands of one step: eight packets of w, the packets of rows g and g + 8 of a.
template <int kKind, bool kTall>
struct Step {
  uint4 w[8], a[kTall ? 2 : 1];
  __device__ __forceinline__ void load(const RowsOp& o, int step, int n0, int g, int t, bool there) {
    if constexpr (kKind == kPlus8) {
      const int k = step * 64 + 16 * t, left = there ? o.K - k : 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int n = n0 + 8 * j + g;
        w[j] = load16_e4m3((const uint8_t*)o.w + (size_t)n * o.ldw + k, n < o.N ? left : 0);
      }
#pragma unroll
      for (int i = 0; i < (kTall ? 2 : 1); ++i) a[i] = load16_e4m3((const uint8_t*)o.a + (size_t)(g + 8 * i) * o.lda + k, g + 8 * i < o.M ? left : 0);
    } else {
      const int k = step * 32 + 8 * t;
      const bool in_k = there && k < o.K;
      const __nv_bfloat16* at = (const __nv_bfloat16*)o.w + (size_t)k * o.N + n0 + 8 * g;
#pragma unroll
      for (int j = 0; j < 8; ++j) w[j] = in_k && n0 + 8 * g < o.N ? load16(at + (size_t)j * o.N) : none16();
#pragma unroll
      for (int i = 0; i < (kTall ? 2 : 1); ++i)
        a[i] = in_k && g + 8 * i < o.M ? load16((const __nv_bfloat16*)o.a + (size_t)(g + 8 * i) * o.lda + k) : none16();
    }
  }
  __device__ __forceinline__ void multiply(float (&acc)[8][4]) const {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const uint32_t a0 = word(a[0], 2 * s), a2 = word(a[0], 2 * s + 1), a1 = kTall ? word(a[kTall ? 1 : 0], 2 * s) : 0, a3 = kTall ? word(a[kTall ? 1 : 0], 2 * s + 1) : 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if constexpr (kKind == kPlus8) {
          mma_e4m3(acc[j], a0, a1, a2, a3, word(w[j], 2 * s), word(w[j], 2 * s + 1));
        } else {
          const uint32_t pick = j % 2 ? 0x7632 : 0x5410;  // the column's half of two rows' words
          mma_bf16(acc[j], a0, a1, a2, a3, __byte_perm(word(w[4 * s], j / 2), word(w[4 * s + 1], j / 2), pick),
                   __byte_perm(word(w[4 * s + 2], j / 2), word(w[4 * s + 3], j / 2), pick));
        }
      }
    }
  }
};

template <int kKind, bool kTall>
__global__ void __launch_bounds__(kWarps * 32, 2) linear_rows_kernel(const RowsOp o, const LinearPlus plus) {
  constexpr int kRows = kTall ? 16 : 8;
  __shared__ __align__(16) float part[kWarps][kRows][kPitch];
  __shared__ __align__(16) float sums[8][kRows][8];  // [rank][row] eights of columns that this CTA finishes, 8 / split of them
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int rank = o.split > 1 ? (int)cluster_rank() : 0, n0 = (int)(blockIdx.x / o.split) * kBlock;
  const int steps = (o.K + (kKind == kPlus8 ? 63 : 31)) / (kKind == kPlus8 ? 64 : 32), parts = kWarps * o.split, p = rank * kWarps + warp;
  const int first = (int)((long long)steps * p / parts), last = (int)((long long)steps * (p + 1) / parts);
  dependency_wait();
  if (threadIdx.x == 0) release_dependents();
  if (o.split > 1) cluster_arrive();

  // rows x 8 threads finish: an eight of columns of a row each, of the eights that are this CTA's
  const int row = threadIdx.x >> 3, oct = threadIdx.x & 7, per = 8 / o.split, n = n0 + oct * 8;
  const bool mine = row < o.M && row < kRows && oct / per == rank && n < o.N;
  uint4 res = none16();
  float acc[8][4] = {};
  Step<kKind, kTall> s0, s1;
  s0.load(o, first, n0, g, t, first < last);
  s1.load(o, first + 1, n0, g, t, first + 1 < last);
  if (mine && plus.residual) res = load16(plus.residual + (size_t)row * plus.ldr + n);
  for (int k = first; k < last; k += 2) {
    s0.multiply(acc);
    if (k + 2 < last) s0.load(o, k + 2, n0, g, t, true);
    if (k + 1 < last) s1.multiply(acc);
    if (k + 3 < last) s1.load(o, k + 3, n0, g, t, true);
  }
#pragma unroll
  for (int i = 0; i < (kTall ? 2 : 1); ++i) {
    float* at = part[warp][g + 8 * i];
    if constexpr (kKind == kPlus8) {
#pragma unroll
      for (int j = 0; j < 8; ++j) *reinterpret_cast<float2*>(at + 8 * j + 2 * t) = make_float2(acc[j][2 * i], acc[j][2 * i + 1]);
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h) {  // columns 8 (2 t + h) + j
        *reinterpret_cast<float4*>(at + 16 * t + 8 * h) = make_float4(acc[0][2 * i + h], acc[1][2 * i + h], acc[2][2 * i + h], acc[3][2 * i + h]);
        *reinterpret_cast<float4*>(at + 16 * t + 8 * h + 4) = make_float4(acc[4][2 * i + h], acc[5][2 * i + h], acc[6][2 * i + h], acc[7][2 * i + h]);
      }
    }
  }
  float v[8];
  add_up<kRows>(part, sums, o.split, rank, row, oct, mine, v);
  if (mine) finish8<kKind>(v, kKind == kPlus8 ? plus.a_scale[row] : 1.f, plus, o.act, res, n, plus.c + (size_t)row * plus.ldc + n);
}

// The same in fp32 on FFMA: a thread has four columns of w and four consecutive contraction elements of every 64, sixteen threads
// beside one another the columns, sixteen the elements.
template <int kRows>
__global__ void __launch_bounds__(kWarps * 32) linear_rows_f32_kernel(const RowsOp o, const float* bias, const float* residual, float* c, int ldr, int ldc) {
  __shared__ __align__(16) float part[kWarps][kRows][kPitch];
  __shared__ __align__(16) float sums[8][kRows][8];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, col = (threadIdx.x & 15) * 4, k_lane = threadIdx.x >> 4;
  const int rank = o.split > 1 ? (int)cluster_rank() : 0, n0 = (int)(blockIdx.x / o.split) * kBlock;
  const int steps = (o.K + 63) / 64, first = (int)((long long)steps * rank / o.split), last = (int)((long long)steps * (rank + 1) / o.split);
  dependency_wait();
  if (threadIdx.x == 0) release_dependents();
  if (o.split > 1) cluster_arrive();
  const int row = threadIdx.x >> 3, oct = threadIdx.x & 7, n = n0 + oct * 8;
  const bool mine = row < o.M && row < kRows && oct / (8 / o.split) == rank && n < o.N;
  const bool in_n = n0 + col < o.N;
  float acc[kRows][4] = {};
  const float4 none = make_float4(0.f, 0.f, 0.f, 0.f);
  float4 w[4], a[kRows];
  const auto load = [&](int step) {
    const int k = step * 64 + k_lane * 4;
    const bool in_k = k < o.K;
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = in_k && in_n ? *reinterpret_cast<const float4*>((const float*)o.w + (size_t)(k + e) * o.N + n0 + col) : none;
#pragma unroll
    for (int r = 0; r < kRows; ++r) a[r] = in_k && r < o.M ? *reinterpret_cast<const float4*>((const float*)o.a + (size_t)r * o.lda + k) : none;
  };
  if (first < last) load(first);
  for (int s = first; s < last; ++s) {
    float4 ww[4], aa[kRows];
#pragma unroll
    for (int e = 0; e < 4; ++e) ww[e] = w[e];
#pragma unroll
    for (int r = 0; r < kRows; ++r) aa[r] = a[r];
    if (s + 1 < last) load(s + 1);
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      const float x[4] = {aa[r].x, aa[r].y, aa[r].z, aa[r].w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        acc[r][0] = fmaf(x[e], ww[e].x, acc[r][0]);
        acc[r][1] = fmaf(x[e], ww[e].y, acc[r][1]);
        acc[r][2] = fmaf(x[e], ww[e].z, acc[r][2]);
        acc[r][3] = fmaf(x[e], ww[e].w, acc[r][3]);
      }
    }
  }
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[r][e] += __shfl_xor_sync(0xffffffffu, acc[r][e], 16);
    if (lane < 16) *reinterpret_cast<float4*>(&part[warp][r][col]) = make_float4(acc[r][0], acc[r][1], acc[r][2], acc[r][3]);
  }
  float v[8];
  add_up<kRows>(part, sums, o.split, rank, row, oct, mine, v);
  if (!mine) return;
#pragma unroll
  for (int h = 0; h < 8; h += 4) {
    if (n + h >= o.N) break;
    const float4 b = bias ? *reinterpret_cast<const float4*>(bias + n + h) : none;
    const float4 r = residual ? *reinterpret_cast<const float4*>(residual + (size_t)row * ldr + n + h) : none;
    *reinterpret_cast<float4*>(c + (size_t)row * ldc + n + h) =
        make_float4(activate_f32(v[h] + b.x, o.act) + r.x, activate_f32(v[h + 1] + b.y, o.act) + r.y, activate_f32(v[h + 2] + b.z, o.act) + r.z,
                    activate_f32(v[h + 3] + b.w, o.act) + r.w);
  }
}

// CTAs that split a block's contraction (1, 2, 4 or 8): twice the SMs in all at most, `least` steps for each, and as many as the device
// places beside one another.
template <typename Kernel>
int split_of(Kernel kernel, ClusterState (&st)[3], int N, int steps, int least) {
  const int blocks = (N + kBlock - 1) / kBlock;
  int split = 1;
  for (int i = 0; i < 3 && blocks * split * 2 <= 2 * sm_count() && steps >= least * split; ++i) {
    if (clusters_at_once(kernel, st[i], 2 << i, kWarps * 32, 0) < 1) break;
    split *= 2;
  }
  return split;
}

template <int kRows>
cudaError_t run_rows_f32(const LinearPlusOp& l, cudaStream_t s) {
  static ClusterState st[3];
  const int blocks = (l.N + kBlock - 1) / kBlock, split = split_of(linear_rows_f32_kernel<kRows>, st, l.N, (l.K + 63) / 64, 4);
  const RowsOp o{l.a, l.w, l.lda, l.ldw, l.M, l.N, l.K, l.act, split};
  return launch_dependent_cluster(linear_rows_f32_kernel<kRows>, dim3((unsigned)(blocks * split)), dim3(kWarps * 32), 0, split, s, o, (const float*)l.bias,
                                  (const float*)l.residual, (float*)l.c, l.ldr, l.ldc);
}

template <int kKind, bool kTall>
cudaError_t run_rows(const LinearPlusOp& l, const LinearPlus& plus, cudaStream_t s) {
  static ClusterState st[3];
  const int step = kKind == kPlus8 ? 64 : 32, split = split_of(linear_rows_kernel<kKind, kTall>, st, l.N, (l.K + step - 1) / step, kWarps);
  const RowsOp o{l.a, l.w, l.lda, l.ldw, l.M, l.N, l.K, l.act, split};
  return launch_dependent_cluster(linear_rows_kernel<kKind, kTall>, dim3((unsigned)((l.N + kBlock - 1) / kBlock) * split), dim3(kWarps * 32), 0, split, s, o,
                                  plus);
}

}  // namespace

cudaError_t launch_linear_rows(const LinearPlusOp& l, bool f32, cudaStream_t s) {
  cudaError_t e;
  if (f32) {
    e = l.M > 8 ? run_rows_f32<16>(l, s) : run_rows_f32<8>(l, s);
  } else {
    const LinearPlus plus{(const __nv_bfloat16*)l.bias, (const __nv_bfloat16*)l.residual, l.a_scale, l.w_scale, (__nv_bfloat16*)l.c, l.ldc, l.ldr};
    e = l.f8 ? (l.M > 8 ? run_rows<kPlus8, true>(l, plus, s) : run_rows<kPlus8, false>(l, plus, s))
             : (l.M > 8 ? run_rows<kPlus, true>(l, plus, s) : run_rows<kPlus, false>(l, plus, s));
  }
  count_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace toma
