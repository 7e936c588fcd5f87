// c = act(a w + bias) + residual for at most 16 rows of a: a modulation vector out of a time embedding, a single token.
//
// What there is to do is to read w once: 2 m <= 32 multiply-adds per weight are far below what the SMs have, and tiles of 128
// rows leave most SMs without a tile.  So 64 columns of w are a cluster's, its CTAs split the contraction between them and their
// eight warps split it further, with no staging in shared memory: a weight goes from global memory into the registers that are multiplied,
// two steps of 4 KB per warp on their way.  With more than two rows in bf16, and in e4m3, these are the operands of an mma.sync (the legacy
// tensor path, whose rate does not matter here: 32 columns of 16 padded rows take 16 instructions per 2 KB of weights).  The order of
// the contraction elements inside an instruction is free as long as both operands use the same, and is chosen so that a thread's elements
// are consecutive in memory:
//   bf16, w [k][n]: 32 elements at a time, thread t of four has elements 8 t .. 8 t + 7, each as 16 bytes of a row of w (eight columns,
//   one of each of eight instructions: columns 8 g + j form instruction j), paired by byte permutations; of a it has 16 bytes.
//   e4m3, w [n][k]: 64 elements at a time, thread t has elements 16 t .. 16 t + 15, 16 bytes of a column, and of a row of a.
// One or two rows in bf16, and fp32, are multiplied on FFMA (linear_few_kernel, linear_rows_f32_kernel).
// The warps' sums are added up through shared memory, the CTAs' through distributed shared memory, in a fixed order; bias, scales and
// residual are on their way meanwhile.
// In us, weights out of L2 / DRAM.  2 rows in bf16: 5120 x 1280 4.8 / 5.9, 1280 x 5120 5.5 / 6.8, 5120 x 5120 9.4 / 12.4 (52 MB, 4.2 TB/s),
// 640 x 640 2.9; in e4m3: 1280 x 5120 5.0 / 5.8, 5120 x 5120 7.7 / 9.8, 10240 x 5120 14.2 / 15.9 (52 MB, 3.3 TB/s); in fp32: 5120 x 1280
// 6.4 / 8.1, 10240 x 5120 36.9 (5.7 TB/s).  8 rows in bf16: 5120 x 1280 6.0 / 7.1, 5120 x 5120 11.7 / 13.6.  Tiles of 128 rows took 9.5 for
// 2 x 5120 x 1280, 6.5 for 1 x 640 x 640 and 14.6 for 2 x 1280 x 5120 in e4m3.
// A norm of one row of 608, all latency, takes 1.8.
#include <climits>
#include <mutex>

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

// An eight of columns of a row: the sums of the warps, and of all CTAs of the cluster where `mine`.  CTA r finishes the eights r,
// r + split, ... and gets every CTA's sums of them, ceil(8 / split) a row.
constexpr int kSums = 14;  // split ceil(8 / split) at most
template <int kRows, int kOcts = kBlock / 8>
__device__ __forceinline__ void add_up(const float (&part)[kWarps][kRows][kPitch], float (&sums)[kSums][kRows][8], int split, int rank, int row, int oct,
                                       bool mine, float (&v)[8]) {
  const int per = (kOcts - 1 + split) / split;
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
      const uint32_t at = peer_addr(smem_u32(&sums[0][0][0]) + (uint32_t)(((rank * kRows + row) * per + oct / split) * 32), (uint32_t)(oct % split));
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
        const float* at = &sums[0][0][0] + ((r * kRows + row) * per + oct / split) * 8;
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
      const int k = step * 64 + 16 * t, cols = o.N - n0 - g;
      const uint8_t* w_at = (const uint8_t*)o.w + (size_t)(n0 + g) * o.ldw + k;
      const uint8_t* a_at = (const uint8_t*)o.a + (size_t)g * o.lda + k;
      if (there && step * 64 + 64 <= o.K) {  // (a step's end inside a packet is tested for once, not for each)
#pragma unroll
        for (int j = 0; j < 8; ++j, w_at += (size_t)8 * o.ldw) w[j] = 8 * j < cols ? load16(w_at) : none16();
#pragma unroll
        for (int i = 0; i < (kTall ? 2 : 1); ++i, a_at += (size_t)8 * o.lda) a[i] = g + 8 * i < o.M ? load16(a_at) : none16();
      } else {
        const int left = there ? o.K - k : 0;
#pragma unroll
        for (int j = 0; j < 8; ++j, w_at += (size_t)8 * o.ldw) w[j] = load16_e4m3(w_at, 8 * j < cols ? left : 0);
#pragma unroll
        for (int i = 0; i < (kTall ? 2 : 1); ++i, a_at += (size_t)8 * o.lda) a[i] = load16_e4m3(a_at, g + 8 * i < o.M ? left : 0);
      }
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
  __shared__ __align__(16) float sums[kSums][kRows][8];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int rank = o.split > 1 ? (int)cluster_rank() : 0, n0 = (int)(blockIdx.x / o.split) * kBlock;
  const int steps = (o.K + (kKind == kPlus8 ? 63 : 31)) / (kKind == kPlus8 ? 64 : 32), parts = kWarps * o.split, p = rank * kWarps + warp;
  const int first = (int)((long long)steps * p / parts), last = (int)((long long)steps * (p + 1) / parts);
  dependency_wait();
  if (threadIdx.x == 0) release_dependents();
  if (o.split > 1) cluster_arrive();

  // rows x 8 threads finish: an eight of columns of a row each, of the eights that are this CTA's
  const int row = threadIdx.x >> 3, oct = threadIdx.x & 7, n = n0 + oct * 8;
  const bool mine = row < o.M && row < kRows && oct % o.split == rank && n < o.N;
  float acc[8][4] = {};
  Step<kKind, kTall> s0, s1;
  s0.load(o, first, n0, g, t, first < last);
  s1.load(o, first + 1, n0, g, t, first + 1 < last);
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
  Finish8<kKind> finish;  // its loads run under the exchange of the sums
  if (mine) finish.fetch(plus, row, n);
  float v[8];
  add_up<kRows>(part, sums, o.split, rank, row, oct, mine, v);
  if (mine) finish.out(v, plus, o.act, plus.c + (size_t)row * plus.ldc + n);
}

// One or two rows in bf16 on FFMA.  An MMA wants lanes beside one another on different rows of w, 32 bytes of each, and each such piece is
// a wavefront of L1 (sixteen for a load of 512 bytes); here kCols / 8 lanes run along a row of w, eight columns each, and 256 / kCols such
// groups have eight rows each.  2 x 5120 x 5120 11.5 -> 9.6 us, split by three both.
template <int kCols>
__global__ void __launch_bounds__(kWarps * 32, 2) linear_few_kernel(const RowsOp o, const LinearPlus plus) {
  constexpr int kRows = 2, kOcts = kCols / 8, kStepK = 256 / kOcts;
  __shared__ __align__(16) float part[kWarps][kRows][kPitch];
  __shared__ __align__(16) float sums[kSums][kRows][8];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, c = lane % kOcts, t = lane / kOcts;
  const int rank = o.split > 1 ? (int)cluster_rank() : 0, n0 = (int)(blockIdx.x / o.split) * kCols;
  const int steps = (o.K + kStepK - 1) / kStepK, parts = kWarps * o.split, p = rank * kWarps + warp;
  const int first = (int)((long long)steps * p / parts), last = (int)((long long)steps * (p + 1) / parts);
  dependency_wait();
  if (threadIdx.x == 0) release_dependents();
  if (o.split > 1) cluster_arrive();
  struct Few {
    uint4 w[8], a[kRows];
  } s[2];
  uint64_t acc[kRows][4] = {};
  const auto load = [&](Few& f, int step) {
    const int k = step * kStepK + 8 * t;
    const bool in_k = step < last && k < o.K;
    const __nv_bfloat16* at = (const __nv_bfloat16*)o.w + (size_t)k * o.N + n0 + 8 * c;
#pragma unroll
    for (int j = 0; j < 8; ++j) f.w[j] = in_k && n0 + 8 * c < o.N ? load16(at + (size_t)j * o.N) : none16();
#pragma unroll
    for (int r = 0; r < kRows; ++r) f.a[r] = in_k && r < o.M ? load16((const __nv_bfloat16*)o.a + (size_t)r * o.lda + k) : none16();
  };
  const auto multiply = [&](const Few& f) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      uint64_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = pack2(__uint_as_float(word(f.w[j], i) << 16), __uint_as_float(word(f.w[j], i) & 0xFFFF0000u));
#pragma unroll
      for (int r = 0; r < kRows; ++r) {
        const uint64_t x = both(__uint_as_float(j % 2 ? word(f.a[r], j / 2) & 0xFFFF0000u : word(f.a[r], j / 2) << 16));
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[r][i] = fma2(x, w[i], acc[r][i]);
      }
    }
  };
  load(s[0], first);
  load(s[1], first + 1);
  for (int k = first; k < last; k += 2) {
    multiply(s[0]);
    load(s[0], k + 2);
    multiply(s[1]);
    load(s[1], k + 3);
  }
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    float v[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) unpack2(acc[r][i], v[2 * i], v[2 * i + 1]);
#pragma unroll
    for (int b = kOcts; b < 32; b *= 2) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += __shfl_xor_sync(0xffffffffu, v[e], b);
    }
    if (t == 0) {
      *reinterpret_cast<float4*>(&part[warp][r][8 * c]) = make_float4(v[0], v[1], v[2], v[3]);
      *reinterpret_cast<float4*>(&part[warp][r][8 * c + 4]) = make_float4(v[4], v[5], v[6], v[7]);
    }
  }
  const int row = threadIdx.x / kOcts, oct = threadIdx.x % kOcts, n = n0 + oct * 8;
  const bool mine = row < o.M && row < kRows && oct % o.split == rank && n < o.N;
  Finish8<kPlus> finish;
  if (mine) finish.fetch(plus, row, n);
  float v[8];
  add_up<kRows, kOcts>(part, sums, o.split, rank, row, oct, mine, v);
  if (mine) finish.out(v, plus, o.act, plus.c + (size_t)row * plus.ldc + n);
}

// The same in fp32 on FFMA: a thread has four columns of w and four consecutive contraction elements of every 64, sixteen threads
// beside one another the columns, sixteen the elements.  As many steps on their way as the registers hold beside the sums, whose
// number is that of the rows: with one step and sums for eight 2 x 10240 x 5120 took 81 us, with three and for two 37.
template <int kRows>
__global__ void __launch_bounds__(kWarps * 32, kRows > 8 ? 1 : 2) linear_rows_f32_kernel(const RowsOp o, const float* bias, const float* residual, float* c, int ldr, int ldc) {
  __shared__ __align__(16) float part[kWarps][kRows][kPitch];
  __shared__ __align__(16) float sums[kSums][kRows][8];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, col = (threadIdx.x & 15) * 4, k_lane = threadIdx.x >> 4;
  const int rank = o.split > 1 ? (int)cluster_rank() : 0, n0 = (int)(blockIdx.x / o.split) * kBlock;
  const int steps = (o.K + 63) / 64, first = (int)((long long)steps * rank / o.split), last = (int)((long long)steps * (rank + 1) / o.split);
  dependency_wait();
  if (threadIdx.x == 0) release_dependents();
  if (o.split > 1) cluster_arrive();
  const int row = threadIdx.x >> 3, oct = threadIdx.x & 7, n = n0 + oct * 8;
  const bool mine = row < o.M && row < kRows && oct % o.split == rank && n < o.N;
  const bool in_n = n0 + col < o.N;
  constexpr int kAhead = kRows > 8 ? 1 : kRows > 2 ? 2 : 3;  // steps on their way: what the registers hold
  float acc[kRows][4] = {};
  const float4 none = make_float4(0.f, 0.f, 0.f, 0.f);
  float4 w[kAhead][4], a[kAhead][kRows];
  const auto load = [&](int step, float4 (&w)[4], float4 (&a)[kRows]) {
    const int k = step * 64 + k_lane * 4;
    const bool in_k = step < last && k < o.K;
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = in_k && in_n ? *reinterpret_cast<const float4*>((const float*)o.w + (size_t)(k + e) * o.N + n0 + col) : none;
#pragma unroll
    for (int r = 0; r < kRows; ++r) a[r] = in_k && r < o.M ? *reinterpret_cast<const float4*>((const float*)o.a + (size_t)r * o.lda + k) : none;
  };
#pragma unroll
  for (int i = 0; i < kAhead; ++i) load(first + i, w[i], a[i]);
  for (int s = first; s < last; s += kAhead) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
#pragma unroll
      for (int r = 0; r < kRows; ++r) {
        const float x[4] = {a[i][r].x, a[i][r].y, a[i][r].z, a[i][r].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          acc[r][0] = fmaf(x[e], w[i][e].x, acc[r][0]);
          acc[r][1] = fmaf(x[e], w[i][e].y, acc[r][1]);
          acc[r][2] = fmaf(x[e], w[i][e].z, acc[r][2]);
          acc[r][3] = fmaf(x[e], w[i][e].w, acc[r][3]);
        }
      }
      load(s + kAhead + i, w[i], a[i]);
    }
  }
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[r][e] += __shfl_xor_sync(0xffffffffu, acc[r][e], 16);
    if (lane < 16) *reinterpret_cast<float4*>(&part[warp][r][col]) = make_float4(acc[r][0], acc[r][1], acc[r][2], acc[r][3]);
  }
  float4 bs[2], rs[2];  // on their way under the exchange of the sums
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const bool in = mine && n + 4 * h < o.N;
    bs[h] = in && bias ? *reinterpret_cast<const float4*>(bias + n + 4 * h) : none;
    rs[h] = in && residual ? *reinterpret_cast<const float4*>(residual + (size_t)row * ldr + n + 4 * h) : none;
  }
  float v[8];
  add_up<kRows>(part, sums, o.split, rank, row, oct, mine, v);
  if (!mine) return;
#pragma unroll
  for (int h = 0; h < 8; h += 4) {
    if (n + h >= o.N) break;
    const float4 b = bs[h / 4], r = rs[h / 4];
    *reinterpret_cast<float4*>(c + (size_t)row * ldc + n + h) =
        make_float4(activate_f32(v[h] + b.x, o.act) + r.x, activate_f32(v[h + 1] + b.y, o.act) + r.y, activate_f32(v[h + 2] + b.z, o.act) + r.z,
                    activate_f32(v[h + 3] + b.w, o.act) + r.w);
  }
}

// How many CTAs split a block's contraction, and the time that it then takes beside what all have in common: what a cluster costs, and a
// part for each step in the longest chain of them (one at least), which is longer where an SM has two CTAs.  In nanoseconds, fitted for
// each kernel (RowsCost) to blocks of 48 matrices between 320 x 200 and 10240 x 5120 split by 1 to 8, with the weights in L2 and in DRAM:
// the split it names takes 1.01 to 1.03 times as long as the best in the mean, 1.21 at most.  What costs most is more CTAs than the
// device has places for (two per SM, fewer for clusters: 33 of eight): a second round of clusters took 3.5 us more for 2 x 5120 x 320 split by
// four.  It is counted as 7, which leaves 2 x 10240 x 5120 in bf16 unsplit (22 us; 24 from DRAM in two rounds) and splits it in fp32 (39 unsplit,
// 37).  Powers of two up to two CTAs per SM, the rule before, had 2 x 5120 x 1280 take 7.0 us, now 4.8, and 2 x 5120 x 640 5.4, now 3.7.
struct RowsCost {
  int cluster, one, two, both, chains;  // ..., a step with one CTA on an SM, with two, what two have besides, chains of steps in a CTA
};
struct RowsSplit {
  int split;
  long long cost;
};
struct RowsDevice {  // (asked once per device)
  std::once_flag once[64];
  int sms[64], at_once[64][8];
  ClusterState st[8];
};
template <typename Kernel>
RowsSplit split_of(Kernel kernel, RowsDevice& known, int blocks, int steps, const RowsCost& c) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return RowsSplit{1, 0};
  std::call_once(known.once[dev], [&] {
    known.sms[dev] = sm_count();
    for (int i = 0; i < 8; ++i) known.at_once[dev][i] = clusters_at_once(kernel, known.st[i], i + 1, kWarps * 32, 0);
  });
  const int tune = g_tune_linear_tile.load(std::memory_order_relaxed);  // test-only: 11 to 18, 21 to 28
  const int asked = tune > 10 ? tune % 10 : 0;
  RowsSplit best{1, LLONG_MAX};
  for (int split = 1; split <= 8; ++split) {
    const int at_once = known.at_once[dev][split - 1];
    if (at_once < 1) continue;
    const int rounds = (blocks + at_once - 1) / at_once;
    const bool both = 2LL * blocks > at_once && at_once * split > known.sms[dev];  // two CTAs on an SM
    const long long step = both ? c.two : c.one, chain = steps * step / (c.chains * split);
    const long long round = (split > 1 ? c.cluster : 0) + (both ? c.both : 0) + (chain > step ? chain : step);
    const long long cost = split == asked ? 0 : rounds * round + (rounds - 1) * (split > 1 ? 7000 : 0);
    if (cost < best.cost) best = RowsSplit{split, cost};
  }
  return best;
}

template <int kRows>
cudaError_t run_rows_f32(const LinearPlusOp& l, const RowsCost& cost, cudaStream_t s) {
  static RowsDevice st;
  const int blocks = (l.N + kBlock - 1) / kBlock, split = split_of(linear_rows_f32_kernel<kRows>, st, blocks, (l.K + 63) / 64, cost).split;
  const RowsOp o{l.a, l.w, l.lda, l.ldw, l.M, l.N, l.K, l.act, split};
  return launch_dependent_cluster(linear_rows_f32_kernel<kRows>, dim3((unsigned)(blocks * split)), dim3(kWarps * 32), 0, split, s, o, (const float*)l.bias,
                                  (const float*)l.residual, (float*)l.c, l.ldr, l.ldc);
}

template <int kKind, bool kTall>
cudaError_t run_rows(const LinearPlusOp& l, const LinearPlus& plus, const RowsCost& cost, cudaStream_t s) {
  static RowsDevice st;
  constexpr int kStepK = kKind == kPlus8 ? 64 : 32;
  const int blocks = (l.N + kBlock - 1) / kBlock, split = split_of(linear_rows_kernel<kKind, kTall>, st, blocks, (l.K + kStepK - 1) / kStepK, cost).split;
  const RowsOp o{l.a, l.w, l.lda, l.ldw, l.M, l.N, l.K, l.act, split};
  return launch_dependent_cluster(linear_rows_kernel<kKind, kTall>, dim3((unsigned)(blocks * split)), dim3(kWarps * 32), 0, split, s, o, plus);
}

template <int kCols>
RowsSplit few_split(const LinearPlusOp& l) {
  static RowsDevice st;
  constexpr int kStepK = 2048 / kCols;
  return split_of(linear_few_kernel<kCols>, st, (l.N + kCols - 1) / kCols, (l.K + kStepK - 1) / kStepK, RowsCost{690, 630, 1240, 100, kWarps});
}
template <int kCols>
cudaError_t run_few(const LinearPlusOp& l, const LinearPlus& plus, int split, cudaStream_t s) {
  const RowsOp o{l.a, l.w, l.lda, l.ldw, l.M, l.N, l.K, l.act, split};
  return launch_dependent_cluster(linear_few_kernel<kCols>, dim3((unsigned)((l.N + kCols - 1) / kCols * split)), dim3(kWarps * 32), 0, split, s, o, plus);
}
// Blocks of 32 columns make twice the CTAs without a cluster where there are few: 2 x 1280 x 640 3.0 us, 3.4 with blocks of 64; those are faster
// where there are enough (2 x 10240 x 1280 6.9, of 32 7.9).  With blocks of 64 alone 40 matrices took 1.06 times as long as the best in the
// mean, of 32 alone 1.08, with both 1.04.
cudaError_t run_few(const LinearPlusOp& l, const LinearPlus& plus, cudaStream_t s) {
  const RowsSplit wide = few_split<64>(l), slim = few_split<32>(l);
  const int tune = g_tune_linear_tile.load(std::memory_order_relaxed);
  return (tune > 10 ? tune > 20 : slim.cost < wide.cost) ? run_few<32>(l, plus, slim.split, s) : run_few<64>(l, plus, wide.split, s);
}

}  // namespace

cudaError_t launch_linear_rows(const LinearPlusOp& l, bool f32, cudaStream_t s) {
  cudaError_t e;
  if (f32) {
    e = l.M > 8   ? run_rows_f32<16>(l, RowsCost{1360, 895, 895, 0, 1}, s)
        : l.M > 4 ? run_rows_f32<8>(l, RowsCost{1320, 550, 925, 1340, 1}, s)
        : l.M > 2 ? run_rows_f32<4>(l, RowsCost{1160, 370, 580, 860, 1}, s)
                  : run_rows_f32<2>(l, RowsCost{1010, 280, 466, 820, 1}, s);
  } else {
    const LinearPlus plus{(const __nv_bfloat16*)l.bias, (const __nv_bfloat16*)l.residual, l.a_scale, l.w_scale, (__nv_bfloat16*)l.c, l.ldc, l.ldr};
    if (l.f8)
      e = l.M > 8 ? run_rows<kPlus8, true>(l, plus, RowsCost{1300, 1300, 2280, 90, kWarps}, s) : run_rows<kPlus8, false>(l, plus, RowsCost{920, 850, 1620, 0, kWarps}, s);
    else
      e = l.M > 8   ? run_rows<kPlus, true>(l, plus, RowsCost{1150, 900, 1680, 320, kWarps}, s)
          : l.M > 2 ? run_rows<kPlus, false>(l, plus, RowsCost{800, 780, 1590, 0, kWarps}, s)
                    : run_few(l, plus, s);
  }
  count_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace toma
