// Dense projection C[m][n] = sum_k A[m][k] W[k][n] on the sm_100a tensor cores (bf16 in, fp32
// accumulation in tensor memory, bf16 out): the QKV and output projections of the attention module
// that ToMA wraps (Algorithm 3's core module F; App. C counts them as the 4 d^2 N term).
//
// Rows of A (tokens) sit on the MMA M dimension.  A is the K-major operand exactly as stored ([m][k] row-major),
// W the MN-major one exactly as stored ([k][n] row-major), so neither is transposed or copied.  Up to three weight /
// output pairs share A (Q, K and V in one launch).  Warp 0 feeds a TMA ring, warp 1 issues the MMAs, the other warps take
// the accumulators out of tensor memory (through the activation when one is asked for: the first layer of the MLP, the
// other module ToMA wraps), stage their 32 rows in shared memory as 64-column slabs in the layout of the output tensor
// map's box and store them with one TMA store per warp and slab: whole lines, asynchronous, instead of 16-byte stores to
// 32 different rows per warp instruction.
//
// C = act(A W + bias) + residual (launch_linear_plus_tc) runs on the same kernels, with A and W in bf16 or in e4m3 (A with a
// scale for each row, W stored [n][k] with a scale for each column): kPlus and kPlus8 below.
#include <climits>
#include <mutex>

#include "clusters.cuh"
#include "common.cuh"
#include "linear_epilogue.cuh"
#include "tc.cuh"

namespace toma {

using namespace tc;
using namespace epi;

namespace {

constexpr int kKC = 64;                  // contraction elements per stage
constexpr int kSlab = kKC * 128;         // [64 k][64 n] slab of W, 128-byte rows
constexpr int kABytes = 128 * 128;       // [128 m][64 k] slab of A

// Contraction elements of a stage, and of an MMA (32 bytes).
template <int kKind> constexpr int kStepK = kKind == kPlus8 ? 2 * kKC : kKC;   // contraction elements per stage
template <int kKind> constexpr int kMmaK = kKind == kPlus8 ? 32 : 16;          // ... per MMA (32 bytes)

// The maps of a stage's slab j of W, and the MMAs of a stage.
template <int kKind>
__device__ __forceinline__ void load_w(void* dst, const CUtensorMap* m, uint64_t* bar, int n, int k) {
  if constexpr (kKind == kPlus8) tma_load_2d(dst, m, bar, k, n);
  else tma_load_2d(dst, m, bar, n, k);
}
template <int kKind>
__device__ __forceinline__ uint64_t w_desc(uint32_t wa, int kk) {
  if constexpr (kKind == kPlus8) return smem_desc_sw128(wa + kk * 32, 16, 1024);
  else return smem_desc_sw128(wa + kk * 2048, kSlab, 1024);
}
// Half a slab: 32 columns, rows of 64 bytes in bf16.
template <int kKind>
__device__ __forceinline__ uint64_t half_desc(uint32_t wa, int kk) {
  if constexpr (kKind == kPlus8) return smem_desc_sw128(wa + kk * 32, 16, 1024);
  else return smem_desc_sw64(wa + kk * 1024, 16, 512);
}
template <int kKind>
__device__ __forceinline__ constexpr uint32_t idesc_of(int M, int N) {
  return kKind == kPlus8 ? idesc_f16(kFmtE4M3, kFmtE4M3, false, false, M, N) : idesc_f16(kFmtBF16, kFmtBF16, false, true, M, N);
}

// One branch for 32 values: a branch for each pair makes a chain of their latencies (16384 x 5120 x 1280 in 8 bits 191 us so).
__device__ __forceinline__ void activate32(uint32_t (&r)[32], int act) {
  if (act == kActGelu) {
#pragma unroll
    for (int e = 0; e < 32; e += 2) gelu2(r[e], r[e + 1]);
  } else if (act == kActSilu) {
#pragma unroll
    for (int e = 0; e < 32; e += 2) by_sigmoid2<kActSilu>(r[e], r[e + 1]);
  } else if (act == kActGeluTanh) {
#pragma unroll
    for (int e = 0; e < 32; e += 2) by_sigmoid2<kActGeluTanh>(r[e], r[e + 1]);
  }
}
// ------------------------------------------------------------------------------------------------
// Persistent form: one CTA per SM walks over tiles of 128 rows x kCols columns.  The ring runs on across tiles, and two
// accumulators in tensor memory alternate, so that a tile's epilogue (eight warps: a GELU per element is as long as the
// tile's MMAs at K = 640) runs under the next tile's loads and MMAs.  Against one tile per CTA, four epilogue warps and
// nothing overlapped: 4096 x 2560 x 640 with GELU 34 -> 22 us, without 20.3 -> 15.9 us, 4096 x 640 x 2560
// 20.5 -> 16.1 us, 8192 x 4096 x 1024 64 -> 53.9 us, 6144 x 640 x 640 8.1 -> 7.8 us (rows x columns x contraction).
// ------------------------------------------------------------------------------------------------
constexpr int kMaxStages = 6;
constexpr int kEpiWarps = 8;
template <int kCols, int kKind> constexpr int kOutWarps = kKind == kPlain ? kEpiWarps : kCols / 64 * 4;  // kPlus: one for each slab

struct PersistBars {
  uint64_t full[kMaxStages], empty[kMaxStages];
  uint64_t acc_full[2], acc_empty[2];
  uint64_t res[20];  // kPlus: the residual's slab of an epilogue warp is there
  uint32_t tmem_base;
  int abort_flag;
};
static_assert(sizeof(PersistBars) <= 512, "barrier block outgrew its reservation");

template <int kCols, int kKind>
struct PersistCfg {
  static constexpr int kStageBytes = kABytes + kCols / 64 * kSlab;
  static constexpr int kStages = kCols == 128 ? 6 : 4;
  static constexpr int kStaging = kOutWarps<kCols, kKind> * 32 * 128;  // per epilogue warp: 32 rows of a 64-column slab
  static constexpr int kSmemBytes = 1024 + kStages * kStageBytes + kStaging + 512;
  static constexpr uint32_t kAccCols = kCols == 128 ? 128 : 256;
};

// A warp's 32 rows of a tile, every second 64-column slab from `half` on: out of tensor memory, through the activation, staged
// in `mine` (32 rows of 128 B) and stored.
__device__ __forceinline__ void tile_out(uint32_t taddr, uint8_t* mine, int lane, const CUtensorMap* tm_c, int half, int slabs, int n0, int m0, int M,
                                         int act) {
#pragma unroll 1
  for (int j = half; j < slabs; j += 2) {
    if (lane == 0) tma_store_wait_read();  // the slab staged before has been read
    __syncwarp();
#pragma unroll 1
    for (int c = 0; c < 64; c += 32) {
      uint32_t r[32];
      tmem_ld32(taddr + j * 64 + c, r);
      tmem_wait_ld();
      if (act == kActGelu) {
#pragma unroll
        for (int e = 0; e < 32; e += 2) gelu2(r[e], r[e + 1]);
      }
#pragma unroll
      for (int e = 0; e < 32; e += 8) {
        __align__(16) __nv_bfloat162 q[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) q[u] = __floats2bfloat162_rn(__uint_as_float(r[e + 2 * u]), __uint_as_float(r[e + 2 * u + 1]));
        *reinterpret_cast<uint4*>(mine + sw128_offset(lane, (c + e) >> 3)) = *reinterpret_cast<const uint4*>(q);
      }
    }
    fence_proxy_async();  // the staged rows are read by the TMA engine
    __syncwarp();
    if (lane == 0 && m0 < M) {  // rows past M and columns past N inside a box are clipped by the store
      tma_store_2d(tm_c, mine, n0 + j * 64, m0);
      tma_store_commit();
    }
  }
}

// The same with bias and residual, and with the scales of 8-bit operands, a warp for each 64-column slab of a quarter: an activation
// takes two MUFU operations and some ten instructions per value, and eight warps for 256 columns (two a scheduler) are left at
// their latencies.  The slab of the residual comes into `mine` before the sums are waited for, in the place that the results then
// take, so nothing of it is left to wait for.  (Packets of 32 bytes straight from and to global memory, a row a thread, were as fast
// without a residual and 5 to 15 % slower with one.)  Bias and scales of the columns are the same for the lanes of a warp, a row
// each: 16-byte reads out of L1 for all of them.
template <int kKind>
struct SlabOut {
  uint8_t* mine;
  uint64_t* res;  // this warp's residual barrier
  const CUtensorMap *tm_c, *tm_r;
  LinearPlus p;
  int M, N, act, lane;
  uint32_t uses;  // slabs of the residual waited for
  bool pending;   // one more is on its way

  // The slab at column n of 32 rows from m0 on: its residual on the way into `mine`, its bias and scales into L1.
  __device__ __forceinline__ void fetch(int n, int m0) {
    if (lane == 0) tma_store_wait_read();  // the slab staged before has been read
    if (p.residual && m0 < M) {
      pending = true;
      if (lane == 0) {
        mbar_expect_tx(res, 4096);  // what lies past M or N comes as zeros and counts
        tma_load_2d(mine, tm_r, res, n, m0);
      }
    }
    const int c = n + 2 * lane;
    uint32_t x;
    if (c < N && p.bias) asm volatile("ld.global.b32 %0, [%1];" : "=r"(x) : "l"(p.bias + c));
    if (kKind == kPlus8 && c < N) asm volatile("ld.global.b32 %0, [%1];" : "=r"(x) : "l"(p.w_scale + c));
  }
  // 32 columns of the slab from c on, n in the matrix.
  __device__ __forceinline__ void chunk(uint32_t (&r)[32], float row_scale, int n, int c) {
    if constexpr (kKind == kPlus8) {
      float4 s[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) s[e] = n + 4 * e < N ? *reinterpret_cast<const float4*>(p.w_scale + n + 4 * e) : make_float4(0.f, 0.f, 0.f, 0.f);
      tmem_wait_ld(r);
      const uint64_t rs = both(row_scale);
#pragma unroll
      for (int e = 0; e < 32; e += 2) {  // (the row's first: two scales multiplied may leave fp32 where the result does not)
        const uint64_t f = e % 4 == 0 ? pack2(s[e / 4].x, s[e / 4].y) : pack2(s[e / 4].z, s[e / 4].w);
        float v0, v1;
        unpack2(mul2(mul2(pack2(__uint_as_float(r[e]), __uint_as_float(r[e + 1])), rs), f), v0, v1);
        r[e] = __float_as_uint(v0);
        r[e + 1] = __float_as_uint(v1);
      }
    } else {
      tmem_wait_ld(r);
    }
    if (p.bias) {
#pragma unroll
      for (int e = 0; e < 4; ++e) add_packet(r + 8 * e, n + 8 * e < N ? *reinterpret_cast<const uint4*>(p.bias + n + 8 * e) : make_uint4(0, 0, 0, 0));
    }
    activate32(r, act);
    if (p.residual) {
#pragma unroll
      for (int e = 0; e < 4; ++e) add_packet(r + 8 * e, *reinterpret_cast<const uint4*>(mine + sw128_offset(lane, (c >> 3) + e)));
    }
#pragma unroll
    for (int e = 0; e < 32; e += 8) {
      __align__(16) __nv_bfloat162 q[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) q[u] = __floats2bfloat162_rn(__uint_as_float(r[e + 2 * u]), __uint_as_float(r[e + 2 * u + 1]));
      *reinterpret_cast<uint4*>(mine + sw128_offset(lane, (c + e) >> 3)) = *reinterpret_cast<const uint4*>(q);
    }
  }
  // The sums of the slab at taddr are there and its residual has been fetched.
  __device__ __forceinline__ bool out(uint32_t taddr, int n, int m0, uint32_t* dev_status, volatile int* abort_flag) {
    const float row_scale = kKind == kPlus8 && m0 + lane < M ? p.a_scale[m0 + lane] : 1.f;
    uint32_t r[32];
    tmem_ld32(taddr, r);
    if (pending) {
      if (!mbar_wait_warp(res, uses & 1, dev_status, abort_flag)) return false;
      pending = false;
      ++uses;
    }
    __syncwarp();
    chunk(r, row_scale, n, 0);
    tmem_ld32(taddr + 32, r);
    chunk(r, row_scale, n + 32, 32);
    fence_proxy_async();  // the staged rows are read by the TMA engine
    __syncwarp();
    if (lane == 0 && m0 < M) {
      tma_store_2d(tm_c, mine, n, m0);
      tma_store_commit();
    }
    return true;
  }
};

template <int kCols, int kKind>
__global__ void __launch_bounds__((2 + kOutWarps<kCols, kKind>) * 32, 1)
linear_persistent_kernel(const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_w0,
                         const __grid_constant__ CUtensorMap tm_w1, const __grid_constant__ CUtensorMap tm_w2,
                         const __grid_constant__ CUtensorMap tm_c0, const __grid_constant__ CUtensorMap tm_c1,
                         const __grid_constant__ CUtensorMap tm_c2, int M, int N, int K, int n_items, int act, uint32_t* dev_status,
                         const LinearPlus plus) {
  using C = PersistCfg<kCols, kKind>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* staging = smem + C::kStages * C::kStageBytes;
  PersistBars* bar = reinterpret_cast<PersistBars*>(staging + C::kStaging);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int nk = (K + kStepK<kKind> - 1) / kStepK<kKind>;
  const int mb = (M + 127) / 128, nb = (N + kCols - 1) / kCols;
  // item -> row block (fastest: CTAs that run together share W slabs), column block, matrix
  auto m_of = [&](int item) { return item % mb * 128; };
  auto n_of = [&](int item) { return item / mb % nb * kCols; };
  auto z_of = [&](int item) { return item / mb / nb; };
  auto slabs_at = [&](int n0) { return (min(kCols, N - n0) + 63) / 64; };

  if (threadIdx.x == 0) {
    for (int s = 0; s < C::kStages; ++s) {
      mbar_init(&bar->full[s], 1);
      mbar_init(&bar->empty[s], 1);
    }
    for (int a = 0; a < 2; ++a) {
      mbar_init(&bar->acc_full[a], 1);
      mbar_init(&bar->acc_empty[a], kOutWarps<kCols, kKind>);
    }
    if constexpr (kKind != kPlain)
      for (int e = 0; e < kOutWarps<kCols, kKind>; ++e) mbar_init(&bar->res[e], 1);
    bar->abort_flag = 0;
    mbar_fence_init();
    prefetch_tmap(&tm_a);
    prefetch_tmap(&tm_w0);
    prefetch_tmap(&tm_c0);
  }
  dependency_wait();
  if (threadIdx.x == 0) release_dependents();
  if (warp == 1) tmem_alloc(&bar->tmem_base, 2 * C::kAccCols);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = bar->tmem_base;
  volatile int* abort_flag = &bar->abort_flag;

  if (warp == 0) {
    if (elect_one()) {
      int kc = 0;  // k-steps so far, over all items: ring slot and phase follow it
      bool ok = true;
      for (int item = blockIdx.x; ok && item < n_items; item += gridDim.x) {
        const int m0 = m_of(item), n0 = n_of(item), z = z_of(item), slabs = slabs_at(n0);
        const CUtensorMap* tm_w = z == 0 ? &tm_w0 : z == 1 ? &tm_w1 : &tm_w2;
        for (int k = 0; k < nk; ++k, ++kc) {
          const int s = kc % C::kStages;
          if (kc >= C::kStages && !mbar_wait(&bar->empty[s], ((kc / C::kStages) - 1) & 1, dev_status, abort_flag)) { ok = false; break; }
          uint8_t* sa = smem + s * C::kStageBytes;
          mbar_expect_tx(&bar->full[s], kABytes + slabs * kSlab);
          tma_load_2d(sa, &tm_a, &bar->full[s], k * kStepK<kKind>, m0);
          for (int j = 0; j < slabs; ++j) load_w<kKind>(sa + kABytes + j * kSlab, tm_w, &bar->full[s], n0 + j * 64, k * kStepK<kKind>);
        }
      }
    }
  } else if (warp == 1) {
    if (elect_one()) {
      int kc = 0, n = 0;
      bool ok = true;
      for (int item = blockIdx.x; item < n_items; item += gridDim.x, ++n) {
        const int a = n & 1;
        if (n >= 2 && !mbar_wait(&bar->acc_empty[a], ((n >> 1) - 1) & 1, dev_status, abort_flag)) break;
        tc_fence_after();
        const uint32_t t_acc = tmem + a * C::kAccCols;
        const uint32_t idesc = idesc_of<kKind>(128, slabs_at(n_of(item)) * 64);
        for (int k = 0; k < nk; ++k, ++kc) {
          const int s = kc % C::kStages;
          if (!mbar_wait(&bar->full[s], (kc / C::kStages) & 1, dev_status, abort_flag)) { ok = false; break; }
          tc_fence_after();
          const uint32_t aa = smem_u32(smem + s * C::kStageBytes), wa = aa + kABytes;
          // (32 bytes of contraction elements per MMA, zero filled past K)
          const int ksteps = min(kStepK<kKind>, K - k * kStepK<kKind> + kMmaK<kKind> - 1) / kMmaK<kKind>;
          for (int kk = 0; kk < ksteps; ++kk)
            mma_ss<kKind == kPlus8>(t_acc, smem_desc_sw128(aa + kk * 32, 16, 1024), w_desc<kKind>(wa, kk), idesc, k > 0 || kk > 0);
          mma_commit(&bar->empty[s]);
        }
        if (!ok) break;
        mma_commit(&bar->acc_full[a]);
      }
    }
  } else {
    // two warps per quarter of the rows, each with every second 64-column slab (kPlain), or one for each slab
    const int quarter = warp & 3, half = (warp - 2) >> 2;
    uint8_t* mine = staging + (warp - 2) * 4096;
    SlabOut<kKind> plus_out{mine, &bar->res[warp - 2], &tm_c0, &tm_w1, plus, M, N, act, lane, 0, false};
    int n = 0;
    for (int item = blockIdx.x; item < n_items; item += gridDim.x, ++n) {
      const int a = n & 1, m0 = m_of(item) + quarter * 32, n0 = n_of(item), z = z_of(item), slabs = slabs_at(n0);
      const CUtensorMap* tm_c = z == 0 ? &tm_c0 : z == 1 ? &tm_c1 : &tm_c2;
      if constexpr (kKind != kPlain) {
        if (half < slabs) plus_out.fetch(n0 + half * 64, m0);
      }
      // one answer per warp: the tensor-memory loads below are warp-wide operations
      if (!__all_sync(0xffffffffu, mbar_wait(&bar->acc_full[a], (n >> 1) & 1, dev_status, abort_flag))) break;
      tc_fence_after();
      const uint32_t taddr = tmem + a * C::kAccCols + ((uint32_t)(quarter * 32) << 16);
      if constexpr (kKind == kPlain) tile_out(taddr, mine, lane, tm_c, half, slabs, n0, m0, M, act);
      else if (half < slabs && !plus_out.out(taddr + half * 64, n0 + half * 64, m0, dev_status, abort_flag)) break;
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&bar->acc_empty[a]);
    }
    if constexpr (kKind != kPlain) {  // (after a wait that ran out: what was fetched still lands)
      if (plus_out.pending) mbar_wait_warp(plus_out.res, plus_out.uses & 1, dev_status, abort_flag);
    }
    if (lane == 0) tma_store_wait_read();  // shared memory must outlive the engine's reads
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, 2 * C::kAccCols);
  }
}

// ------------------------------------------------------------------------------------------------
// The same by pairs of SMs: a cluster of two CTAs walks over tiles of 256 rows x 256 columns.  Each CTA loads and keeps 128 of
// the rows of A and 128 of the columns of W, the first one's thread issues the MMAs of both (cta_group::2).  An SM then takes
// in 32 KB and reads 32 KB out of shared memory per 128 x 256 x 64 multiply-adds (512 cycles) where one working alone takes in
// and reads 48 KB each, which is more than the 128 bytes a cycle that shared memory has.  4096 x 2560 x 640 16.5 -> 15.0 us,
// 8192 x 1280 x 1280 25.6 -> 23.9, 16384 x 8192 x 4096 1092 -> 925 (rows x columns x contraction; against 256 x 256 by one CTA
// for the last).  A k-step still takes about 650 cycles: six stages do not quite cover the way from a free slot to its loads.
// Both CTAs' loads count on the first one's barrier; MMA completion is committed to both.
// ------------------------------------------------------------------------------------------------
constexpr int kPairRows = 256, kPairCols = 256;
// Row blocks that are walked over together.  The 74 tiles under way then need 12 row blocks of A and six or seven column blocks
// of W at a time, which they read in step; with all rows of A first (61 blocks and one) every k-step came out of DRAM where A is
// larger than L2.  Panels of 4 to 16 timed on 23 shapes: 12 takes 0.95 to 1.0 of the time of all rows first (1.01 once), 8 and 16 up
// to 1 and 2 % more than 12.  Twelve at most, all panels of a matrix alike: a last one of a few rows shares nothing (6585 x 8448 x 2112 and
// others of 13 to 37 row blocks 3 % slower with panels of twelve and a rest).
constexpr int kPanel = 12;
// With bias and residual there is a form of 256 x 320 besides, whose tiles divide the widths of these models' layers (multiples of
// 320) and read 36 KB per SM for 1.25 times the multiply-adds of 32.  Its 64 columns behind the 256 are an
// MMA of their own (32 in each CTA, half a slab: 64-byte rows in bf16, 32 rows in e4m3), and it has one accumulator, whose
// epilogue nothing overlaps but the loads of the next tile's first stages.
template <int kCols, int kKind>
struct PairCfg {
  static constexpr int kSlabs = kCols / 128;                        // of W in a CTA
  static constexpr bool kMore = kCols == 320;                       // ... and half a slab
  static constexpr int kStageBytes = kABytes + kSlabs * kSlab + (kMore ? kSlab / 2 : 0);  // a CTA's half
  static constexpr int kStages = kKind == kPlain ? 6 : kMore ? 4 : 5;
  static constexpr int kAccs = kMore ? 1 : 2;                       // accumulators in tensor memory
  static constexpr int kStaging = kOutWarps<kCols, kKind> * 32 * 128;
  static constexpr int kSmemBytes = 1024 + kStages * kStageBytes + kStaging + 512;
};
struct PairBars {
  uint64_t full[6], empty[6];  // (full: of the first CTA)
  uint64_t acc_full[2], acc_empty[2];
  uint64_t res[20];  // kPlus: the residual's slab of an epilogue warp is there
  uint32_t tmem_base;
  int abort_flag;
};
static_assert(sizeof(PairBars) <= 512, "barrier block outgrew its reservation");

template <int kKind, int kCols>
__global__ void __launch_bounds__((2 + kOutWarps<kCols, kKind>) * 32, 1)
linear_pair_kernel(const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_w0,
                   const __grid_constant__ CUtensorMap tm_w1, const __grid_constant__ CUtensorMap tm_w2,
                   const __grid_constant__ CUtensorMap tm_c0, const __grid_constant__ CUtensorMap tm_c1,
                   const __grid_constant__ CUtensorMap tm_c2, int M, int N, int K, int n_items, int act, uint32_t* dev_status,
                   const LinearPlus plus) {
  using C = PairCfg<kCols, kKind>;
  constexpr int kStages = C::kStages;
  extern __shared__ uint8_t smem_raw[];
  // (the same offset in both CTAs: they are launched alike)
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* staging = smem + kStages * C::kStageBytes;
  PairBars* bar = reinterpret_cast<PairBars*>(staging + C::kStaging);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_rank();
  const int nk = (K + kStepK<kKind> - 1) / kStepK<kKind>;
  const int mb = (M + kPairRows - 1) / kPairRows, nb = (N + kCols - 1) / kCols;
  const int pair = blockIdx.x / 2, pairs = gridDim.x / 2;
  const int panels = (mb + kPanel - 1) / kPanel, panel = (mb + panels - 1) / panels;  // row blocks of a panel, alike but for the last
  // item -> matrix, panel, column block, row block (fastest)
  auto place = [&](int item, int& m0, int& n0, int& z) {
    z = item / (mb * nb);
    const int in_z = item - z * mb * nb, first = in_z / (panel * nb) * panel, in_panel = in_z - first * nb, rows = min(panel, mb - first);
    n0 = in_panel / rows * kCols;
    m0 = (first + in_panel % rows) * kPairRows;
  };

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&bar->full[s], 1);
      mbar_init(&bar->empty[s], 1);
    }
    for (int a = 0; a < 2; ++a) {
      mbar_init(&bar->acc_full[a], 1);
      mbar_init(&bar->acc_empty[a], 2 * kOutWarps<kCols, kKind>);
    }
    if constexpr (kKind != kPlain)
      for (int e = 0; e < kOutWarps<kCols, kKind>; ++e) mbar_init(&bar->res[e], 1);
    bar->abort_flag = 0;
    mbar_fence_init();
    prefetch_tmap(&tm_a);
    prefetch_tmap(&tm_w0);
    prefetch_tmap(&tm_c0);
  }
  cluster_sync();  // both CTAs' barriers are there
  dependency_wait();
  if (threadIdx.x == 0) release_dependents();
  if (warp == 1) tmem_alloc_pair(&bar->tmem_base, 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = bar->tmem_base;
  volatile int* abort_flag = &bar->abort_flag;

  if (warp == 0) {
    if (elect_one()) {
      int kc = 0;  // k-steps so far, over all items: ring slot and phase follow it
      bool ok = true;
      for (int item = pair; ok && item < n_items; item += pairs) {
        int m0, n0, z;
        place(item, m0, n0, z);
        const int more = n0 + 256 + rank * 32;
        m0 += rank * 128, n0 += rank * (C::kMore ? 128 : kCols / 2);  // this CTA's rows and columns
        const CUtensorMap* tm_w = z == 0 ? &tm_w0 : z == 1 ? &tm_w1 : &tm_w2;
        for (int k = 0; k < nk; ++k, ++kc) {
          const int s = kc % kStages;
          if (kc >= kStages && !mbar_wait(&bar->empty[s], ((kc / kStages) - 1) & 1, dev_status, abort_flag)) { ok = false; break; }
          uint8_t* sa = smem + s * C::kStageBytes;
          if (rank == 0) mbar_expect_tx(&bar->full[s], 2 * C::kStageBytes);  // what lies past M or N comes as zeros and counts
          tma_load_2d_pair(sa, &tm_a, &bar->full[s], k * kStepK<kKind>, m0);
          for (int j = 0; j < C::kSlabs; ++j) {
            if constexpr (kKind == kPlus8) tma_load_2d_pair(sa + kABytes + j * kSlab, tm_w, &bar->full[s], k * kStepK<kKind>, n0 + j * 64);
            else tma_load_2d_pair(sa + kABytes + j * kSlab, tm_w, &bar->full[s], n0 + j * 64, k * kKC);
          }
          if constexpr (C::kMore) {
            if constexpr (kKind == kPlus8) tma_load_2d_pair(sa + kABytes + C::kSlabs * kSlab, &tm_w2, &bar->full[s], k * kStepK<kKind>, more);
            else tma_load_2d_pair(sa + kABytes + C::kSlabs * kSlab, &tm_w2, &bar->full[s], more, k * kKC);
          }
        }
      }
    }
  } else if (warp == 1) {
    if (rank == 0) {
      if (elect_one()) {
        constexpr uint32_t idesc = idesc_of<kKind>(kPairRows, C::kMore ? 256 : kCols), idesc_more = idesc_of<kKind>(kPairRows, 64);
        int kc = 0, n = 0;
        bool ok = true;
        for (int item = pair; ok && item < n_items; item += pairs, ++n) {
          const int a = n % C::kAccs;
          if (n >= C::kAccs && !mbar_wait(&bar->acc_empty[a], (n / C::kAccs - 1) & 1, dev_status, abort_flag)) break;
          tc_fence_after();
          for (int k = 0; k < nk; ++k, ++kc) {
            const int s = kc % kStages;
            if (!mbar_wait(&bar->full[s], (kc / kStages) & 1, dev_status, abort_flag)) { ok = false; break; }
            tc_fence_after();
            const uint32_t aa = smem_u32(smem + s * C::kStageBytes), wa = aa + kABytes;
            // (32 bytes of contraction elements per MMA, zero filled past K)
            const int ksteps = min(kStepK<kKind>, K - k * kStepK<kKind> + kMmaK<kKind> - 1) / kMmaK<kKind>;
            for (int kk = 0; kk < ksteps; ++kk) {
              mma_ss_pair<kKind == kPlus8>(tmem + a * 256, smem_desc_sw128(aa + kk * 32, 16, 1024), w_desc<kKind>(wa, kk), idesc, k > 0 || kk > 0);
              if constexpr (C::kMore)
                mma_ss_pair<kKind == kPlus8>(tmem + 256, smem_desc_sw128(aa + kk * 32, 16, 1024), half_desc<kKind>(wa + C::kSlabs * kSlab, kk), idesc_more,
                                             k > 0 || kk > 0);
            }
            mma_commit_pair(&bar->empty[s]);
          }
          if (ok) mma_commit_pair(&bar->acc_full[a]);
        }
      }
    }
  } else {
    // two warps per quarter of the CTA's rows, each with every second 64-column slab
    const int quarter = warp & 3, half = (warp - 2) >> 2;
    uint8_t* mine = staging + (warp - 2) * 4096;
    SlabOut<kKind> plus_out{mine, &bar->res[warp - 2], &tm_c0, &tm_w1, plus, M, N, act, lane, 0, false};
    int n = 0;
    for (int item = pair; item < n_items; item += pairs, ++n) {
      int m0, n0, z;
      place(item, m0, n0, z);
      m0 += rank * 128 + quarter * 32;
      const int a = n % C::kAccs, slabs = (min(kCols, N - n0) + 63) / 64;
      const CUtensorMap* tm_c = z == 0 ? &tm_c0 : z == 1 ? &tm_c1 : &tm_c2;
      if constexpr (kKind != kPlain) {
        if (half < slabs) plus_out.fetch(n0 + half * 64, m0);
      }
      // one answer per warp: the tensor-memory loads below are warp-wide operations
      if (!__all_sync(0xffffffffu, mbar_wait(&bar->acc_full[a], (n / C::kAccs) & 1, dev_status, abort_flag))) break;
      tc_fence_after();
      const uint32_t taddr = tmem + a * 256 + ((uint32_t)(quarter * 32) << 16);
      if constexpr (kKind == kPlain) tile_out(taddr, mine, lane, tm_c, half, slabs, n0, m0, M, act);
      else if (half < slabs && !plus_out.out(taddr + half * 64, n0 + half * 64, m0, dev_status, abort_flag)) break;
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_at(peer_addr(smem_u32(&bar->acc_empty[a]), 0));  // of the issuing CTA, which may be this one
    }
    if constexpr (kKind != kPlain) {  // (after a wait that ran out: what was fetched still lands)
      if (plus_out.pending) mbar_wait_warp(plus_out.res, plus_out.uses & 1, dev_status, abort_flag);
    }
    if (lane == 0) tma_store_wait_read();  // shared memory must outlive the engine's reads
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc_pair(tmem, 512);
  }
  cluster_sync();  // neither leaves while the other's MMAs read its shared memory or its arrivals are under way
}

template <int kCols, int kKind>
cudaError_t run_persistent(int M, int N, int K, int n_mats, const CUtensorMap& ta, const CUtensorMap (&tw)[3], const CUtensorMap (&tc)[3], int act,
                           const LinearPlus& plus, uint32_t* dev_status, cudaStream_t s) {
  using C = PersistCfg<kCols, kKind>;
  static std::atomic<unsigned long long> raised{0};
  if (cudaError_t e = raise_dynamic_smem(linear_persistent_kernel<kCols, kKind>, C::kSmemBytes, raised); e != cudaSuccess) return e;
  const long long items = (long long)((M + 127) / 128) * ((N + kCols - 1) / kCols) * n_mats;
  if (items > INT32_MAX / 2) return cudaErrorInvalidValue;
  const int grid = items < sm_count() ? (int)items : sm_count();
  return launch_dependent(linear_persistent_kernel<kCols, kKind>, dim3(grid), dim3((2 + kOutWarps<kCols, kKind>) * 32), (size_t)C::kSmemBytes, s, ta, tw[0], tw[1],
                          tw[2], tc[0], tc[1], tc[2], M, N, K, (int)items, act, dev_status, plus);
}

// How many pairs the device holds at once: 0 where it places no cluster of this size (the other forms need none).
int pairs_at_once() {
  static ClusterState st;
  return clusters_at_once(linear_pair_kernel<kPlain, kPairCols>, st, 2, (2 + kEpiWarps) * 32, PairCfg<kPairCols, kPlain>::kSmemBytes);
}

template <int kCols, int kKind>
cudaError_t run_pair(int at_once, int M, int N, int K, int n_mats, const CUtensorMap& ta, const CUtensorMap (&tw)[3], const CUtensorMap (&tc)[3],
                     int act, const LinearPlus& plus, uint32_t* dev_status, cudaStream_t s) {
  using C = PairCfg<kCols, kKind>;
  static std::atomic<unsigned long long> raised{0};
  if (cudaError_t e = raise_dynamic_smem(linear_pair_kernel<kKind, kCols>, C::kSmemBytes, raised); e != cudaSuccess) return e;
  const long long items = (long long)((M + kPairRows - 1) / kPairRows) * ((N + kCols - 1) / kCols) * n_mats;
  if (items > INT32_MAX / 2) return cudaErrorInvalidValue;
  const int pairs = items < at_once ? (int)items : at_once;
  return launch_dependent_cluster(linear_pair_kernel<kKind, kCols>, dim3(2 * pairs), dim3((2 + kOutWarps<kCols, kKind>) * 32), (size_t)C::kSmemBytes, 2, s, ta, tw[0],
                                  tw[1], tw[2], tc[0], tc[1], tc[2], M, N, K, (int)items, act, dev_status, plus);
}

// One launch in the given tile form.
template <int kKind>
cudaError_t run_form(int form, int at_once, int M, int N, int K, int n_mats, const CUtensorMap& ta, const CUtensorMap (&tw)[3],
                     const CUtensorMap (&tc)[3], int act, const LinearPlus& plus, uint32_t* dev_status, cudaStream_t s) {
  cudaError_t e = cudaErrorInvalidValue;
  if (form == 4) e = run_persistent<128, kKind>(M, N, K, n_mats, ta, tw, tc, act, plus, dev_status, s);
  else if (form == 3) e = run_pair<kPairCols, kKind>(at_once, M, N, K, n_mats, ta, tw, tc, act, plus, dev_status, s);
  else if (form == 2) e = run_persistent<192, kKind>(M, N, K, n_mats, ta, tw, tc, act, plus, dev_status, s);
  if constexpr (kKind == kPlain)
    if (form == 1) e = run_persistent<256, kKind>(M, N, K, n_mats, ta, tw, tc, act, plus, dev_status, s);
  if constexpr (kKind != kPlain)
    if (form == 5) e = run_pair<320, kKind>(at_once, M, N, K, n_mats, ta, tw, tc, act, plus, dev_status, s);
  count_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

// The tile form of a launch: linear_tc_form()'s, or the test's.
int form_of(int M, int N, int K, int n_mats, int at_once) {
  const int v = g_tune_linear_tile.load(std::memory_order_relaxed);  // test-only override
  if (v && v <= 4 && (v != 3 || (M > 128 && at_once > 0))) return v;
  return linear_tc_form(M, N, K, n_mats, sm_count(), at_once);
}

// ------------------------------------------------------------------------------------------------
// Few tiles (few rows): a cluster of 2, 4 or 8 CTAs splits the contraction of one tile of 128 x 128.  Each sums up its steps in its
// tensor memory, sends every other CTA the partial sums of the columns that one finishes (a part of 128 / S columns each, through
// distributed shared memory, fp32), and finishes its own: the parts of all CTAs added up in the order of their ranks, then the
// epilogue, a row a thread.  No scratch, no atomics, one launch; what is added up in which order is fixed by the shape.
// ------------------------------------------------------------------------------------------------
constexpr int kSplitStages = 4, kSplitStageBytes = kABytes + 2 * kSlab;
constexpr int kSplitSmem = 1024 + kSplitStages * kSplitStageBytes + 128 * 128 * 4 + 256;
struct SplitBars {
  uint64_t full[kSplitStages], empty[kSplitStages], acc_full;
  uint32_t tmem_base;
  int abort_flag;
};
static_assert(sizeof(SplitBars) <= 256, "barrier block outgrew its reservation");
template <int kKind, int S>
__global__ void __launch_bounds__((2 + kEpiWarps) * 32, 1)
linear_split_kernel(const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_w, int M, int N, int K, int act,
                    uint32_t* dev_status, const LinearPlus plus) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* parts = smem + kSplitStages * kSplitStageBytes;  // [other rank][column / 4][row] packets of four columns
  SplitBars* bar = reinterpret_cast<SplitBars*>(parts + 128 * 128 * 4);
  constexpr int kPart = 128 / S;  // columns that a CTA finishes
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = (int)cluster_rank(), tile = blockIdx.x / S;
  const int nk = (K + kStepK<kKind> - 1) / kStepK<kKind>, k_first = rank * nk / S, k_last = (rank + 1) * nk / S;  // (nk >= S: no CTA without a step)
  const int mb = (M + 127) / 128, m0 = tile % mb * 128, n0 = tile / mb * 128, slabs = (min(128, N - n0) + 63) / 64;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kSplitStages; ++s) {
      mbar_init(&bar->full[s], 1);
      mbar_init(&bar->empty[s], 1);
    }
    mbar_init(&bar->acc_full, 1);
    bar->abort_flag = 0;
    mbar_fence_init();
    prefetch_tmap(&tm_a);
    prefetch_tmap(&tm_w);
  }
  dependency_wait();
  if (threadIdx.x == 0) release_dependents();
  if (warp == 1) tmem_alloc(&bar->tmem_base, 128);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = bar->tmem_base;
  volatile int* abort_flag = &bar->abort_flag;
  cluster_arrive();  // this CTA's shared memory is there: peers wait for it before they write into it

  const int quarter = warp & 3, half = (warp - 2) >> 2, row = quarter * 32 + lane, m = m0 + row;
  const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16);
  constexpr int kUnits = kPart / 16;  // eights of columns that a warp finishes: the part's first or second half
  const int c0 = rank * kPart + half * (kPart / 2);
  uint4 res[kUnits];
  bool ok = true;
  if (warp == 0) {
    if (elect_one()) {
      for (int k = k_first, i = 0; k < k_last; ++k, ++i) {
        const int s = i % kSplitStages;
        if (i >= kSplitStages && !mbar_wait(&bar->empty[s], ((i / kSplitStages) - 1) & 1, dev_status, abort_flag)) break;
        uint8_t* sa = smem + s * kSplitStageBytes;
        mbar_expect_tx(&bar->full[s], kABytes + slabs * kSlab);
        tma_load_2d(sa, &tm_a, &bar->full[s], k * kStepK<kKind>, m0);
        for (int j = 0; j < slabs; ++j) load_w<kKind>(sa + kABytes + j * kSlab, &tm_w, &bar->full[s], n0 + j * 64, k * kStepK<kKind>);
      }
    }
  } else if (warp == 1) {
    if (elect_one()) {
      const uint32_t idesc = idesc_of<kKind>(128, slabs * 64);
      bool all = true;
      for (int k = k_first, i = 0; k < k_last; ++k, ++i) {
        const int s = i % kSplitStages;
        if (!mbar_wait(&bar->full[s], (i / kSplitStages) & 1, dev_status, abort_flag)) { all = false; break; }
        tc_fence_after();
        const uint32_t aa = smem_u32(smem + s * kSplitStageBytes), wa = aa + kABytes;
        const int ksteps = min(kStepK<kKind>, K - k * kStepK<kKind> + kMmaK<kKind> - 1) / kMmaK<kKind>;
        for (int kk = 0; kk < ksteps; ++kk)
          mma_ss<kKind == kPlus8>(tmem, smem_desc_sw128(aa + kk * 32, 16, 1024), w_desc<kKind>(wa, kk), idesc, k > k_first || kk > 0);
        mma_commit(&bar->empty[s]);
      }
      if (all) mma_commit(&bar->acc_full);
    }
  } else {
    // what the epilogue reads besides the sums, on its way while they are waited for
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      const int n = n0 + c0 + u * 8;
      res[u] = plus.residual && m < M && n < N ? *reinterpret_cast<const uint4*>(plus.residual + (size_t)m * plus.ldr + n) : make_uint4(0, 0, 0, 0);
      if (lane < 8 && n < N) {
        uint32_t x;
        if (plus.bias) asm volatile("ld.global.b32 %0, [%1];" : "=r"(x) : "l"(plus.bias + n));
        if (kKind == kPlus8) asm volatile("ld.global.b32 %0, [%1];" : "=r"(x) : "l"(plus.w_scale + n + lane));
      }
    }
    ok = mbar_wait_warp(&bar->acc_full, 0, dev_status, abort_flag);
  }
  cluster_wait();  // all peers have begun
  if (warp >= 2 && ok && m0 + quarter * 32 < M) {
    tc_fence_after();
    // sixteen columns at a time to whom finishes them, the two warps of a quarter in turns
#pragma unroll
    for (int g = 0; g < 8; ++g) {
      const int col = g * 16, to = col / kPart;
      if ((g & 1) != half || to == rank || n0 + col >= N) continue;
      uint32_t r[16];
      tmem_ld16(lanes + col, r);
      tmem_wait_ld();
      const int slot = rank < to ? rank : rank - 1;
      const uint32_t at = peer_addr(smem_u32(parts + ((size_t)(slot * (kPart / 4) + (col - to * kPart) / 4) * 128 + row) * 16), (uint32_t)to);
#pragma unroll
      for (int e = 0; e < 4; ++e) st_peer_v4(at + e * 2048, r + 4 * e);
    }
  }
  cluster_arrive();
  cluster_wait();  // the parts of all are there; nobody writes any more
  if (warp >= 2 && ok && m0 + quarter * 32 < M) {
    const float row_scale = kKind == kPlus8 && m < M ? plus.a_scale[m] : 1.f;
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      const int n = n0 + c0 + u * 8, in_part = half * (kPart / 2) + u * 8;
      if (n >= N) continue;
      uint32_t own[8];
      tmem_ld8(lanes + c0 + u * 8, own);
      tmem_wait_ld();
      float v[8] = {};
#pragma unroll
      for (int r = 0; r < S; ++r) {
        if (r == rank) {
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] += __uint_as_float(own[e]);
        } else {
          const uint8_t* at = parts + ((size_t)((r < rank ? r : r - 1) * (kPart / 4) + in_part / 4) * 128 + row) * 16;
          const float4 p0 = *reinterpret_cast<const float4*>(at), p1 = *reinterpret_cast<const float4*>(at + 2048);
          v[0] += p0.x, v[1] += p0.y, v[2] += p0.z, v[3] += p0.w, v[4] += p1.x, v[5] += p1.y, v[6] += p1.z, v[7] += p1.w;
        }
      }
      if (m < M) finish8<kKind>(v, row_scale, plus, act, res[u], n, plus.c + (size_t)m * plus.ldc + n);
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, 128);
  }
}

// ------------------------------------------------------------------------------------------------
// The same by pairs of SMs for more rows: a cluster of S pairs (S = 2, 3) splits the contraction of one tile of 256 x 256.  Eight
// parts of 32 columns are dealt out to the pairs to finish, part u to pair u S / 8; a CTA has 128 of the rows, as in its
// accumulator, so partial sums go between CTAs of the same half.  They have room of their own, since a peer may still multiply when
// this pair is through.
// ------------------------------------------------------------------------------------------------
template <int S>
struct PairSplitCfg {
  static constexpr int kStages = S == 2 ? 5 : 4;
  static constexpr int kStageBytes = kABytes + 2 * kSlab;
  static constexpr int kMost = S == 2 ? 4 : 3;          // parts that a pair finishes, at most
  static constexpr int kParts = (S - 1) * kMost * 32 * 128 * 4;
  static constexpr int kSmemBytes = 1024 + kStages * kStageBytes + kParts + 256;
  static constexpr int kWarps = 16;
};
struct PairSplitBars {
  uint64_t full[5], empty[5], acc_full;
  uint32_t tmem_base;
  int abort_flag;
};
static_assert(sizeof(PairSplitBars) <= 256, "barrier block outgrew its reservation");

template <int kKind, int S>
__global__ void __launch_bounds__((2 + PairSplitCfg<S>::kWarps) * 32, 1)
linear_pair_split_kernel(const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_w, int M, int N, int K, int act,
                         uint32_t* dev_status, const LinearPlus plus) {
  using C = PairSplitCfg<S>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* parts = smem + C::kStages * C::kStageBytes;  // [other pair][part][column / 4][row] packets of four columns
  PairSplitBars* bar = reinterpret_cast<PairSplitBars*>(parts + C::kParts);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = (int)cluster_rank(), pair = rank >> 1, side = rank & 1, leader = rank & ~1, tile = blockIdx.x / (2 * S);
  const int nk = (K + kStepK<kKind> - 1) / kStepK<kKind>, k_first = pair * nk / S, k_last = (pair + 1) * nk / S;  // (nk >= S)
  const int mb = (M + 255) / 256, m0 = tile % mb * 256 + side * 128, n0 = tile / mb * 256;

  if (threadIdx.x == 0) {
    for (int s = 0; s < C::kStages; ++s) {
      mbar_init(&bar->full[s], 1);
      mbar_init(&bar->empty[s], 1);
    }
    mbar_init(&bar->acc_full, 1);
    bar->abort_flag = 0;
    mbar_fence_init();
    prefetch_tmap(&tm_a);
    prefetch_tmap(&tm_w);
  }
  cluster_sync();  // all CTAs' barriers and shared memory are there
  dependency_wait();
  if (threadIdx.x == 0) release_dependents();
  if (warp == 1) tmem_alloc_pair(&bar->tmem_base, 256);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = bar->tmem_base;
  volatile int* abort_flag = &bar->abort_flag;
  const int quarter = warp & 3, group = (warp - 2) >> 2, row = quarter * 32 + lane, m = m0 + row;
  const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16);
  const bool out = warp >= 2 && m0 + quarter * 32 < M;
  bool ok = true;

  if (warp == 0) {
    if (elect_one()) {
      for (int k = k_first, i = 0; k < k_last; ++k, ++i) {
        const int s = i % C::kStages;
        if (i >= C::kStages && !mbar_wait(&bar->empty[s], ((i / C::kStages) - 1) & 1, dev_status, abort_flag)) break;
        uint8_t* sa = smem + s * C::kStageBytes;
        if (side == 0) mbar_expect_tx(&bar->full[s], 2 * C::kStageBytes);  // what lies past M or N comes as zeros and counts
        const uint32_t full = peer_addr(smem_u32(&bar->full[s]), (uint32_t)leader);
        tma_load_2d_pair_at(sa, &tm_a, full, k * kStepK<kKind>, m0);
        for (int j = 0; j < 2; ++j) {
          const int n = n0 + side * 128 + j * 64;
          if constexpr (kKind == kPlus8) tma_load_2d_pair_at(sa + kABytes + j * kSlab, &tm_w, full, k * kStepK<kKind>, n);
          else tma_load_2d_pair_at(sa + kABytes + j * kSlab, &tm_w, full, n, k * kKC);
        }
      }
    }
  } else if (warp == 1) {
    if (side == 0) {
      if (elect_one()) {
        constexpr uint32_t idesc = idesc_of<kKind>(256, 256);
        const uint16_t both_ctas = (uint16_t)(3u << leader);
        bool all = true;
        for (int k = k_first, i = 0; k < k_last; ++k, ++i) {
          const int s = i % C::kStages;
          if (!mbar_wait(&bar->full[s], (i / C::kStages) & 1, dev_status, abort_flag)) { all = false; break; }
          tc_fence_after();
          const uint32_t aa = smem_u32(smem + s * C::kStageBytes), wa = aa + kABytes;
          const int ksteps = min(kStepK<kKind>, K - k * kStepK<kKind> + kMmaK<kKind> - 1) / kMmaK<kKind>;
          for (int kk = 0; kk < ksteps; ++kk)
            mma_ss_pair<kKind == kPlus8>(tmem, smem_desc_sw128(aa + kk * 32, 16, 1024), w_desc<kKind>(wa, kk), idesc, k > k_first || kk > 0);
          mma_commit_pair_to(&bar->empty[s], both_ctas);
        }
        if (all) mma_commit_pair_to(&bar->acc_full, both_ctas);
      }
    }
  } else {
    if (out) {  // what the epilogue reads besides the sums, on its way into L1
      uint32_t x;
      const int n = n0 + group * 64 + lane * 2;
      if (n < N && plus.bias) asm volatile("ld.global.b32 %0, [%1];" : "=r"(x) : "l"(plus.bias + n));
      if (kKind == kPlus8 && n < N) asm volatile("ld.global.b32 %0, [%1];" : "=r"(x) : "l"(plus.w_scale + n));
    }
    ok = mbar_wait_warp(&bar->acc_full, 0, dev_status, abort_flag);
    if (ok && out) {
      tc_fence_after();
      // the parts of others to who finishes them, every fourth a warp's
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int u = group + 4 * h, to = u * S / 8, first = (to * 8 + S - 1) / S;  // part, its pair, that pair's first part
        if (to == pair || n0 + u * 32 >= N) continue;
        uint32_t r[32];
        tmem_ld32(lanes + u * 32, r);
        tmem_wait_ld();
        const int slot = pair < to ? pair : pair - 1;
        const uint32_t at = peer_addr(smem_u32(parts + ((size_t)((slot * C::kMost + u - first) * 8) * 128 + row) * 16), (uint32_t)(2 * to + side));
#pragma unroll
        for (int e = 0; e < 8; ++e) st_peer_v4(at + e * 2048, r + 4 * e);
      }
    }
  }
  cluster_arrive();
  const int first = (pair * 8 + S - 1) / S, count = ((pair + 1) * 8 + S - 1) / S - first;  // this pair's parts
  constexpr int kPieces = (2 * C::kMost + 3) / 4;  // of sixteen columns of them, every fourth a warp's
  uint4 res[kPieces][2];
#pragma unroll
  for (int i = 0; i < kPieces; ++i)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int piece = group + 4 * i, n = n0 + first * 32 + piece * 16 + h * 8;
      res[i][h] = out && plus.residual && piece < 2 * count && m < M && n < N ? *reinterpret_cast<const uint4*>(plus.residual + (size_t)m * plus.ldr + n) : make_uint4(0, 0, 0, 0);
    }
  cluster_wait();  // the parts of all are there; nobody writes any more
  if (ok && out) {
    const float row_scale = kKind == kPlus8 && m < M ? plus.a_scale[m] : 1.f;
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int piece = group + 4 * i, col = first * 32 + piece * 16;
      if (piece >= 2 * count || n0 + col >= N) continue;
      uint32_t own[16];
      tmem_ld16(lanes + col, own);
      tmem_wait_ld();
      float v[2][8] = {};
#pragma unroll
      for (int r = 0; r < S; ++r) {
        if (r == pair) {
#pragma unroll
          for (int e = 0; e < 16; ++e) v[e / 8][e % 8] += __uint_as_float(own[e]);
        } else {
          const uint8_t* at = parts + ((size_t)(((r < pair ? r : r - 1) * C::kMost + piece / 2) * 8 + piece % 2 * 4) * 128 + row) * 16;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float4 p = *reinterpret_cast<const float4*>(at + e * 2048);
            float* x = &v[e / 2][e % 2 * 4];
            x[0] += p.x, x[1] += p.y, x[2] += p.z, x[3] += p.w;
          }
        }
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int n = n0 + col + h * 8;
        if (m < M && n < N) finish8<kKind>(v[h], row_scale, plus, act, res[i][h], n, plus.c + (size_t)m * plus.ldc + n);
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc_pair(tmem, 256);
  }
  cluster_sync();  // neither of a pair leaves while the other's MMAs read its shared memory or its arrivals are under way
}

template <int kKind, int S>
int splits_at_once() {
  static ClusterState st;
  return clusters_at_once(linear_split_kernel<kKind, S>, st, S, (2 + kEpiWarps) * 32, kSplitSmem);
}
template <int kKind, int S>
int pair_splits_at_once() {
  static ClusterState st;
  return clusters_at_once(linear_pair_split_kernel<kKind, S>, st, 2 * S, (2 + PairSplitCfg<S>::kWarps) * 32, PairSplitCfg<S>::kSmemBytes);
}
template <int kKind, int S>
cudaError_t run_split(int M, int N, int K, const CUtensorMap& ta, const CUtensorMap& tw, int act, const LinearPlus& plus, uint32_t* dev_status,
                      cudaStream_t s) {
  const long long ctas = (long long)((M + 127) / 128) * ((N + 127) / 128) * S;
  if (ctas > INT32_MAX) return cudaErrorInvalidValue;
  const cudaError_t e = launch_dependent_cluster(linear_split_kernel<kKind, S>, dim3((unsigned)ctas), dim3((2 + kEpiWarps) * 32), (size_t)kSplitSmem, S, s,
                                                 ta, tw, M, N, K, act, dev_status, plus);
  count_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}
template <int kKind, int S>
cudaError_t run_pair_split(int M, int N, int K, const CUtensorMap& ta, const CUtensorMap& tw, int act, const LinearPlus& plus, uint32_t* dev_status,
                           cudaStream_t s) {
  using C = PairSplitCfg<S>;
  const long long ctas = (long long)((M + 255) / 256) * ((N + 255) / 256) * 2 * S;
  if (ctas > INT32_MAX) return cudaErrorInvalidValue;
  const cudaError_t e = launch_dependent_cluster(linear_pair_split_kernel<kKind, S>, dim3((unsigned)ctas), dim3((2 + C::kWarps) * 32),
                                                 (size_t)C::kSmemBytes, 2 * S, s, ta, tw, M, N, K, act, dev_status, plus);
  count_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

// Tile form: the one with the least serial work per SM, i.e. tiles per SM (rounded up) times the time of one, which was
// timed on seventeen shapes between 200 x 640 x 640 and 16384 x 8192 x 4096: a tile of 128 x 192 takes 1.2 times, one of
// 128 x 256 1.35 times as long as one of 128 x 128 (they read fewer operand bytes per multiply-add), a pair's of 256 x 256
// 1.25 times - 1.1 from about 2048 contraction elements on - and a fifth more per launch for the cluster's start and end.
// Returns 128 x 256 (1), 128 x 192 (2), 256 x 256 by pairs (3) or 128 x 128 (4).
int linear_tc_form(int M, int N, int K, int n_mats, int sms, int pairs) {
  auto cost = [&](int rows, int cols, int tile, int at_once) {
    const long long tiles = (long long)((M + rows - 1) / rows) * ((N + cols - 1) / cols) * n_mats;
    return (tiles + at_once - 1) / at_once * tile;
  };
  const long long cost128 = cost(128, 128, 20, sms), cost192 = cost(128, 192, 24, sms), cost256 = cost(128, 256, 27, sms);
  const long long cost_pair = M > 128 && pairs > 0 ? cost(kPairRows, kPairCols, K >= 2048 ? 22 : 25, pairs) + 4 : LLONG_MAX;
  if (cost_pair < cost128 && cost_pair < cost192 && cost_pair < cost256) return 3;
  return cost128 <= cost192 && cost128 <= cost256 ? 4 : cost192 <= cost256 ? 2 : 1;
}

bool linear_tc_shape_ok(int M, int N, int K) { return M >= 1 && N >= 8 && K >= 8 && N % 8 == 0 && K % 8 == 0; }

// c[i] = a * w[i] for i < n_mats (1..3); a [M][K], w[i] [K][N], c[i] [M][N], all bf16 row-major.
cudaError_t launch_linear_tc(int M, int N, int K, const void* a, const void* const* w, void* const* c, int n_mats, int act,
                             uint32_t* dev_status, cudaStream_t s) {
  CUtensorMap ta, tw[3], tc_[3];
  const uint64_t adims[2] = {(uint64_t)K, (uint64_t)M};
  const uint64_t astr[1] = {(uint64_t)K * 2};
  const uint32_t abox[2] = {64, 128};
  if (!encode_tmap_16bit(&ta, a, 2, adims, astr, abox)) return cudaErrorInvalidValue;
  const uint64_t wdims[2] = {(uint64_t)N, (uint64_t)K};
  const uint64_t wstr[1] = {(uint64_t)N * 2};
  const uint32_t wbox[2] = {64, 64};
  const uint64_t cdims[2] = {(uint64_t)N, (uint64_t)M};
  const uint32_t cbox[2] = {64, 32};  // a warp's 32 rows of one 64-column slab
  for (int i = 0; i < 3; ++i) {
    const int j = i < n_mats ? i : 0;
    if (!encode_tmap_16bit(&tw[i], w[j], 2, wdims, wstr, wbox) || !encode_tmap_16bit(&tc_[i], c[j], 2, cdims, wstr, cbox))
      return cudaErrorInvalidValue;
  }
  const int at_once = pairs_at_once();
  return run_form<kPlain>(form_of(M, N, K, n_mats, at_once), at_once, M, N, K, n_mats, ta, tw, tc_, act, LinearPlus{}, dev_status, s);
}

namespace {

// What a device holds at once: SMs, pairs, and clusters of 2, 4, 8 CTAs and of 2, 3 pairs that split a contraction.
struct PlusDevice {
  int sms, pairs, split[3], pair_split[2];
};
// The form of a launch: 128 x 128 (4), 128 x 192 (2), 256 x 256 (3) or 256 x 320 (5) by pairs, or, with the contraction split, 128 x 128 by 2,
// 4, 8 CTAs (6, 7, 8) or 256 x 256 by 2, 3 pairs (9, 10).  It is the one with the least time by this account: rounds of tiles over
// the SMs, each a fixed part and a part per step (64 contraction elements of bf16, 128 of e4m3), and what is left of a launch.
// Nanoseconds, fitted to 266 shapes between 20 x 320 x 1280 and 16384 x 5120 x 1280 in both types, each timed in every form: within 4
// to 6 % in the mean (10 to 14 % for the split forms), and the form it names takes 1.02 times as long as the best in the mean;
// linear_tc_form()'s choice took 1.15 times as long (3.4 at most: few tiles).  Timed too and never the best by more than 2 %: 128 x 256,
// 256 x 128 by pairs, 256 x 256 by 4 pairs; 256 x 512 by pairs, one accumulator, was slower everywhere (16384 x 5120 x 1280 in 8 bits 106 us
// against 91).
// The forms of 256 rows are for more than 128.  An activation is hidden under the next tile's steps but for the form that has one
// accumulator.
int plus_form(int M, int N, int steps, int act, const PlusDevice& d) {
  const auto tiles = [&](int rows, int cols) { return (long long)((M + rows - 1) / rows) * ((N + cols - 1) / cols); };
  int best = 4;
  long long least = LLONG_MAX;
  const auto offer = [&](int form, long long count, int at_once, int parts, int launch, int round, int step) {
    if (at_once < 1 || steps < parts) return;
    const long long cost = launch + (count + at_once - 1) / at_once * (round + (long long)((steps + parts - 1) / parts) * step);
    if (cost < least) least = cost, best = form;
  };
  offer(4, tiles(128, 128), d.sms, 1, 3840, 1020, 252);
  offer(2, tiles(128, 192), d.sms, 1, 3660, 1520, 265);
  for (int i = 0; i < 3; ++i) offer(6 + i, tiles(128, 128), d.split[i], 2 << i, 0, i == 1 ? 5400 : 5680, i == 0 ? 254 : 282);
  if (M > 128) {
    offer(3, tiles(kPairRows, kPairCols), d.pairs, 1, 5030, 1470, 293);
    offer(5, tiles(kPairRows, 320), d.pairs, 1, 3930, act == kActNone ? 3510 : 5000, 382);
    for (int i = 0; i < 2; ++i) offer(9 + i, tiles(kPairRows, kPairCols), d.pair_split[i], 2 + i, 0, 7700, i == 0 ? 298 : 327);
  }
  return best;
}

template <int kKind>
cudaError_t run_plus(const LinearPlusOp& o, int form, const PlusDevice& d, uint32_t* dev_status, cudaStream_t s) {
  constexpr bool f8 = kKind == kPlus8;
  constexpr auto encode = f8 ? encode_tmap_8bit : encode_tmap_16bit;
  CUtensorMap ta, tw;
  const uint64_t adims[2] = {(uint64_t)o.K, (uint64_t)o.M}, astr[1] = {(uint64_t)o.lda * (f8 ? 1 : 2)};
  const uint32_t abox[2] = {f8 ? 128u : 64u, 128};
  const uint64_t wdims[2] = {(uint64_t)(f8 ? o.K : o.N), (uint64_t)(f8 ? o.N : o.K)}, wstr[1] = {(uint64_t)o.ldw * (f8 ? 1 : 2)};
  const uint32_t wbox[2] = {f8 ? 128u : 64u, 64};
  if (!encode(&ta, o.a, 2, adims, astr, abox) || !encode(&tw, o.w, 2, wdims, wstr, wbox)) return cudaErrorInvalidValue;
  const LinearPlus plus{(const __nv_bfloat16*)o.bias, (const __nv_bfloat16*)o.residual, o.a_scale, o.w_scale, (__nv_bfloat16*)o.c, o.ldc, o.ldr};
  switch (form) {
    case 6: return run_split<kKind, 2>(o.M, o.N, o.K, ta, tw, o.act, plus, dev_status, s);
    case 7: return run_split<kKind, 4>(o.M, o.N, o.K, ta, tw, o.act, plus, dev_status, s);
    case 8: return run_split<kKind, 8>(o.M, o.N, o.K, ta, tw, o.act, plus, dev_status, s);
    case 9: return run_pair_split<kKind, 2>(o.M, o.N, o.K, ta, tw, o.act, plus, dev_status, s);
    case 10: return run_pair_split<kKind, 3>(o.M, o.N, o.K, ta, tw, o.act, plus, dev_status, s);
    default: break;
  }
  CUtensorMap tc, tr = tw, th = tw;
  const uint64_t cdims[2] = {(uint64_t)o.N, (uint64_t)o.M}, cstr[1] = {(uint64_t)o.ldc * 2}, rstr[1] = {(uint64_t)o.ldr * 2};
  const uint32_t cbox[2] = {64, 32};  // a warp's 32 rows of one 64-column slab
  const uint32_t hbox[2] = {f8 ? 128u : 32u, f8 ? 32u : 64u};  // half a slab of W
  if (!encode_tmap_16bit(&tc, o.c, 2, cdims, cstr, cbox) || (o.residual && !encode_tmap_16bit(&tr, o.residual, 2, cdims, rstr, cbox)) ||
      (form == 5 && !encode(&th, o.w, 2, wdims, wstr, hbox)))
    return cudaErrorInvalidValue;
  const CUtensorMap tws[3] = {tw, tr, th}, tcs[3] = {tc, tc, tc};
  return run_form<kKind>(form, d.pairs, o.M, o.N, o.K, 1, ta, tws, tcs, o.act, plus, dev_status, s);
}

template <int kKind>
PlusDevice plus_device() {  // (asked once per device)
  static std::once_flag once[64];
  static PlusDevice known[64];
  const auto ask = [] {
    return PlusDevice{sm_count(),
                      pairs_at_once(),
                      {splits_at_once<kKind, 2>(), splits_at_once<kKind, 4>(), splits_at_once<kKind, 8>()},
                      {pair_splits_at_once<kKind, 2>(), pair_splits_at_once<kKind, 3>()}};
  };
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return ask();
  std::call_once(once[dev], [&] { known[dev] = ask(); });
  return known[dev];
}

// The form that a launch takes: plus_form()'s, or the test's where the shape and the device allow it.
template <int kKind>
int plus_form_of(int M, int N, int K, int act, const PlusDevice& d) {
  const int steps = (K + kStepK<kKind> - 1) / kStepK<kKind>;
  if (const int v = g_tune_linear_tile.load(std::memory_order_relaxed); v >= 2 && v <= 10) {  // test-only override
    const bool pair = v == 3 || v == 5, split = v >= 6 && v <= 8;
    if (pair ? M > 128 && d.pairs > 0 : split ? steps >= 1 << (v - 5) && d.split[v - 6] > 0 : v < 9 || (steps >= v - 7 && d.pair_split[v - 9] > 0)) return v;
  }
  return plus_form(M, N, steps, act, d);
}
bool few_rows(int M) {
  const int tune = g_tune_linear_tile.load(std::memory_order_relaxed);  // test-only
  return M <= 16 && (tune < 2 || tune > 10);
}

template <int kKind>
cudaError_t launch_plus(const LinearPlusOp& o, uint32_t* dev_status, cudaStream_t s) {
  const PlusDevice d = plus_device<kKind>();
  return run_plus<kKind>(o, plus_form_of<kKind>(o.M, o.N, o.K, o.act, d), d, dev_status, s);
}

}  // namespace

// c = act(a w + bias) + residual; strides in elements.  bf16: w [K][N].  e4m3 (f8): a and w [N][K] with a_scale [M], w_scale [N].
cudaError_t launch_linear_plus_tc(const LinearPlusOp& o, uint32_t* dev_status, cudaStream_t s) {
  if (few_rows(o.M)) return launch_linear_rows(o, false, s);
  return o.f8 ? launch_plus<kPlus8>(o, dev_status, s) : launch_plus<kPlus>(o, dev_status, s);
}

int linear_plus_form(int M, int N, int K, bool f8, int act) {
  if (few_rows(M)) return 1;
  return f8 ? plus_form_of<kPlus8>(M, N, K, act, plus_device<kPlus8>()) : plus_form_of<kPlus>(M, N, K, act, plus_device<kPlus>());
}

}  // namespace toma
