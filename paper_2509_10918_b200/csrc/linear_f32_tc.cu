// c = act(a w + bias) + residual in fp32 on the tensor cores, for more than 16 rows.
//
// A float is the sum of three bf16 numbers, exactly: x = x0 + x1 + x2 with x0 = bf16(x), x1 = bf16(x - x0), x2 = x - x0 - x1 (8 bits
// each of the 24).  Of the nine products of two such sums three are left out (two of at most 2^-25 of the whole, one of 2^-34), the other six are
// multiplied by tcgen05, whose products are exact and whose sums are in fp32.  A long chain of such sums is not as exact as one of
// fused multiply-adds (they are cut off, not rounded), so a chain ends after 128 contraction elements, the five small products have one
// of their own, and the chains' sums are added up by the threads, rounded: 512 x 256 x 640 is 2.0 units of 2^-24 off 64 bits
// (root mean square), 7.6 on FFMA; with 4096 contraction elements 2.3 and 19.  At the rate of a large bf16 product six of them make
// 275 TFLOP/s, FFMA has 75; 2048 x 1152 x 1280 takes 44 us (137 TFLOP/s).
//
// A CTA has a tile of 128 x 128 or 128 x 64.  Two groups of eight warps take the floats of every second stage of 32 contraction elements from
// global memory, the group's next stage in registers meanwhile, and cut them into three planes each in shared memory (four
// stages); a stage is a chain of latencies for a warp, which the other group's stage covers (sixteen warps on every stage took
// 1900 cycles for each, whose instructions take 650 and MMAs 770).  All sixteen add up the chains' sums, 32 or 16 columns of a row a
// thread; a seventeenth issues the MMAs.  Where there are few tiles a cluster of 2 or 4 CTAs splits the contraction
// and exchanges its parts through distributed shared memory.
#include <climits>

#include "clusters.cuh"
#include "common.cuh"
#include "linear_epilogue.cuh"
#include "tc.cuh"

namespace toma {

using namespace tc;

namespace {

constexpr int kWarps = 16;                       // that cut and add
constexpr int kStep = 32, kSlots = 4, kChunk = 4;  // contraction elements of a stage, stages in shared memory, stages of a chain
constexpr int kPlaneA = 128 * kStep * 2, kSlab = kStep * 128;  // rows of 64 bytes of a; 64 columns of w
template <int NT> constexpr int kPlaneW = NT / 64 * kSlab;
template <int NT> constexpr int kStageBytes = 3 * (kPlaneA + kPlaneW<NT>);
template <int NT> constexpr int kSmem = 1024 + kSlots * kStageBytes<NT> + 256;

struct F32Bars {
  uint64_t full[kSlots], empty[kSlots];  // the planes are there; have been multiplied
  uint64_t done[2], taken[2];            // a chain's sums are there; have been taken
  uint32_t tmem_base;
  int abort_flag;
};
static_assert(sizeof(F32Bars) <= 256, "barrier block outgrew its reservation");

struct F32Op {
  const float *a, *w, *bias, *residual;
  float* c;
  int lda, ldw, ldr, ldc, M, N, K, act;
};

// Eight floats, the first and the second four of which are there or zeros; wide: on a 32-byte boundary, and all or none.
__device__ __forceinline__ void load_floats(uint32_t (&v)[8], const float* p, bool first, bool second, bool wide) {
  if (wide) {
    if (first) {
      asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                   : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7])
                   : "l"(p));
      return;
    }
  }
  const uint4 none = make_uint4(0, 0, 0, 0);
  const uint4 lo = !wide && first ? *reinterpret_cast<const uint4*>(p) : none, hi = !wide && second ? *reinterpret_cast<const uint4*>(p + 4) : none;
  v[0] = lo.x, v[1] = lo.y, v[2] = lo.z, v[3] = lo.w, v[4] = hi.x, v[5] = hi.y, v[6] = hi.z, v[7] = hi.w;
}
// Eight floats as three packets of bf16.
__device__ __forceinline__ void cut(const uint32_t (&x)[8], uint8_t* at, int plane) {
  float v[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(x[e]);
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
__global__ void __launch_bounds__((kWarps + 1) * 32, 1) linear_f32_kernel(const F32Op o, const bool wide, uint32_t* dev_status) {
  constexpr int kCols = NT / 4, kPart = kCols / S;  // columns of a thread; of which its CTA finishes
  constexpr int kPacksW = NT / 64;                  // packets of eight of w of a thread and stage (two of a)
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  F32Bars* bar = reinterpret_cast<F32Bars*>(smem + kSlots * kStageBytes<NT>);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = S > 1 ? (int)cluster_rank() : 0, tile = blockIdx.x / S;
  const int nk = (o.K + kStep - 1) / kStep, first = rank * nk / S, steps = (rank + 1) * nk / S - first;  // (nk >= S: one at least)
  const int chains = (steps + kChunk - 1) / kChunk;
  const int mb = (o.M + 127) / 128, m0 = tile % mb * 128, n0 = tile / mb * NT;

  if (tid == 0) {
    for (int s = 0; s < kSlots; ++s) {
      mbar_init(&bar->full[s], kWarps / 2);
      mbar_init(&bar->empty[s], 1);
    }
    for (int s = 0; s < 2; ++s) {
      mbar_init(&bar->done[s], 1);
      mbar_init(&bar->taken[s], kWarps);
    }
    bar->abort_flag = 0;
    mbar_fence_init();
  }
  dependency_wait();
  if (tid == 0) release_dependents();
  if (warp == kWarps) tmem_alloc(&bar->tmem_base, 4 * NT);
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
        const int s = i % kSlots, chain = i / kChunk, c = chain & 1;
        const bool begins = i % kChunk == 0;
        if (!mbar_wait(&bar->full[s], (i / kSlots) & 1, dev_status, abort_flag)) break;
        if (begins && chain >= 2 && !mbar_wait(&bar->taken[c], ((chain >> 1) - 1) & 1, dev_status, abort_flag)) break;
        tc_fence_after();
        const uint32_t aa = smem_u32(smem + s * kStageBytes<NT>), wa = aa + 3 * kPlaneA, large = tmem + c * 2 * NT, small = large + NT;
        constexpr int pa[6] = {2, 0, 1, 1, 0, 0}, pw[6] = {0, 2, 1, 0, 1, 0};
#pragma unroll
        for (int p = 0; p < 6; ++p)
#pragma unroll
          for (int kk = 0; kk < kStep / 16; ++kk)
            mma_ss(p < 5 ? small : large, smem_desc_sw64(aa + pa[p] * kPlaneA + kk * 32, 16, 512),
                   smem_desc_sw128(wa + pw[p] * kPlaneW<NT> + kk * 2048, kSlab, 1024), idesc, !begins || kk > 0 || (p > 0 && p < 5));
        mma_commit(&bar->empty[s]);
        if (i % kChunk == kChunk - 1 || i == steps - 1) mma_commit(&bar->done[c]);
      }
    }
  } else {
    // a thread's packets of eight: rows t / 4 and 64 further on of a; of w a row of 128 columns and 16 further on, or of 64
    const int half = warp >> 3, t = tid & 255, a_row = t >> 2, a_pk = t & 3, w_row = t / (NT / 8), w_pk = t % (NT / 8);
    const bool w_in = n0 + w_pk * 8 < o.N, w_whole = n0 + w_pk * 8 + 4 < o.N;
    const float* a_at = o.a + (size_t)(m0 + a_row) * o.lda + a_pk * 8;
    const float* w_at = o.w + (size_t)w_row * o.ldw + n0 + w_pk * 8;
    const uint32_t a_to = (uint32_t)a_row * 64u + (uint32_t)((a_pk ^ ((a_row >> 1) & 3)) << 4);
    const uint32_t w_to = 3 * kPlaneA + (w_pk >> 3) * kSlab + sw128_offset(w_row, w_pk & 7);
    uint32_t xa[2][8], xw[kPacksW][8];
    const auto fetch = [&](int step) {
      const int k0 = (first + step) * kStep, ka = k0 + a_pk * 8;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const bool in = m0 + a_row + 64 * j < o.M;
        load_floats(xa[j], a_at + (size_t)64 * j * o.lda + k0, in && ka < o.K, in && ka + 4 < o.K, wide);
      }
#pragma unroll
      for (int j = 0; j < kPacksW; ++j) {
        const bool in = k0 + w_row + 16 * j < o.K;
        load_floats(xw[j], w_at + (size_t)(k0 + 16 * j) * o.ldw, w_in && in, w_whole && in, wide);
      }
    };
    const auto take = [&](int chain) {
      const int c = chain & 1;
      if (!mbar_wait_warp(&bar->done[c], (chain >> 1) & 1, dev_status, abort_flag)) return false;
      tc_fence_after();
      const uint32_t at = tmem + c * 2 * NT + group * kCols + ((uint32_t)(quarter * 32) << 16);
#pragma unroll
      for (int h = 0; h < kCols; h += 16) {
        uint32_t large[16], small[16];
        tmem_ld16(at + h, large);
        tmem_ld16(at + NT + h, small);
        tmem_wait_ld();
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[h + e] += __uint_as_float(large[e]) + __uint_as_float(small[e]);
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&bar->taken[c]);
      return true;
    };
    int taken = 0;
    if (half < steps) fetch(half);
    for (int i = half; ok && i < steps; i += 2) {
      const int s = i % kSlots;
      if (i >= kSlots && !mbar_wait_warp(&bar->empty[s], (i / kSlots - 1) & 1, dev_status, abort_flag)) { ok = false; break; }
      uint8_t* at = smem + s * kStageBytes<NT>;
#pragma unroll
      for (int j = 0; j < 2; ++j) cut(xa[j], at + a_to + j * 64 * 64, kPlaneA);
#pragma unroll
      for (int j = 0; j < kPacksW; ++j) cut(xw[j], at + w_to + j * 16 * 128, kPlaneW<NT>);
      fence_proxy_async();
      __syncwarp();
      if (lane == 0) mbar_arrive(&bar->full[s]);
      if (i + 2 < steps) fetch(i + 2);
      if (i % kChunk >= 2 && i >= kChunk) ok = take(taken++);  // the chain before
    }
    while (ok && taken < chains) ok = take(taken++);
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
    // An infinity is no sum of three numbers: where one or a none-number has come in, the sums are taken as they are defined, four
    // columns at a time.  (A row with a none-number in it has nothing else, so that rows of padding do not cost their length times the
    // columns.  4096 x 2560 x 2560 takes 0.39 ms, with an infinity in one row 2.3, in one column 2.3, in each row 28; an element at a
    // time 24, 1.3 and 117.  Eight columns and four rows of w at a time 1.5, 1.1 and 7.4, but all other products 2 to 4 % longer: the forms
    // of 128 columns have no register left, and spill 104 to 156 bytes as they are.)
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
      for (int c = 0; c < kPart; c += 4) {
        if (n_first + c >= o.N) continue;
        float4 sum = none ? make_float4(NAN, NAN, NAN, NAN) : make_float4(0.f, 0.f, 0.f, 0.f);
        const float* at = o.w + n_first + c;
#pragma unroll 4
        for (int k = none ? o.K : 0; k < o.K; ++k, at += o.ldw) {
          const float x = row[k];
          const float4 w = *reinterpret_cast<const float4*>(at);
          sum.x = fmaf(x, w.x, sum.x), sum.y = fmaf(x, w.y, sum.y), sum.z = fmaf(x, w.z, sum.z), sum.w = fmaf(x, w.w, sum.w);
        }
        if (!(fabsf(v[c]) < INFINITY)) v[c] = sum.x;
        if (!(fabsf(v[c + 1]) < INFINITY)) v[c + 1] = sum.y;
        if (!(fabsf(v[c + 2]) < INFINITY)) v[c + 2] = sum.z;
        if (!(fabsf(v[c + 3]) < INFINITY)) v[c + 3] = sum.w;
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
        for (int u = 0; u < 4; ++u) v[e + u] = epi::activate_f32(v[e + u], o.act);
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
    tmem_dealloc(tmem, 4 * NT);
  }
}

template <int NT, int S>
int f32_at_once() {
  static ClusterState st;
  if (S == 1) return sm_count();  // (a CTA's shared memory is an SM's)
  return clusters_at_once(linear_f32_kernel<NT, S>, st, S, (kWarps + 1) * 32, kSmem<NT>);
}
template <int NT, int S>
cudaError_t run_f32(const F32Op& o, uint32_t* dev_status, cudaStream_t s) {
  const long long ctas = (long long)((o.M + 127) / 128) * ((o.N + NT - 1) / NT) * S;
  if (ctas > INT32_MAX) return cudaErrorInvalidValue;
  static std::atomic<unsigned long long> raised{0};
  if (cudaError_t e = raise_dynamic_smem(linear_f32_kernel<NT, S>, kSmem<NT>, raised); e != cudaSuccess) return e;
  const bool wide = (((uintptr_t)o.a | (uintptr_t)o.w) & 31) == 0 && o.lda % 8 == 0 && o.ldw % 8 == 0 && o.N % 8 == 0 && o.K % 8 == 0;
  if (S == 1) return launch_dependent(linear_f32_kernel<NT, S>, dim3((unsigned)ctas), dim3((kWarps + 1) * 32), (size_t)kSmem<NT>, s, o, wide, dev_status);
  return launch_dependent_cluster(linear_f32_kernel<NT, S>, dim3((unsigned)ctas), dim3((kWarps + 1) * 32), (size_t)kSmem<NT>, S, s, o, wide, dev_status);
}

// Rounds of tiles, each a fixed part and a part per stage: nanoseconds, fitted to 20 shapes between 20 x 312 x 3272 and 4096 x 2560 x 640
// that were timed in every form (the form named takes at most 1.07 times as long as the best).
struct F32Form {
  int cols, parts, at_once, round, step;
  cudaError_t (*run)(const F32Op&, uint32_t*, cudaStream_t);
};
struct F32Choice {
  int form;
  long long cost;
};
F32Choice f32_choice(const F32Form (&forms)[6], int M, int N, int steps) {
  F32Choice best{-1, LLONG_MAX};
  for (int i = 0; i < 6; ++i) {
    const F32Form& f = forms[i];
    if (f.at_once < 1 || steps < f.parts) continue;
    const long long tiles = (long long)((M + 127) / 128) * ((N + f.cols - 1) / f.cols);
    const long long cost = (tiles + f.at_once - 1) / f.at_once * (f.round + (long long)((steps + f.parts - 1) / f.parts) * f.step);
    if (cost < best.cost) best = F32Choice{i, cost};
  }
  return best;
}

}  // namespace

// Where the last round of tiles of 128 x 128 would leave most SMs idle, the columns (or rows) of the whole rounds are one launch and
// the rest is another, in the form that suits it: 1003 x 2560 x 640, 160 tiles on 148 SMs, 38 us instead of 52.
cudaError_t launch_linear_f32_tc(const LinearPlusOp& l, uint32_t* dev_status, cudaStream_t s) {
  const F32Op whole{(const float*)l.a, (const float*)l.w, (const float*)l.bias, (const float*)l.residual, (float*)l.c, l.lda, l.ldw, l.ldr, l.ldc, l.M, l.N, l.K, l.act};
  const F32Form forms[] = {{128, 1, f32_at_once<128, 1>(), 9600, 810, run_f32<128, 1>}, {64, 1, f32_at_once<64, 1>(), 6000, 530, run_f32<64, 1>},
                           {128, 2, f32_at_once<128, 2>(), 8600, 740, run_f32<128, 2>}, {128, 4, f32_at_once<128, 4>(), 8000, 790, run_f32<128, 4>},
                           {64, 2, f32_at_once<64, 2>(), 6100, 540, run_f32<64, 2>},    {64, 4, f32_at_once<64, 4>(), 5800, 570, run_f32<64, 4>}};
  const int steps = (l.K + kStep - 1) / kStep, mb = (l.M + 127) / 128, nb = (l.N + 127) / 128;
  F32Choice one = f32_choice(forms, l.M, l.N, steps), rest{-1, 0};
  F32Op first = whole, second = whole;
  if (const int tune = g_tune_linear_tile.load(std::memory_order_relaxed); tune >= 1 && tune <= 6) {  // test-only
    if (forms[tune - 1].at_once > 0 && steps >= forms[tune - 1].parts) one.form = tune - 1;
  } else if (const int at_once = forms[0].at_once; at_once > 0) {
    const long long rounds = (long long)mb * nb / at_once;
    const bool by_columns = mb <= at_once;
    const int blocks = (int)(rounds * at_once / (by_columns ? mb : nb)) * 128;  // columns (rows) of the whole rounds
    if (blocks > 0 && blocks < (by_columns ? l.N : l.M)) {
      F32Op f = whole, r = whole;
      if (by_columns) {
        f.N = blocks, r.N -= blocks;
        r.w += blocks, r.c += blocks;
        if (r.bias) r.bias += blocks;
        if (r.residual) r.residual += blocks;
      } else {
        f.M = blocks, r.M -= blocks;
        r.a += (size_t)blocks * r.lda, r.c += (size_t)blocks * r.ldc;
        if (r.residual) r.residual += (size_t)blocks * r.ldr;
      }
      const F32Choice behind = f32_choice(forms, r.M, r.N, steps);
      const long long cost = rounds * (forms[0].round + (long long)steps * forms[0].step) + behind.cost;
      if (behind.form >= 0 && cost < one.cost) one = F32Choice{0, cost}, rest = behind, first = f, second = r;
    }
  }
  if (one.form < 0) return cudaErrorInvalidValue;
  cudaError_t e = forms[one.form].run(first, dev_status, s);
  count_launch();
  if (e == cudaSuccess && rest.form >= 0) {
    e = forms[rest.form].run(second, dev_status, s);
    count_launch();
  }
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace toma
