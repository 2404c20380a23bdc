// Products of a few packed rows with 4-bit weights (the projections of Algorithm 1 lines 10, 12, 15 for weights held in
// four bits):
//
//   C[r][n] = sum_k A[r][k] W[n][k],   W[n][k] = (u[n][k] - z[n][k / g]) * s[n][k / g],   u = 0 ... 15
//
// with the epilogues of surelock_gemm_fused.  What bounds it with few rows: the weights, K / 2 bytes per output feature and
// their scales, are streamed once; the instructions that make operands of the codes come next, 46 codes per clock and SM at
// the memory's rate.
//
// A 4-bit code in a byte IS a number of the e4m3 format: the byte u = 0 ... 15 means u 2^-9 (subnormal up to 7, then exponent
// field 1).  So the codes enter an 8-bit tcgen05.mma after three instructions per eight of them (even and odd ones masked
// into two words), and the activations take the other side of the bargain: a small kernel in front splits every row, group
// by group of k, into two e4m3 terms, a = 2^e (t1 + t2), e from the group's largest magnitude in the row.  A bf16 number's 8
// bits are 4 + 4, so the split is exact down to 2^-9 of that magnitude, and off by at most 2^-17 of it below.  Per group
//   sum_k (u - z) a = 2^(e + 9) (D - z q),   D = sum_k (u 2^-9) (t1 + t2),   q = 2^-9 sum_k (t1 + t2),
// D from the products (both terms into one accumulator), q and 2^e from the splitting kernel; the bracket is formed in fp32
// and multiplied by its group's scale in fp32, so a weight is never rounded.
// The weights are the 128-row operand, read from TENSOR MEMORY: one thread per feature takes its codes from a TMA stage and
// stores twice as many bytes there.  The rows' terms, NP = 16 ... 128 rows, are the N operand, by TMA.
//   warps 0-7  feature 32 (w % 4) + lane; w / 4 = half of the k of a step for unpacking, half of the rows for adding up
//   warp 8     one thread issues the TMA copies: codes (128 features x 128 bytes per matrix), terms, q and 2^e of a stage's 256 k
//   warp 9     one thread issues the MMAs of a step, 8 per 128 k
// The eight warps unpack step i into one of two operand tiles while the MMAs of step i - 1 run, hand it over and add up step
// i - 1; with two sets of accumulators (where tensor memory has room) it is handed over before that.  The first codes are
// requested before the splitting kernel has finished: it does not write them.
// Many features: a CTA goes on from tile to tile, results are stored from the registers.  Few: K is split over the CTAs of a
// cluster, whose sums meet through distributed shared memory in a fixed order: deterministic.  With SwiGLU a step is two
// tiles, gate and up, that share the rows' terms.  All waits are bounded.
#include <cuda_fp16.h>

#include <mutex>

#include "tc_common.cuh"

namespace sl {

namespace {

constexpr int GQ_THREADS = 320;
constexpr int GQ_BK = 256;             // k per stage: 128 bytes of a feature's codes (64-byte rows stream at two thirds of the rate)
constexpr int GQ_CODES = 128 * GQ_BK / 2;

struct GqArgs {
  const uint8_t* zeros[2];
  const void* scales[2];
  void* C;
  const int32_t* n_active;
  int max_rows, n_out, K, ng;
  int vec;                             // a 16-byte load of scales (and the zero points with it) is aligned
  int32_t* status;
};

__device__ __forceinline__ void gq_mma_ta(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc, uint32_t accum) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d_tmem), "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accum)
      : "memory");
}
__device__ __forceinline__ void tc_ld8(uint32_t taddr, uint32_t* r) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tc_ld16(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
        "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ float4 ld_cluster_f4(uint32_t a) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ uint4 gq_lds128(uint32_t a) {
  uint4 r;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "r"(a) : "memory");
  return r;
}
__device__ __forceinline__ void tc_st16(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ float gq_pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }   // -126 <= e <= 127

// Scales and zero points of one feature, group after group: 16 bytes of scales (8 bf16 or 4 fp32) with their zero points at a
// time, the next ones requested one such chunk ahead.
template <bool FP32> struct GroupReader {
  static constexpr int CHUNK = FP32 ? 4 : 8;
  const uint8_t *s0, *z0;      // of feature 0; z0 may be null
  const uint8_t *s, *z;        // of the present feature
  uint32_t c[4], n[4];         // present and next chunk of scales
  uint32_t cz[2], nz[2];       // ... and of zero points
  int grp, end, ng;            // next group, end of this CTA's range, groups of the feature
  bool vec;

  __device__ __forceinline__ void fetch(int g0) {   // chunk of groups from g0 (a multiple of the chunk) -> n, nz
    if (g0 >= end) return;
    if (vec) {
      const uint4 x = __ldg(reinterpret_cast<const uint4*>(s + (size_t)g0 * (FP32 ? 4 : 2)));
      n[0] = x.x; n[1] = x.y; n[2] = x.z; n[3] = x.w;
      if (z) {
        nz[0] = __ldg(reinterpret_cast<const uint32_t*>(z + g0));
        if (!FP32) nz[1] = __ldg(reinterpret_cast<const uint32_t*>(z + g0 + 4));
      }
      return;
    }
#pragma unroll
    for (int i = 0; i < CHUNK; ++i)                   // features whose scales do not start on 16-byte boundaries
      if (g0 + i < ng) {
        if (FP32) n[i & 3] = __ldg(reinterpret_cast<const uint32_t*>(s) + g0 + i);
        else n[i >> 1] = __byte_perm(n[i >> 1], __ldg(reinterpret_cast<const uint16_t*>(s) + g0 + i), i & 1 ? 0x5410 : 0x3254);
        if (z) {
          const uint32_t x = (uint32_t)__ldg(z + g0 + i) << (8 * (i & 3));
          nz[i >> 2] = (nz[i >> 2] & ~(0xffu << (8 * (i & 3)))) | x;
        }
      }
  }
  __device__ __forceinline__ void rotate() {          // drop the first group of the chunk
    if (FP32) {
      c[0] = c[1]; c[1] = c[2]; c[2] = c[3];
    } else {
      c[0] = __funnelshift_r(c[0], c[1], 16); c[1] = __funnelshift_r(c[1], c[2], 16); c[2] = __funnelshift_r(c[2], c[3], 16); c[3] >>= 16;
    }
    cz[0] = __funnelshift_r(cz[0], cz[1], 8);
    cz[1] >>= 8;
  }
  __device__ __forceinline__ void turn() {
#pragma unroll
    for (int i = 0; i < 4; ++i) c[i] = n[i];
    cz[0] = nz[0];
    cz[1] = nz[1];
  }
  __device__ __forceinline__ void begin(long long feature, int g, int e) {   // requests the first chunk
    s = s0 + feature * ng * (FP32 ? 4 : 2);
    z = z0 ? z0 + feature * ng : nullptr;
#pragma unroll
    for (int i = 0; i < 4; ++i) n[i] = 0;
    nz[0] = nz[1] = 0x08080808u;
    grp = g;
    end = e;
    fetch(g & ~(CHUNK - 1));
  }
  __device__ __forceinline__ void prime() {                                  // before the first next()
    const int at = grp & ~(CHUNK - 1);
    turn();
    fetch(at + CHUNK);
    for (int i = at; i < grp; ++i) rotate();
  }
  // scale times 2^9 and minus the zero point of the next group (behind the feature's last one anything finite: its D and q are 0)
  __device__ __forceinline__ void next(float& scale, float& minus_z) {
    scale = __uint_as_float(FP32 ? c[0] : c[0] << 16) * 512.f;
    minus_z = -(float)(cz[0] & 0xffu);
    ++grp;
    if ((grp & (CHUNK - 1)) == 0) {
      turn();
      fetch(grp + CHUNK);
    } else {
      rotate();
    }
  }
};

template <int G, int NP, bool DUAL> struct GqPlan {
  static constexpr int T = DUAL ? 2 : 1;
  static constexpr int GPT = GQ_BK / G;                       // groups per stage
  static constexpr int KS = NP <= 32 && GPT * NP <= 64 ? GQ_BK : GQ_BK / 2;   // k per step: as the accumulators' columns allow
  static constexpr int H = GQ_BK / KS;                        // steps per stage and matrix
  static constexpr int GPS = KS / G;                          // groups per step
  static constexpr int SLAB = NP * 128;                       // bytes of one term of NP rows of 128 k
  static constexpr int TERMS = 4 * SLAB;                      // t1 and t2 of the first 128 k, then of the second
  static constexpr int SUMS = GPT * NP * 8;                   // q and 2^e of a stage
  static constexpr int LOADED = T * GQ_CODES + TERMS + SUMS;
  static constexpr int STAGE = T * GQ_CODES + TERMS + (SUMS + 1023) / 1024 * 1024;
  static constexpr uint32_t A_COLS = KS / 4, D_COL = 2 * A_COLS, D_COLS = GPS * NP;   // two operand tiles, then accumulators
  static constexpr bool TWICE = D_COL + 2 * D_COLS <= 512;    // two sets of accumulators
  static constexpr uint32_t USED = D_COL + (TWICE ? 2 : 1) * D_COLS, COLS = USED <= 128 ? 128 : USED <= 256 ? 256 : 512;
  static constexpr int OCC = NP * T <= 32 && COLS <= 256 ? 2 : 1;
  static constexpr int ROOM = (OCC == 2 ? 112 : 220) * 1024 - 2048;
  static constexpr int STAGES = ROOM / STAGE > 6 ? 6 : ROOM / STAGE;
  static constexpr int PITCH = T * 128;                       // floats per packed row of the partial sums
  static constexpr int SMEM = 1024 + STAGES * STAGE + 512;
  static_assert(USED <= 512, "tensor memory");
  static_assert(STAGES >= 2 && NP * PITCH * 4 <= STAGES * STAGE, "partial sums take the place of the stages");
};

// ---- the rows' terms -------------------------------------------------------------------------------------------------
// 8 k per thread; per (row, group): e from the largest magnitude, a' = a 2^-e in [-256, 256], t1 = e4m3(a'), t2 = e4m3(a' -
// t1); the bytes of 8 k in the order 0 2 4 6 1 3 5 7 in which the codes come out of their words.  A group with an infinity
// or a NaN is NaN throughout.  terms: [2][max_rows][Kp], Kp = K rounded up to 256, zeros behind K; sums: [Kp / g][ld] of (q, 2^e).
constexpr int GS_THREADS = 256;

template <int G>
__global__ void __launch_bounds__(GS_THREADS)
gq_split_rows_kernel(const bf16* __restrict__ A, const int32_t* __restrict__ n_active, int max_rows, int K, int Kp, int ld,
                     uint8_t* __restrict__ terms, float2* __restrict__ sums) {
  griddep_wait();
  griddep_launch();
  const int r = blockIdx.y, i = blockIdx.x * GS_THREADS + threadIdx.x;
  if (r >= min(*n_active, max_rows)) return;
  uint4 v = make_uint4(0, 0, 0, 0);
  if (i < K / 8) v = __ldg(reinterpret_cast<const uint4*>(A + (long long)r * K) + i);
  constexpr uint32_t MAG = 0x7fff7fffu;
  uint32_t top = __vmaxu2(__vmaxu2(v.x & MAG, v.y & MAG), __vmaxu2(v.z & MAG, v.w & MAG));
#pragma unroll
  for (int o = 1; o < G / 8; o <<= 1) top = __vmaxu2(top, __shfl_xor_sync(0xffffffffu, top, o));
  top = max(top & 0xffffu, top >> 16);
  const bool bad = top >= 0x7f80u;
  int e = (int)(top >> 7) - 127 - 7;                 // the largest magnitude becomes 128 ... 256
  if (top == 0 || bad) e = 0;
  e = max(e, -133);                                  // subnormal numbers
  const float d0 = gq_pow2(-e / 2), d1 = gq_pow2(-e - (-e / 2));
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  float x[8], sum = 0.f;
  uint32_t t1[2] = {}, t2[2] = {};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    x[2 * j] = __uint_as_float(w[j] << 16) * d0 * d1;
    x[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u) * d0 * d1;
  }
  auto widen = [](uint16_t two) {
    uint32_t f;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(f) : "h"(two));
    return __half22float2(*reinterpret_cast<const __half2*>(&f));
  };
#pragma unroll
  for (int h = 0; h < 2; ++h)                        // even k, odd k
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int a = 4 * j + h, b = a + 2;
      uint16_t c, d;
      asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(c) : "f"(x[b]), "f"(x[a]));
      const float2 high = widen(c);
      asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(d) : "f"(x[b] - high.y), "f"(x[a] - high.x));
      const float2 low = widen(d);
      t1[h] |= (uint32_t)c << (16 * j);
      t2[h] |= (uint32_t)d << (16 * j);
      sum += (high.x + low.x) + (high.y + low.y);
    }
  if (bad) {
    t1[0] = t1[1] = 0x7f7f7f7fu;
    sum = __uint_as_float(0x7fffffffu);
  }
#pragma unroll
  for (int o = 1; o < G / 8; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (i < Kp / 8) {
    const long long at = (long long)r * Kp + 8 * i;
    *reinterpret_cast<uint2*>(terms + at) = make_uint2(t1[0], t1[1]);
    *reinterpret_cast<uint2*>(terms + (long long)max_rows * Kp + at) = make_uint2(t2[0], t2[1]);
    if (i % (G / 8) == 0) sums[(long long)(i / (G / 8)) * ld + r] = make_float2(sum * 0.001953125f, ldexpf(1.f, e));
  }
}

}  // namespace

template <int G, int NP, bool DUAL, bool FP32>
__global__ void __launch_bounds__(GQ_THREADS, GqPlan<G, NP, DUAL>::OCC)
gemm_quantized_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmW2,
                      const __grid_constant__ CUtensorMap tmT, const __grid_constant__ CUtensorMap tmQ, const GqArgs a,
                      const int epilogue) {
  using P = GqPlan<G, NP, DUAL>;
  constexpr int T = P::T, H = P::H, GPS = P::GPS, HC = NP / 2;   // HC: rows that a thread adds up
  constexpr int SPS = T * H;                                  // steps per stage: for every part of its k, gate then up
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  float* sRed = reinterpret_cast<float*>(smem);               // [NP][PITCH] after the last step
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + P::STAGES * P::STAGE);
  const uint32_t bar0 = smem_u32(bars);
  auto full = [&](int s) { return bar0 + 8u * s; };
  auto empty = [&](int s) { return bar0 + 8u * (P::STAGES + s); };
  auto a_full = [&](int i) { return bar0 + 8u * (2 * P::STAGES + (i & 1)); };       // of step i: operand tile written
  auto done = [&](int i) { return bar0 + 8u * (2 * P::STAGES + 2 + (i & 1)); };     // of step i: MMAs finished
  uint32_t* s_tmem = reinterpret_cast<uint32_t*>(bars + 2 * P::STAGES + 4);
  volatile int* s_abort = reinterpret_cast<volatile int*>(s_tmem + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < P::STAGES; ++i) {
      mbar_init(full(i), 1);
      mbar_init(empty(i), 8 + 8 + 1);                         // readers of the codes, of q (a step later), and the MMAs
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(a_full(i), 8);
      mbar_init(done(i), 1);
    }
    *s_abort = 0;
    fence_mbar_init();
  }
  if (warp == 9) tc_alloc(smem_u32(s_tmem), P::COLS);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *s_tmem;

  uint32_t S, rank = 0;
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(S));
  if (S > 1) rank = cluster_ctarank();
  const int r0 = blockIdx.y * NP, tiles = (a.n_out + 127) / 128;
  const int tile0 = blockIdx.x / S, tile_step = gridDim.x / S;   // a cluster of more than one CTA has one tile
  // *n_active, the weights and C were written before the splitting kernel began; its terms come after griddep_wait()
  const int M = min(*a.n_active, a.max_rows) - r0;            // rows of this tile; none: the whole cluster leaves
  const int nblk = (a.K + GQ_BK - 1) / GQ_BK;
  const int b0 = (int)((long long)nblk * rank / S), b1 = (int)((long long)nblk * (rank + 1) / S);
  const int my_tiles = M > 0 && tile0 < tiles ? (tiles - tile0 + tile_step - 1) / tile_step : 0;
  const int nstage = b1 - b0, per_tile = nstage * SPS, steps = my_tiles * per_tile;

  float acc[T][HC];
  auto clear = [&]() {
#pragma unroll
    for (int i = 0; i < T; ++i)
#pragma unroll
      for (int c = 0; c < HC; ++c) acc[i][c] = 0.f;
  };
  clear();

  if (warp == 8) {
    if (lane == 0) {
      const uint64_t once = gridDim.y > 1 ? l2_policy_evict_normal() : l2_policy_evict_first();   // a code is read once per row tile
      const int n = my_tiles * nstage, ahead = min(n, P::STAGES);
      int ct = tile0, cb = b0;                                // tile and block of the next codes
      auto codes = [&](int i) {
        const int st = i % P::STAGES;
        const uint32_t at = smem_u32(smem + st * P::STAGE);
        mbar_expect_tx(full(st), P::LOADED);
        tma_load_2d_hint(at, &tmW, cb * (GQ_BK / 2), ct * 128, full(st), once);
        if (DUAL) tma_load_2d_hint(at + GQ_CODES, &tmW2, cb * (GQ_BK / 2), ct * 128, full(st), once);
        if (++cb == b1) {
          cb = b0;
          ct += tile_step;
        }
      };
      for (int i = 0; i < ahead; ++i) codes(i);
      griddep_wait();
      griddep_launch();
      bool ok = true;
      int i = 0, b = b0;
      for (; i < n; ++i) {
        const int st = i % P::STAGES;
        if (i >= ahead) {
          if (!(ok = mbar_wait(empty(st), ((i / P::STAGES) & 1) ^ 1, s_abort))) break;
          codes(i);
        }
        const uint32_t at = smem_u32(smem + st * P::STAGE) + T * GQ_CODES;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          tma_load_2d(at + (2 * k) * P::SLAB, &tmT, b * GQ_BK + k * 128, r0, full(st));
          tma_load_2d(at + (2 * k + 1) * P::SLAB, &tmT, b * GQ_BK + k * 128, a.max_rows + r0, full(st));
        }
        tma_load_2d(at + P::TERMS, &tmQ, 2 * r0, b * P::GPT, full(st));
        if (++b == b1) b = b0;
      }
      if (!ok) {
        // gave up: wait (bounded) for the copies in flight, which write to this CTA's shared memory
        const unsigned long long t0 = clock64();
        for (int k = max(0, i - P::STAGES); k < i; ++k)
          while (!mbar_try(full(k % P::STAGES), (k / P::STAGES) & 1) && clock64() - t0 < TC_WAIT_CYCLES) {}
        set_status(a.status, SL_DEV_GEMM_TIMEOUT);
      }
    }
  } else if (warp == 9) {
    if (lane == 0) {
      constexpr uint32_t idesc = (1u << 4) | ((uint32_t)(NP >> 3) << 17) | (8u << 24);   // e4m3 x e4m3 -> fp32, M = 128, N = NP
      for (int i = 0; i < steps; ++i) {
        const int sg = i / SPS, st = sg % P::STAGES, part = i % SPS / T;
        if (!mbar_wait(full(st), (sg / P::STAGES) & 1, s_abort) || !mbar_wait(a_full(i), (i >> 1) & 1, s_abort)) {
          set_status(a.status, SL_DEV_GEMM_TIMEOUT);
          const unsigned long long t0 = clock64();            // the last step issued still uses the tensor memory
          while (i > 0 && !mbar_try(done(i - 1), ((i - 1) >> 1) & 1) && clock64() - t0 < TC_WAIT_CYCLES) {}
          break;
        }
        tc_fence_after();
        const uint32_t rows = smem_u32(smem + st * P::STAGE + T * GQ_CODES) + part * 2 * P::SLAB;
        const uint32_t d = tmem + P::D_COL + (P::TWICE ? (i & 1) * P::D_COLS : 0), op = tmem + (i & 1) * P::A_COLS;
#pragma unroll
        for (int k = 0; k < P::KS / 32; ++k)                  // 32 k: 8 columns of the operand, 32 bytes of the terms' rows
#pragma unroll
          for (int term = 0; term < 2; ++term)
            gq_mma_ta(d + (k / (G / 32)) * NP, op + k * 8, smem_desc_k_sw128(rows + (2 * (k >> 2) + term) * P::SLAB + (k & 3) * 32), idesc,
                      k % (G / 32) != 0 || term != 0);
        if (i % SPS == SPS - 1) tc_commit(empty(st));
        tc_commit(done(i));
      }
    }
  } else {
    const int lane_feature = (warp & 3) * 32 + lane, half = warp >> 2;
    const uint32_t lanes = (uint32_t)(warp & 3) << 21;        // this warp's lanes of the tensor memory
    constexpr int CH = P::KS / 64;                            // 16-byte chunks of a feature's codes that a thread unpacks in a step
    GroupReader<FP32> rd[T];
#pragma unroll
    for (int i = 0; i < T; ++i) {
      rd[i].vec = a.vec != 0;
      rd[i].s0 = (const uint8_t*)a.scales[i];
      rd[i].z0 = a.zeros[i];
      rd[i].ng = a.ng;
    }
    bool ok = true, fresh = false;
    // the codes of step i -> operand tile i & 1; `at` = its place among the stage's steps
    auto unpack = [&](int i, const int at) {
      const int sg = i / SPS, st = sg % P::STAGES, tile = at % T, part = at / T;
      if (at == 0) ok = __all_sync(0xffffffffu, mbar_wait(full(st), (sg / P::STAGES) & 1, s_abort));
      if (!ok) return;
      const uint32_t row = smem_u32(smem + st * P::STAGE + tile * GQ_CODES) + lane_feature * 128;
      const uint32_t dst = tmem + lanes + (i & 1) * P::A_COLS + half * (P::A_COLS / 2);
#pragma unroll
      for (int c = 0; c < CH; c += 2) {
        const uint32_t chunk = part * (8 / H) + half * CH + c;   // of the 128-byte row, swizzled
        const uint4 v0 = gq_lds128(row + ((chunk ^ (lane & 7)) << 4)), v1 = gq_lds128(row + (((chunk + 1) ^ (lane & 7)) << 4));
        const uint32_t w[8] = {v0.x, v0.y, v0.z, v0.w, v1.x, v1.y, v1.z, v1.w};
        uint32_t x[16];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          x[2 * j] = w[j] & 0x0f0f0f0fu;
          x[2 * j + 1] = (w[j] >> 4) & 0x0f0f0f0fu;
        }
        tc_st16(dst + c * 8, x);
      }
      if (at == SPS - 1) {
        __syncwarp();
        if (lane == 0) mbar_arrive(empty(st));
      }
    };
    // add up step i (accumulators of its groups)
    auto add = [&](int i, const int at) {
      const int st = i / SPS % P::STAGES, tile = at % T, part = at / T;
      if (fresh) {                                            // a new tile's first scales have arrived by now
#pragma unroll
        for (int m = 0; m < T; ++m) rd[m].prime();
        fresh = false;
      }
      ok = __all_sync(0xffffffffu, mbar_wait(done(i), (i >> 1) & 1, s_abort));
      if (!ok) return;
      tc_fence_after();
      const float4* sq = reinterpret_cast<const float4*>(smem + st * P::STAGE + T * GQ_CODES + P::TERMS) + part * GPS * (NP / 2) + half * (HC / 2);
      const uint32_t d0 = tmem + lanes + P::D_COL + (P::TWICE ? (i & 1) * P::D_COLS : 0) + half * HC;
      constexpr int LD = HC < 16 ? 8 : 16, LOADS = GPS * HC / LD;   // accumulators are requested one load ahead
      uint32_t d[2][LD];
      auto request = [&](int k) {
        const uint32_t col = d0 + (k * LD / HC) * NP + k * LD % HC;
        if (LD == 8) tc_ld8(col, d[k & 1]);
        else tc_ld16(col, d[k & 1]);
      };
      request(0);
      float sc = 0.f, mz = 0.f;
#pragma unroll
      for (int k = 0; k < LOADS; ++k) {
        const int g = k * LD / HC, c = k * LD % HC;
        if (c == 0) rd[tile].next(sc, mz);
        float4 qf[LD / 2];
#pragma unroll
        for (int e = 0; e < LD / 2; ++e) qf[e] = sq[g * (NP / 2) + c / 2 + e];
        tc_wait_ld();
        if (k + 1 < LOADS) request(k + 1);
#pragma unroll
        for (int e = 0; e < LD; ++e) {
          const float q = e & 1 ? qf[e / 2].z : qf[e / 2].x, f = e & 1 ? qf[e / 2].w : qf[e / 2].y;
          acc[tile][c + e] = fmaf(sc * f, fmaf(mz, q, __uint_as_float(d[k & 1][e])), acc[tile][c + e]);
        }
      }
      if (at == SPS - 1) {
        __syncwarp();
        if (lane == 0) mbar_arrive(empty(st));
      }
    };
    auto release = [&](int i) {                               // operand tile written; the accumulators of step i are free
      tc_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(a_full(i));
    };
    // one CTA to a tile: results straight from the registers, a warp's lanes are neighbouring features
    auto store = [&](int tile) {
      const int n = tile * 128 + lane_feature;
      if (n < a.n_out) {
#pragma unroll
        for (int c = 0; c < HC; ++c) {
          const int r = half * HC + c;
          if (r >= M) break;
          const long long out = (long long)(r0 + r) * a.n_out + n;
          const float x = acc[0][c];
          if (DUAL) reinterpret_cast<bf16*>(a.C)[out] = __float2bfloat16_rn(x / (1.f + __expf(-x)) * acc[T - 1][c]);
          else if (epilogue == EPI_RESIDUAL) reinterpret_cast<float*>(a.C)[out] += x;
          else reinterpret_cast<bf16*>(a.C)[out] = __float2bfloat16_rn(x);
        }
      }
      clear();
    };
    const int stages = my_tiles * nstage;
    for (int sg = 0, in_tile = 0, tile = tile0; sg < stages && ok; ++sg) {
#pragma unroll
      for (int at = 0; at < SPS; ++at) {
        const int i = sg * SPS + at;
        unpack(i, at);
        if (!ok) break;
        if (P::TWICE) release(i);
        if (i > 0) add(i - 1, (at + SPS - 1) % SPS);
        if (!ok) break;
        if (at == 0 && in_tile == 0) {                        // the tile before this one is complete
          if (sg > 0) {
            if (S == 1) store(tile);
            tile += tile_step;
          }
          const long long feature = min(tile * 128 + lane_feature, a.n_out - 1);
#pragma unroll
          for (int m = 0; m < T; ++m) rd[m].begin(feature, b0 * P::GPT, min(b1 * P::GPT, a.ng));
          fresh = true;
        }
        if (!P::TWICE) release(i);
      }
      if (++in_tile == nstage) in_tile = 0;
      if (sg == stages - 1 && ok) {
        add(steps - 1, SPS - 1);
        if (ok && S == 1) store(tile);
      }
    }
    if (!ok && lane == 0) set_status(a.status, SL_DEV_GEMM_TIMEOUT);
  }

  // ---- sums of the cluster, epilogue ----
  __syncthreads();
  if (warp == 9) {
    __syncwarp();
    tc_fence_after();
    tc_dealloc(tmem, P::COLS);
  }
  if (S == 1) return;
  const bool good = *s_abort == 0;
  if (warp < 8) {
    const int lane_feature = (warp & 3) * 32 + lane, half = warp >> 2;
#pragma unroll
    for (int i = 0; i < T; ++i)
#pragma unroll
      for (int c = 0; c < HC; ++c) sRed[(half * HC + c) * P::PITCH + i * 128 + lane_feature] = acc[i][c];
  }
  cluster_sync_all();
  if (my_tiles > 0 && good) {
    const uint32_t sred = smem_u32(sRed);
    auto total = [&](int at) {                                // four neighbouring features, the CTAs in order
      float4 p[8], x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (uint32_t s = 0; s < 8; ++s)
        if (s < S) p[s] = ld_cluster_f4(mapa_u32(sred + 4 * at, s));
#pragma unroll
      for (uint32_t s = 0; s < 8; ++s)
        if (s < S) {
          x.x += p[s].x; x.y += p[s].y; x.z += p[s].z; x.w += p[s].w;
        }
      return x;
    };
    const int c0 = (int)(32 * rank / S), cols = (int)(32 * (rank + 1) / S) - c0;   // features in fours that this CTA finishes
    for (int i = threadIdx.x; i < min(M, NP) * cols; i += GQ_THREADS) {
      const int r = i / cols, col = 4 * (c0 + i % cols), n = tile0 * 128 + col;
      if (n >= a.n_out) continue;
      const long long out = (long long)(r0 + r) * a.n_out + n;
      const float4 t = total(r * P::PITCH + col);
      float x[4] = {t.x, t.y, t.z, t.w};
      if (DUAL) {
        const float4 u = total(r * P::PITCH + 128 + col);
        const float up[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = x[e] / (1.f + __expf(-x[e])) * up[e];
      }
      if (epilogue == EPI_RESIDUAL && !DUAL) {
        float* c = reinterpret_cast<float*>(a.C) + out;
        if ((a.n_out & 3) == 0) {
          float4 y = *reinterpret_cast<const float4*>(c);
          y.x += x[0]; y.y += x[1]; y.z += x[2]; y.w += x[3];
          *reinterpret_cast<float4*>(c) = y;
        } else {
          for (int e = 0; e < 4; ++e)
            if (n + e < a.n_out) c[e] += x[e];
        }
      } else {
        bf16* c = reinterpret_cast<bf16*>(a.C) + out;
        if ((a.n_out & 3) == 0) {
          *reinterpret_cast<uint2*>(c) = make_uint2(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]));
        } else {
          for (int e = 0; e < 4; ++e)
            if (n + e < a.n_out) c[e] = __float2bfloat16_rn(x[e]);
        }
      }
    }
  }
  cluster_sync_all();                                         // the others may still be reading this CTA's partial sums
}

namespace {

// 2-D row-major tensor map, zeros out of bounds
int gq_map(CUtensorMap* out, const void* p, CUtensorMapDataType type, int elem, long long rows, long long cols, int box_rows, int box_cols,
           CUtensorMapSwizzle swizzle) {
  TensorMapEncodeFn fn = tensor_map_encode_fn();
  if (!fn) return SL_ECUDA;
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)cols * elem};
  const cuuint32_t box[2] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows}, one[2] = {1, 1};
  const CUresult r = fn(out, type, 2, const_cast<void*>(p), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
                        CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? SL_OK : SL_ECUDA;
}

// the workspace: terms, then (q, 2^e) with room for the smallest groups
struct GqWs {
  long long kp, ld;
  size_t q_at, bytes;
};
GqWs gq_ws(int max_rows, int K) {
  GqWs w;
  w.kp = ((long long)K + GQ_BK - 1) / GQ_BK * GQ_BK;
  w.ld = ((long long)max_rows + 1) / 2 * 2;          // rows of 16 bytes
  w.q_at = ((size_t)2 * max_rows * w.kp + 255) / 256 * 256;
  w.bytes = w.q_at + (size_t)w.kp / 32 * w.ld * 8;
  return w;
}

template <int G, int NP, bool DUAL, bool FP32>
int launch_gq(const CUtensorMap* w, void* ws, const GqWs& lay, const GqArgs& a, int epilogue, cudaStream_t st) {
  using P = GqPlan<G, NP, DUAL>;
  CUtensorMap terms, q;
  int rc = gq_map(&terms, ws, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, 2ll * a.max_rows, lay.kp, NP, 128, CU_TENSOR_MAP_SWIZZLE_128B);
  if (rc == SL_OK)
    rc = gq_map(&q, (char*)ws + lay.q_at, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 4, lay.kp / G, 2 * lay.ld, P::GPT, 2 * NP, CU_TENSOR_MAP_SWIZZLE_NONE);
  if (rc != SL_OK) return rc;
  const int tiles = (a.n_out + 127) / 128, nblk = (a.K + GQ_BK - 1) / GQ_BK, row_tiles = (a.max_rows + NP - 1) / NP;
  // With S = 1 the CTAs go on to further tiles, all of them resident.  Otherwise K is split over S CTAs: the S with the least
  // estimated time, rounds of CTAs times (stages of one + 3 stages' time to start and to join).
  const long long slots = (long long)sm_count() * P::OCC, work = (long long)tiles * row_tiles;
  int S = 1;
  long long best = (work + slots - 1) / slots * nblk * P::T + 2;
  for (int s = 2; s <= 8 && s <= nblk; ++s) {
    const long long t = (work * s + slots - 1) / slots * ((nblk + s - 1) / s * P::T + 3);
    if (t < best) {
      best = t;
      S = s;
    }
  }
  int grid = tiles * S;
  if (S == 1) {
    const int most = (int)(slots / row_tiles > 0 ? slots / row_tiles : 1), rounds = (tiles + most - 1) / most;
    grid = (tiles + rounds - 1) / rounds;
  }
  auto kernel = gemm_quantized_kernel<G, NP, DUAL, FP32>;
  static std::once_flag once;
  static cudaError_t attr;
  std::call_once(once, [&] { attr = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, P::SMEM); });
  SL_CUDA_TRY(attr);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid, row_tiles);
  cfg.blockDim = dim3(GQ_THREADS);
  cfg.dynamicSmemBytes = P::SMEM;
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  int n = 0;
  at[n].id = cudaLaunchAttributeClusterDimension;
  at[n].val.clusterDim.x = S;
  at[n].val.clusterDim.y = at[n].val.clusterDim.z = 1;
  ++n;
  if (pdl_enabled()) {
    at[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[n].val.programmaticStreamSerializationAllowed = 1;
    ++n;
  }
  cfg.attrs = at;
  cfg.numAttrs = n;
  SL_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, w[0], w[1], terms, q, a, epilogue));
  return SL_OK;
}

// rows to a pass: what the accumulators of a step's groups leave of the tensor memory, and the sums of two matrices of the registers
template <int G, bool DUAL, bool FP32>
int by_rows(const CUtensorMap* w, void* ws, const GqWs& lay, const GqArgs& a, int epilogue, cudaStream_t st) {
  if (a.max_rows <= 16) return launch_gq<G, 16, DUAL, FP32>(w, ws, lay, a, epilogue, st);
  if (a.max_rows <= 32) return launch_gq<G, 32, DUAL, FP32>(w, ws, lay, a, epilogue, st);
  if (G == 32 || DUAL || a.max_rows <= 64) return launch_gq<G, 64, DUAL, FP32>(w, ws, lay, a, epilogue, st);
  return launch_gq<G, G == 32 || DUAL ? 64 : 128, DUAL, FP32>(w, ws, lay, a, epilogue, st);
}
template <int G>
int by_kind(const CUtensorMap* w, const void* A, void* ws, const GqArgs& a, int epilogue, bool fp32, cudaStream_t st) {
  const GqWs lay = gq_ws(a.max_rows, a.K);
  if (a.max_rows > 65535) return SL_EUNSUPPORTED;
  SL_CUDA_TRY(launch_pdl(gq_split_rows_kernel<G>, dim3((unsigned)((lay.kp / 8 + GS_THREADS - 1) / GS_THREADS), a.max_rows), dim3(GS_THREADS),
                         0, st, (const bf16*)A, a.n_active, a.max_rows, a.K, (int)lay.kp, (int)lay.ld, (uint8_t*)ws,
                         (float2*)((char*)ws + lay.q_at)));
  if (epilogue == EPI_SWIGLU)
    return fp32 ? by_rows<G, true, true>(w, ws, lay, a, epilogue, st) : by_rows<G, true, false>(w, ws, lay, a, epilogue, st);
  return fp32 ? by_rows<G, false, true>(w, ws, lay, a, epilogue, st) : by_rows<G, false, false>(w, ws, lay, a, epilogue, st);
}

}  // namespace

size_t gemm_quantized_workspace_bytes(int max_rows, int K) { return gq_ws(max_rows, K).bytes; }

int launch_gemm_quantized(const void* A, const surelock_w4* W, const surelock_w4* W2, void* C, const int32_t* n_active, int max_rows,
                          int n_out, int K, int epilogue, void* workspace, int32_t* status, cudaStream_t st) {
  GqArgs a{};
  CUtensorMap maps[2];
  const int ng = K / W->group;
  const bool fp32 = W->scale_dtype == SL_FP32;
  a.vec = ng % (fp32 ? 4 : 8) == 0;
  for (int i = 0; i < 2; ++i) {
    const surelock_w4* w = i && W2 ? W2 : W;
    a.zeros[i] = (const uint8_t*)w->zeros;
    a.scales[i] = w->scales;
    if ((reinterpret_cast<uintptr_t>(w->scales) & 15) || (reinterpret_cast<uintptr_t>(w->zeros) & 3)) a.vec = 0;
    const int rc = gq_map(&maps[i], w->codes, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, n_out, K / 2, 128, GQ_BK / 2, CU_TENSOR_MAP_SWIZZLE_128B);
    if (rc != SL_OK) return rc;
  }
  a.C = C;
  a.n_active = n_active;
  a.max_rows = max_rows;
  a.n_out = n_out;
  a.K = K;
  a.ng = ng;
  a.status = status;
  switch (W->group) {
    case 32: return by_kind<32>(maps, A, workspace, a, epilogue, fp32, st);
    case 64: return by_kind<64>(maps, A, workspace, a, epilogue, fp32, st);
    default: return by_kind<128>(maps, A, workspace, a, epilogue, fp32, st);
  }
}

}  // namespace sl
