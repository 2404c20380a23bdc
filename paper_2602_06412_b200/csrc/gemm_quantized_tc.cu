// Products with 4-bit weights for more rows than gemm_quantized.cu takes in one pass: 33 to 128 rows, in passes of 64 or 128.
// Same operands: codes alone in 16 bits are fp16 numbers u 2^-24 or u 2^-20, the rows are rewritten to match, and per group
// the bracket D - z q is formed in fp32 and multiplied by the group's scale (see there for the formulas).
//
// With this many rows the products themselves would bound mma.sync (970 multiply-adds per clock and SM: 22 us for 128 rows of
// 4096 x 12288), so they go to tcgen05: the weights are the 128-row operand, read from TENSOR MEMORY, where one thread per
// feature and quarter of the k puts its codes after unpacking; the rows are the N operand, by TMA.  What bounds it then is
// adding up: every group's accumulator (128 features x rows) is read back and takes two fma per element.
//   warps 0-15  feature 32 (w % 4) + lane; w / 4 = quarter of the step's k for unpacking, of the rows for adding up
//   warp 16     one thread issues the TMA copies: a stage is 256 k of 128 features (with SwiGLU 64 of the gate and the same 64
//               of the up matrix), the rows and their q
//   warp 17     one thread issues the MMAs of a step (128 k)
// A step is unpacked into one of two operand tiles while the MMAs of the step before run; it is handed over before that one is
// added up where tensor memory holds two sets of accumulators, after it otherwise.  K is split over a cluster of up to 8 CTAs
// (sums through distributed shared memory in a fixed order).  All waits are bounded.
#include "gemm_quantized.cuh"

namespace sl {

namespace {

constexpr int GT_WORKERS = 16, GT_THREADS = 32 * (GT_WORKERS + 2);

__device__ __forceinline__ void gt_mma(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc, uint32_t accum) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d_tmem), "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accum)
      : "memory");
}
__device__ __forceinline__ void tc_ld16(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
        "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tc_st16(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}

// Scales and zero points of one feature, group after group: 8 bytes of scales (4 bf16 or 2 fp32) with their zero points at a
// time, the next ones requested one such chunk ahead.
template <bool FP32> struct FeatureGroups {
  static constexpr int CHUNK = FP32 ? 2 : 4;
  const uint8_t *s, *z;        // of the feature; z may be null
  uint32_t c0, c1, n0, n1;     // present and next chunk of scales
  uint32_t cz, nz;             // ... and of zero points
  int grp;

  __device__ __forceinline__ void fetch(int g0, int ng, bool aligned) {
    n0 = n1 = 0;
    nz = 0x08080808u;
    if (aligned) {
      if (g0 < ng) {
        const uint2 x = __ldg(reinterpret_cast<const uint2*>(s + (size_t)g0 * (FP32 ? 4 : 2)));
        n0 = x.x;
        n1 = x.y;
        if (z) nz = FP32 ? (uint32_t)__ldg(reinterpret_cast<const uint16_t*>(z + g0)) : __ldg(reinterpret_cast<const uint32_t*>(z + g0));
      }
      return;
    }
#pragma unroll
    for (int i = 0; i < CHUNK; ++i)
      if (g0 + i < ng) {
        const uint32_t x = FP32 ? __ldg(reinterpret_cast<const uint32_t*>(s) + g0 + i) : __ldg(reinterpret_cast<const uint16_t*>(s) + g0 + i);
        if (FP32) (i ? n1 : n0) = x;
        else (i < 2 ? n0 : n1) |= x << (16 * (i & 1));
        if (z) nz = (nz & ~(0xffu << (8 * i))) | (uint32_t)__ldg(z + g0 + i) << (8 * i);
      }
  }
  __device__ __forceinline__ void turn() {
    c0 = n0;
    c1 = n1;
    cz = nz;
  }
  __device__ __forceinline__ void rotate() {          // drop the first group of the chunk
    if (FP32) {
      c0 = c1;
    } else {
      c0 = __funnelshift_r(c0, c1, 16);
      c1 >>= 16;
    }
    cz >>= 8;
  }
  __device__ __forceinline__ void prime(int ng, bool aligned) {   // before the first next(): the first chunk was requested
    const int at = grp & ~(CHUNK - 1);
    turn();
    fetch(at + CHUNK, ng, aligned);
    for (int i = at; i < grp; ++i) rotate();
  }
  // scale and minus the zero point of the next group (behind the feature's last one anything finite: its D and q are 0)
  __device__ __forceinline__ void next(float& scale, float& minus_z, int ng, bool aligned) {
    scale = __uint_as_float(FP32 ? c0 : c0 << 16);
    minus_z = -(float)(cz & 0xffu);
    if ((++grp & (CHUNK - 1)) == 0) {
      turn();
      fetch(grp + CHUNK, ng, aligned);
    } else {
      rotate();
    }
  }
};

template <int G, int NP> struct GtPlan {
  static constexpr int KS = 128, GPS = KS / G, GPT = GQ_BK / G;   // k and groups of a step, groups of a stage
  static constexpr int SLAB = NP * 128;                       // bytes of 64 k of the rows
  static constexpr int SUMS = GPT * NP * 4;                   // q of a stage
  static constexpr int LOADED = GQ_CODES + 4 * SLAB + SUMS;
  static constexpr int STAGE = GQ_CODES + 4 * SLAB + (SUMS + 1023) / 1024 * 1024;
  static constexpr int STAGES = 220 * 1024 / STAGE > 4 ? 4 : 220 * 1024 / STAGE;
  static constexpr uint32_t A_COLS = KS / 2, D_COL = 2 * A_COLS, D_COLS = GPS * NP;   // two operand tiles, then accumulators
  static constexpr bool TWICE = D_COL + 2 * D_COLS <= 512;    // two sets of accumulators
  static constexpr int PITCH = 128;                           // floats per row of the partial sums
  static constexpr int SMEM = 1024 + STAGES * STAGE + 256;
  static_assert(D_COL + D_COLS <= 512, "tensor memory");
  static_assert(STAGES >= 2 && NP * PITCH * 4 <= STAGES * STAGE, "partial sums take the place of the stages");
};

}  // namespace

template <int G, int NP, bool DUAL, bool FP32>
__global__ void __launch_bounds__(GT_THREADS, 1)
gemm_quantized_tc_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmW2,
                         const __grid_constant__ CUtensorMap tmR, const __grid_constant__ CUtensorMap tmQ, const GqArgs a, const int epilogue) {
  using P = GtPlan<G, NP>;
  constexpr int GPS = P::GPS, HC = NP / 4;                    // HC: rows that a thread adds up
  constexpr int TO = DUAL ? 64 : 128;                         // output features of the CTA
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
      mbar_init(empty(i), 2 * GT_WORKERS + 1);                // readers of the codes, of q (a step later), and the MMAs
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(a_full(i), GT_WORKERS);
      mbar_init(done(i), 1);
    }
    *s_abort = 0;
    fence_mbar_init();
  }
  if (warp == GT_WORKERS + 1) tc_alloc(smem_u32(s_tmem), 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *s_tmem;

  uint32_t S, rank = 0;
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(S));
  if (S > 1) rank = cluster_ctarank();
  const int n0 = (int)(blockIdx.x / S) * TO, r0 = blockIdx.y * NP;
  // *n_active, the weights and C were written before the rewriting kernel began; its rows come after griddep_wait()
  const int M = min(*a.n_active, a.max_rows) - r0;            // rows of this tile; none: the whole cluster leaves
  const int nblk = (a.K + GQ_BK - 1) / GQ_BK;
  const int b0 = (int)((long long)nblk * rank / S), b1 = (int)((long long)nblk * (rank + 1) / S);
  const int stages = M > 0 ? b1 - b0 : 0, steps = 2 * stages;   // 128 k each

  float acc[HC];
#pragma unroll
  for (int c = 0; c < HC; ++c) acc[c] = 0.f;

  if (warp == GT_WORKERS) {
    if (lane == 0) {
      const uint64_t once = gridDim.y > 1 ? l2_policy_evict_normal() : l2_policy_evict_first();   // a code is read once per row tile
      const int ahead = min(stages, P::STAGES);
      auto codes = [&](int i) {
        const int st = i % P::STAGES;
        const uint32_t at = smem_u32(smem + st * P::STAGE);
        mbar_expect_tx(full(st), P::LOADED);
        tma_load_2d_hint(at, &tmW, (b0 + i) * (GQ_BK / 2), n0, full(st), once);
        if (DUAL) tma_load_2d_hint(at + GQ_CODES / 2, &tmW2, (b0 + i) * (GQ_BK / 2), n0, full(st), once);
      };
      for (int i = 0; i < ahead; ++i) codes(i);
      griddep_wait();
      griddep_launch();
      bool ok = true;
      int i = 0;
      for (; i < stages; ++i) {
        const int st = i % P::STAGES;
        if (i >= ahead) {
          if (!(ok = mbar_wait(empty(st), ((i / P::STAGES) & 1) ^ 1, s_abort))) break;
          codes(i);
        }
        const uint32_t at = smem_u32(smem + st * P::STAGE) + GQ_CODES;
#pragma unroll
        for (int k = 0; k < 4; ++k) tma_load_2d(at + k * P::SLAB, &tmR, (b0 + i) * GQ_BK + k * 64, r0, full(st));
        tma_load_2d(at + 4 * P::SLAB, &tmQ, r0, (b0 + i) * P::GPT, full(st));
      }
      if (!ok) {
        // gave up: wait (bounded) for the copies in flight, which write to this CTA's shared memory
        const unsigned long long t0 = clock64();
        for (int k = max(0, i - P::STAGES); k < i; ++k)
          while (!mbar_try(full(k % P::STAGES), (k / P::STAGES) & 1) && clock64() - t0 < TC_WAIT_CYCLES) {}
        set_status(a.status, SL_DEV_GEMM_TIMEOUT);
      }
    }
  } else if (warp == GT_WORKERS + 1) {
    if (lane == 0) {
      constexpr uint32_t idesc = (1u << 4) | ((uint32_t)(NP >> 3) << 17) | (8u << 24);   // fp16 x fp16 -> fp32, M = 128, N = NP
      for (int i = 0; i < steps; ++i) {
        const int sg = i >> 1, st = sg % P::STAGES, part = i & 1;
        if (!mbar_wait(full(st), (sg / P::STAGES) & 1, s_abort) || !mbar_wait(a_full(i), (i >> 1) & 1, s_abort)) {
          set_status(a.status, SL_DEV_GEMM_TIMEOUT);
          const unsigned long long t0 = clock64();            // the last step issued still uses the tensor memory
          while (i > 0 && !mbar_try(done(i - 1), ((i - 1) >> 1) & 1) && clock64() - t0 < TC_WAIT_CYCLES) {}
          break;
        }
        tc_fence_after();
        const uint32_t rows = smem_u32(smem + st * P::STAGE + GQ_CODES) + part * 2 * P::SLAB;
        const uint32_t d = tmem + P::D_COL + (P::TWICE ? (i & 1) * P::D_COLS : 0), op = tmem + (i & 1) * P::A_COLS;
#pragma unroll
        for (int k = 0; k < P::KS / 16; ++k)                  // 16 k: 8 columns of the operand, 32 bytes of a slab's rows
          gt_mma(d + (k / (G / 16)) * NP, op + k * 8, smem_desc_k_sw128(rows + (k >> 2) * P::SLAB + (k & 3) * 32), idesc, k % (G / 16) != 0);
        if (part == 1) tc_commit(empty(st));
        tc_commit(done(i));
      }
    }
  } else {
    const int feature = (warp & 3) * 32 + lane, quarter = warp >> 2;
    const uint32_t lanes = (uint32_t)(warp & 3) << 21;        // this warp's lanes of the tensor memory
    const bool aligned = a.pairs != 0;
    FeatureGroups<FP32> rd;
    {
      const int m = DUAL ? feature >> 6 : 0;                  // with SwiGLU the first 64 are the gate's, the others the up matrix's
      const long long f = (long long)min(n0 + (DUAL ? feature & 63 : feature), a.n_out - 1) * a.ng;   // behind the last feature: any scales, codes are 0
      rd.s = (const uint8_t*)a.scales[m] + f * (FP32 ? 4 : 2);
      rd.z = a.zeros[m] ? a.zeros[m] + f : nullptr;
      rd.grp = b0 * P::GPT;
      if (stages > 0) rd.fetch(rd.grp & ~(FeatureGroups<FP32>::CHUNK - 1), a.ng, aligned);
    }
    bool ok = true;
    // the codes of step i, half `part` of its stage -> operand tile i & 1
    auto unpack = [&](int i, const int part) {
      const int sg = i >> 1, st = sg % P::STAGES;
      if (part == 0) ok = __all_sync(0xffffffffu, mbar_wait(full(st), (sg / P::STAGES) & 1, s_abort));
      if (!ok) return;
      const uint32_t chunk = part * 4 + quarter;              // of the 128-byte row, swizzled
      const uint4 v = gq_lds128(smem_u32(smem + st * P::STAGE) + feature * 128 + ((chunk ^ (lane & 7)) << 4));
      const uint32_t w[4] = {v.x, v.y, v.z, v.w};
      uint32_t x[16];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t hi = w[j] >> 8;
        x[4 * j] = w[j] & 0x000f000fu;
        x[4 * j + 1] = w[j] & 0x00f000f0u;
        x[4 * j + 2] = hi & 0x000f000fu;
        x[4 * j + 3] = hi & 0x00f000f0u;
      }
      tc_st16(tmem + lanes + (i & 1) * P::A_COLS + quarter * 16, x);
      if (part == 1) {
        __syncwarp();
        if (lane == 0) mbar_arrive(empty(st));
      }
    };
    // add up step i
    auto add = [&](int i, const int part) {
      const int st = (i >> 1) % P::STAGES;
      if (i == 0) rd.prime(a.ng, aligned);
      ok = __all_sync(0xffffffffu, mbar_wait(done(i), (i >> 1) & 1, s_abort));
      if (!ok) return;
      tc_fence_after();
      const float4* sq = reinterpret_cast<const float4*>(smem + st * P::STAGE + GQ_CODES + 4 * P::SLAB) + part * GPS * (NP / 4) + quarter * (HC / 4);
      const uint32_t d0 = tmem + lanes + P::D_COL + (P::TWICE ? (i & 1) * P::D_COLS : 0) + quarter * HC;
#pragma unroll
      for (int g = 0; g < GPS; ++g) {
        float sc, mz;
        rd.next(sc, mz, a.ng, aligned);
#pragma unroll
        for (int c = 0; c < HC; c += 16) {
          uint32_t d[16];
          tc_ld16(d0 + g * NP + c, d);
          tc_wait_ld();
#pragma unroll
          for (int e = 0; e < 16; e += 4) {
            const float4 q = sq[g * (NP / 4) + (c + e) / 4];
            float* x = &acc[c + e];
            x[0] = fmaf(sc, fmaf(mz, q.x, __uint_as_float(d[e])), x[0]);
            x[1] = fmaf(sc, fmaf(mz, q.y, __uint_as_float(d[e + 1])), x[1]);
            x[2] = fmaf(sc, fmaf(mz, q.z, __uint_as_float(d[e + 2])), x[2]);
            x[3] = fmaf(sc, fmaf(mz, q.w, __uint_as_float(d[e + 3])), x[3]);
          }
        }
      }
      if (part == 1) {
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
    for (int sg = 0; sg < stages && ok; ++sg) {
#pragma unroll
      for (int part = 0; part < 2; ++part) {
        const int i = sg * 2 + part;
        unpack(i, part);
        if (!ok) break;
        if (P::TWICE) release(i);
        if (i > 0) add(i - 1, part ^ 1);
        if (!ok) break;
        if (!P::TWICE) release(i);
      }
    }
    if (stages > 0 && ok) add(steps - 1, 1);
    if (!ok && lane == 0) set_status(a.status, SL_DEV_GEMM_TIMEOUT);
  }

  // ---- sums of the cluster, epilogue ----
  tc_fence_before();
  __syncthreads();
  const bool good = *s_abort == 0;
  if (warp == GT_WORKERS + 1) {
    __syncwarp();
    tc_fence_after();
    tc_dealloc(tmem, 512);
  }
  if (warp < GT_WORKERS) {
    const int feature = (warp & 3) * 32 + lane, quarter = warp >> 2;
#pragma unroll
    for (int c = 0; c < HC; ++c) sRed[(quarter * HC + c) * P::PITCH + feature] = acc[c];
  }
  if (S > 1) cluster_sync_all(); else __syncthreads();
  if (M > 0 && good) {
    const int c0 = (int)(TO / 4 * rank / S), cols = (int)(TO / 4 * (rank + 1) / S) - c0;   // features in fours that this CTA finishes
    for (int i = threadIdx.x; i < min(M, NP) * cols; i += GT_THREADS) {
      const int r = i / cols, col = 4 * (c0 + i % cols);
      if (n0 + col >= a.n_out) continue;
      const float4 y = gq_total(sRed, S, r * P::PITCH + col);
      gq_store<DUAL>(a, epilogue, r0 + r, n0 + col, y, DUAL ? gq_total(sRed, S, r * P::PITCH + 64 + col) : y);
    }
  }
  if (S > 1) cluster_sync_all();                              // the others may still be reading this CTA's partial sums
}

namespace {

template <int G, int NP, bool DUAL, bool FP32>
int launch_gt(const CUtensorMap* w, const GqArgs& a, const float* q, int ld, int epilogue, cudaStream_t st) {
  using P = GtPlan<G, NP>;
  constexpr int TO = DUAL ? 64 : 128;
  const int nblk = (a.K + GQ_BK - 1) / GQ_BK;
  CUtensorMap rows, sums;
  int rc = gq_map(&rows, a.rows, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, a.max_rows, (long long)nblk * GQ_BK, NP, 64);
  if (rc == SL_OK) rc = gq_map(&sums, q, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 4, (long long)nblk * P::GPT, ld, P::GPT, NP);
  if (rc != SL_OK) return rc;
  // the split of K with the least estimated time: rounds of CTAs (one per SM) times (stages of one + two stages' time to start and join)
  const long long work = (long long)((a.n_out + TO - 1) / TO) * ((a.max_rows + NP - 1) / NP);
  int S = 1;
  long long best = 0;
  for (int s = 1; s <= 8 && s <= nblk; ++s) {
    const long long t = ((work * s + sm_count() - 1) / sm_count()) * ((nblk + s - 1) / s + 2);
    if (s == 1 || t < best) {
      best = t;
      S = s;
    }
  }
  auto kernel = gemm_quantized_tc_kernel<G, NP, DUAL, FP32>;
  static std::once_flag once;
  static cudaError_t attr;
  std::call_once(once, [&] { attr = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, P::SMEM); });
  SL_CUDA_TRY(attr);
  const dim3 grid((a.n_out + TO - 1) / TO * S, (a.max_rows + NP - 1) / NP);
  SL_CUDA_TRY(gq_launch(kernel, grid, GT_THREADS, P::SMEM, S, st, w[0], w[1], rows, sums, a, epilogue));
  return SL_OK;
}

// rows to a pass: with groups of 32 the accumulators of a step leave room for 64
template <int G, bool DUAL, bool FP32>
int tc_rows(const CUtensorMap* w, const GqArgs& a, const float* q, int ld, int epilogue, cudaStream_t st) {
  if (G == 32 || a.max_rows <= 64) return launch_gt<G, 64, DUAL, FP32>(w, a, q, ld, epilogue, st);
  return launch_gt<G, G == 32 ? 64 : 128, DUAL, FP32>(w, a, q, ld, epilogue, st);
}
template <int G> int tc_kind(const CUtensorMap* w, const GqArgs& a, const float* q, int ld, bool fp32, int epilogue, cudaStream_t st) {
  if (epilogue == EPI_SWIGLU) return fp32 ? tc_rows<G, true, true>(w, a, q, ld, epilogue, st) : tc_rows<G, true, false>(w, a, q, ld, epilogue, st);
  return fp32 ? tc_rows<G, false, true>(w, a, q, ld, epilogue, st) : tc_rows<G, false, false>(w, a, q, ld, epilogue, st);
}

}  // namespace

int launch_gemm_quantized_tc(const CUtensorMap* w, const GqArgs& a, const float* q, int ld, int group, bool fp32, int epilogue, cudaStream_t st) {
  switch (group) {
    case 32: return tc_kind<32>(w, a, q, ld, fp32, epilogue, st);
    case 64: return tc_kind<64>(w, a, q, ld, fp32, epilogue, st);
    default: return tc_kind<128>(w, a, q, ld, fp32, epilogue, st);
  }
}

}  // namespace sl
