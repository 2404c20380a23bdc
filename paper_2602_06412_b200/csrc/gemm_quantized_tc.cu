// Products with 4-bit weights for more rows than the kernel in gemm_quantized.cu takes (the rule is there), in passes of 64 or 128.
// Same operands: codes alone in 16 bits are fp16 numbers u 2^-24 or u 2^-20, the rows are rewritten to match, and every group's
// sum of products is multiplied by its scale in fp32 (see there for the formulas).
//
// With this many rows the products themselves would bound mma.sync (970 multiply-adds per clock and SM: 22 us for 128 rows of
// 4096 x 12288), so they go to tcgen05: the weights are the 128-row operand, read from TENSOR MEMORY, where one thread per
// feature puts its codes after unpacking, less their zero points (u - z is exact in fp16 as u is, so there is no q here: a
// multiply-add less per element and group); the rows are the N operand, by TMA.  Every group's accumulator (128 features x
// rows) is read back and takes one multiply-add per element.  What bounds it: the chain unpack -> product -> add, some 1200
// clocks per 128 k, each satisfied wait of it 100 - 150; at 128 rows also the rows that every CTA reads from L2 (9 TB/s).
// Measured in replayed graphs: 4096 x 12288 in groups of 64, 128 rows 29 us, 64 rows 22 us; 4096 x 4096 13 and 11 us; gate and up 12288 x 4096 with
// SwiGLU 50 and 43 us; 126464 x 4096 163 and 136 us.
//   warps 0-15  add up: feature 32 (w % 4) + lane, w / 4 = quarter of the rows
//   4 or 8      unpack: feature 32 (w % 4) + lane (16 warps that did both: 192 against 166 us, 128 rows of the 4096 x 126464
//               head: a step's chain of waits was twice as long)
//   1           one thread issues the TMA copies: codes in stages of 256 k of 128 features (with SwiGLU 64 of the gate and the
//               same 64 of the up matrix), rows in stages of a step
//   2           issue the MMAs of a step (128 k), group by group, each of every other step
// A step is unpacked into one of two operand tiles while the MMAs of the step before run, and that one is added up while its
// own run: tensor memory holds 3 (128 rows) or 6 (64 rows) groups' accumulators.  K is split over a cluster of up to 8 CTAs
// (sums through distributed shared memory in a fixed order).  All waits are bounded.
#include "gemm_quantized.cuh"

namespace sl {

namespace {

constexpr int GT_ADDERS = 16;          // warps

__device__ __forceinline__ void gt_mma(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc, uint32_t accum) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d_tmem), "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accum)
      : "memory");
}
// true in one lane of the (whole) warp
__device__ __forceinline__ bool elect_one() {
  uint32_t yes;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(yes));
  return yes != 0;
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

// acc[0..1] += s d[0..1], two products to an instruction
__device__ __forceinline__ void fma2(float* acc, float s, const uint32_t* d) {
  asm("{\n\t.reg .b64 a, b, c;\n\t"
      "mov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %4};\n\tmov.b64 c, {%0, %1};\n\t"
      "fma.rn.f32x2 c, a, b, c;\n\tmov.b64 {%0, %1}, c;\n\t}"
      : "+f"(acc[0]), "+f"(acc[1]) : "f"(__uint_as_float(d[0])), "f"(__uint_as_float(d[1])), "f"(s));
}

// Scales of one feature, a stage's groups at a time; the next stage's are requested when one begins.
template <int G, bool FP32> struct FeatureScales {
  static constexpr int GPT = GQ_BK / G, WORDS = GPT * (FP32 ? 4 : 2) / 4;
  const uint8_t* s;            // of the feature
  uint32_t c[WORDS], n[WORDS];

  __device__ __forceinline__ void fetch(int g0, int ng, bool aligned) {   // groups from g0 on -> n
#pragma unroll
    for (int i = 0; i < WORDS; ++i) n[i] = 0;
    if (aligned) {
      if (g0 < ng) {
        const uint8_t* p = s + (size_t)g0 * (FP32 ? 4 : 2);
#pragma unroll
        for (int i = 0; i < WORDS; i += 4) {
          if (WORDS == 1) {
            n[0] = __ldg(reinterpret_cast<const uint32_t*>(p));
          } else if (WORDS == 2) {
            const uint2 x = __ldg(reinterpret_cast<const uint2*>(p));
            n[0] = x.x; n[1 % WORDS] = x.y;
          } else {
            const uint4 x = __ldg(reinterpret_cast<const uint4*>(p) + i / 4);
            n[i] = x.x; n[(i + 1) % WORDS] = x.y; n[(i + 2) % WORDS] = x.z; n[(i + 3) % WORDS] = x.w;
          }
        }
      }
      return;
    }
#pragma unroll
    for (int i = 0; i < GPT; ++i)
      if (g0 + i < ng) {
        if (FP32) n[i % WORDS] = __ldg(reinterpret_cast<const uint32_t*>(s) + g0 + i);
        else n[i / 2 % WORDS] |= (uint32_t)__ldg(reinterpret_cast<const uint16_t*>(s) + g0 + i) << (16 * (i & 1));
      }
  }
  __device__ __forceinline__ void turn() {
#pragma unroll
    for (int i = 0; i < WORDS; ++i) c[i] = n[i];
  }
  __device__ __forceinline__ float get(int i) const {   // behind the feature's last group 0
    return __uint_as_float(FP32 ? c[i % WORDS] : i & 1 ? c[i / 2 % WORDS] & 0xffff0000u : c[i / 2 % WORDS] << 16);
  }
};

// Zero points of one feature likewise, packed; behind the feature's last group anything (the rows are 0 there)
template <int G> struct FeatureZeros {
  static constexpr int GPT = GQ_BK / G;
  const uint8_t* z;            // of the feature, or null
  uint32_t c[2], n[2];

  __device__ __forceinline__ void fetch(int g0, int ng, bool aligned) {
    n[0] = n[1] = 0x08080808u;
    if (!z) return;
    if (aligned) {
      if (g0 < ng) {
        if (GPT == 2) {
          n[0] = __ldg(reinterpret_cast<const uint16_t*>(z + g0));
        } else if (GPT == 4) {
          n[0] = __ldg(reinterpret_cast<const uint32_t*>(z + g0));
        } else {
          const uint2 x = __ldg(reinterpret_cast<const uint2*>(z + g0));
          n[0] = x.x; n[1] = x.y;
        }
      }
      return;
    }
    n[0] = n[1] = 0;
#pragma unroll
    for (int i = 0; i < GPT; ++i)
      if (g0 + i < ng) n[i / 4] |= (uint32_t)__ldg(z + g0 + i) << (8 * (i & 3));
  }
  __device__ __forceinline__ void turn() {
    c[0] = n[0];
    c[1] = n[1];
  }
  __device__ __forceinline__ uint32_t get(int i) const { return c[i / 4] >> (8 * (i & 3)) & 0xffu; }
};

template <int G, int NP> struct GtPlan {
  // warps: unpacking in teams of four, that take steps in turn (a second team at 128 rows would leave 72 registers to a thread,
  // which then spills: 203 against 166 us)
  static constexpr int TEAMS = NP == 128 ? 1 : 2, COPY = GT_ADDERS + 4 * TEAMS, MMA = COPY + 1, THREADS = 32 * (MMA + 2);
  static constexpr int KS = 128, GPS = KS / G, GPT = GQ_BK / G;   // k and groups of a step, groups of a stage
  static constexpr int SLAB = NP * 128;                       // bytes of 64 k of the rows
  static constexpr int CODES = NP == 128 ? 3 : 4, ROWS = NP == 128 ? 5 : 8;   // stages of codes (two steps each) and of rows (a step)
  static constexpr uint32_t A_COLS = KS / 2, D_COL = 2 * A_COLS;   // tensor memory: two operand tiles, then accumulators of a group
  static constexpr int SETS = (512 - D_COL) / NP;
  static constexpr int PITCH = 128;                           // floats per row of the partial sums
  static constexpr int BUFFERS = CODES * GQ_CODES + ROWS * 2 * SLAB, BARS = 2 * CODES + 2 * ROWS + 2 + 2 * SETS;
  static constexpr int SMEM = 1024 + BUFFERS + 384;
  static_assert(SETS > GPS, "the first group of a step must not wait for the last step's adding up");
  static_assert(NP * PITCH * 4 <= BUFFERS && BARS * 8 + 8 <= 384 && SMEM <= 227 * 1024, "shared memory");
};

}  // namespace

template <int G, int NP, bool DUAL, bool FP32>
__global__ void __launch_bounds__(GtPlan<G, NP>::THREADS, 1)
gemm_quantized_tc_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmW2, const __grid_constant__ CUtensorMap tmR,
                         const GqArgs a, const int epilogue) {
  using P = GtPlan<G, NP>;
  constexpr int GPS = P::GPS, HC = NP / 4;                    // HC: rows that a thread adds up
  constexpr int TO = DUAL ? 64 : 128;                         // output features of the CTA
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  float* sRed = reinterpret_cast<float*>(smem);               // [NP][PITCH] after the last step
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + P::BUFFERS);
  const uint32_t codes0 = smem_u32(smem), rows0 = codes0 + P::CODES * GQ_CODES, bar0 = smem_u32(bars);
  // barriers: of stage s of codes, step i, set of accumulators
  auto c_full = [&](int s) { return bar0 + 8u * (s % P::CODES); };
  auto c_empty = [&](int s) { return bar0 + 8u * (P::CODES + s % P::CODES); };
  auto r_full = [&](int i) { return bar0 + 8u * (2 * P::CODES + i % P::ROWS); };
  auto r_empty = [&](int i) { return bar0 + 8u * (2 * P::CODES + P::ROWS + i % P::ROWS); };
  auto unpacked = [&](int i) { return bar0 + 8u * (2 * P::CODES + 2 * P::ROWS + (i & 1)); };            // operand tile written
  auto done = [&](int set) { return bar0 + 8u * (2 * P::CODES + 2 * P::ROWS + 2 + set); };              // MMAs finished
  auto added = [&](int set) { return bar0 + 8u * (2 * P::CODES + 2 * P::ROWS + 2 + P::SETS + set); };
  uint32_t* s_tmem = reinterpret_cast<uint32_t*>(bars + P::BARS);
  volatile int* s_abort = reinterpret_cast<volatile int*>(s_tmem + 1);

  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < P::CODES; ++i) {
      mbar_init(c_full(i), 1);
      mbar_init(c_empty(i), 4 * P::TEAMS);
    }
    for (int i = 0; i < P::ROWS; ++i) {
      mbar_init(r_full(i), 1);
      mbar_init(r_empty(i), 1);
    }
    for (int i = 0; i < 2; ++i) mbar_init(unpacked(i), 4);
    for (int i = 0; i < P::SETS; ++i) {
      mbar_init(done(i), 1);
      mbar_init(added(i), GT_ADDERS);
    }
    *s_abort = 0;
    fence_mbar_init();
  }
  if (warp == P::MMA) tc_alloc(smem_u32(s_tmem), 512);
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

  if (warp == P::COPY) {
    if (lane == 0) {
      const uint64_t once = gridDim.y > 1 ? l2_policy_evict_normal() : l2_policy_evict_first();   // a code is read once per row tile
      const int ahead = min(stages, P::CODES);
      auto codes = [&](int s) {
        const uint32_t at = codes0 + s % P::CODES * GQ_CODES;
        mbar_expect_tx(c_full(s), GQ_CODES + (s == 0 && blockIdx.x + blockIdx.y == 0 ? a.lost : 0));
        tma_load_2d_hint(at, &tmW, (b0 + s) * (GQ_BK / 2), n0, c_full(s), once);
        if (DUAL) tma_load_2d_hint(at + GQ_CODES / 2, &tmW2, (b0 + s) * (GQ_BK / 2), n0, c_full(s), once);
      };
      for (int s = 0; s < ahead; ++s) codes(s);
      griddep_wait();
      griddep_launch();
      bool ok = true;
      int i = 0, asked = ahead;                               // steps of rows and stages of codes that were requested
      for (; i < steps; ++i) {
        if (!(i & 1) && (i >> 1) >= ahead) {
          const int s = i >> 1;
          if (!(ok = mbar_wait(c_empty(s), ((s / P::CODES) & 1) ^ 1, s_abort))) break;
          codes(s);
          ++asked;
        }
        if (!(ok = mbar_wait(r_empty(i), ((i / P::ROWS) & 1) ^ 1, s_abort))) break;
        const uint32_t at = rows0 + i % P::ROWS * 2 * P::SLAB;
        mbar_expect_tx(r_full(i), 2 * P::SLAB);
#pragma unroll
        for (int k = 0; k < 2; ++k) tma_load_2d(at + k * P::SLAB, &tmR, b0 * GQ_BK + i * P::KS + k * 64, r0, r_full(i));
      }
      // The copies in flight still write to this CTA's shared memory: they have landed (a bounded wait) before this thread goes
      // on, whichever warp's wait may have run out.
      const unsigned long long t0 = clock64();
      for (int k = max(0, asked - P::CODES); k < asked; ++k)
        while (!mbar_try(c_full(k), (k / P::CODES) & 1) && clock64() - t0 < TC_WAIT_CYCLES) {}
      for (int k = max(0, i - P::ROWS); k < i; ++k)
        while (!mbar_try(r_full(k), (k / P::ROWS) & 1) && clock64() - t0 < TC_WAIT_CYCLES) {}
      if (!ok) set_status(a.status, SL_DEV_GEMM_TIMEOUT);
    }
  } else if (warp >= P::MMA) {
    // Two warps take turns, as the waits before a step's first MMA take as long as issuing its MMAs.  A warp stays together and
    // elects a lane per group: in a branch of one lane every operand of an MMA would first have to be moved to the uniform
    // registers that it is issued from (170 clocks per MMA).
    constexpr uint32_t idesc = (1u << 4) | ((uint32_t)(NP >> 3) << 17) | (8u << 24);   // fp16 x fp16 -> fp32, M = 128, N = NP
    const uint32_t base = __shfl_sync(0xffffffffu, tmem, 0), ring = __shfl_sync(0xffffffffu, rows0, 0), bars0 = __shfl_sync(0xffffffffu, bar0, 0);
    const int n_steps = __shfl_sync(0xffffffffu, steps, 0);
    auto bar = [&](int i) { return bars0 + 8u * i; };
    constexpr int R_FULL = 2 * P::CODES, R_EMPTY = R_FULL + P::ROWS, UNPACKED = R_EMPTY + P::ROWS, DONE = UNPACKED + 2, ADDED = DONE + P::SETS;
    bool ok = true;
    const int first = warp - P::MMA;                          // of this warp's steps, every other one
    int set = first * GPS, last = -1, slot = first;           // set of the group at hand, of the last one issued; stage of rows
    uint32_t phase = 0, last_phase = 0, rphase = 0;
    for (int i = first; i < n_steps && ok; i += 2) {
      const uint32_t rows = ring + slot * 2 * P::SLAB, op = base + first * P::A_COLS;
      ok = mbar_wait(bar(R_FULL + slot), rphase, s_abort) && mbar_wait(bar(UNPACKED + first), (i >> 1) & 1, s_abort);
#pragma unroll
      for (int q = 0; q < GPS; ++q) {
        ok = __all_sync(0xffffffffu, ok && mbar_wait(bar(ADDED + set), phase ^ 1, s_abort));
        if (!ok) break;
        tc_fence_after();
        const uint32_t d = base + P::D_COL + set * NP;
        if (elect_one()) {
#pragma unroll
          for (int k = q * (G / 16); k < (q + 1) * (G / 16); ++k)   // 16 k: 8 columns of the operand, 32 bytes of a slab's rows
            gt_mma(d, op + k * 8, smem_desc_k_sw128(rows + (k >> 2) * P::SLAB + (k & 3) * 32), idesc, k % (G / 16) != 0);
          tc_commit(bar(DONE + set));
          if (q == GPS - 1) tc_commit(bar(R_EMPTY + slot));
        }
        __syncwarp();
        last = set;
        last_phase = phase;
        set += q == GPS - 1 ? GPS + 1 : 1;                    // past the other warp's step
        if (set >= P::SETS) {
          set -= P::SETS;
          phase ^= 1;
        }
      }
      slot += 2;
      if (slot >= P::ROWS) {
        slot -= P::ROWS;
        rphase ^= 1;
      }
    }
    // The tensor memory is freed behind the barrier below: this warp's MMAs, which end in order, are through with it (a bounded
    // wait), whichever warp's wait may have run out.  When both warps finish, at most GPS groups, of the other warp, were issued
    // after its last one, on other accumulators (SETS > GPS), so that group's barrier has not gone on a phase; after a wait that ran
    // out it may have, and then this one runs to its limit.
    if (lane == 0) {
      if (!ok) set_status(a.status, SL_DEV_GEMM_TIMEOUT);
      const unsigned long long t0 = clock64();
      while (last >= 0 && !mbar_try(done(last), last_phase) && clock64() - t0 < TC_WAIT_CYCLES) {}
    }
  } else {
    const int feature = (warp & 3) * 32 + lane;
    const uint32_t lanes = (uint32_t)(warp & 3) << 21;        // this warp's lanes of the tensor memory
    const bool aligned = a.pairs != 0;
    const int m = DUAL ? feature >> 6 : 0;                    // with SwiGLU the first 64 are the gate's, the others the up matrix's
    const long long f = (long long)min(n0 + (DUAL ? feature & 63 : feature), a.n_out - 1) * a.ng;   // behind the last feature any will do
    bool ok = true;
    if (warp >= GT_ADDERS) {
      FeatureZeros<G> rd;
      rd.z = m ? a.zeros[1] : a.zeros[0];
      if (rd.z) rd.z += f;
      if (stages > 0) rd.fetch(b0 * P::GPT, a.ng, aligned);
      for (int i = (warp - GT_ADDERS) / 4; i < steps; i += P::TEAMS) {
        const int sg = i >> 1, part = i & 1;
        if (P::TEAMS == 2 || part == 0) {
          rd.turn();
          if (sg + 1 < stages) rd.fetch((b0 + sg + 1) * P::GPT, a.ng, aligned);
          ok = __all_sync(0xffffffffu, mbar_wait(c_full(sg), (sg / P::CODES) & 1, s_abort));
        }
        if (part) rd.c[0] = P::GPS == 4 ? rd.c[1] : rd.c[0] >> (8 * P::GPS % 32);
        // the operand tile is free when the MMAs of step i - 2 are finished
        if (ok && i >= 2) ok = __all_sync(0xffffffffu, mbar_wait(r_empty(i - 2), ((i - 2) / P::ROWS) & 1, s_abort));
        if (!ok) break;
        const uint32_t from = codes0 + sg % P::CODES * GQ_CODES + feature * 128, to = tmem + lanes + part * P::A_COLS;
#pragma unroll
        for (int q = 0; q < 4; ++q) {                         // 32 k: the codes minus their zero points, exact in fp16
          const uint4 v = gq_lds128(from + (((part * 4 + q) ^ (lane & 7)) << 4));   // of the 128-byte row, swizzled
          const uint32_t w[4] = {v.x, v.y, v.z, v.w};
          const uint32_t zl = rd.get(q * P::GPS / 4) * 0x00010001u, zh = zl << 4;   // like the codes: z 2^-24 and z 2^-20
          auto minus = [](uint32_t x, uint32_t z) {
            const __half2 d = __hsub2(*reinterpret_cast<__half2*>(&x), *reinterpret_cast<__half2*>(&z));
            return *reinterpret_cast<const uint32_t*>(&d);
          };
          uint32_t x[16];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint32_t hi = w[j] >> 8;
            x[4 * j] = minus(w[j] & 0x000f000fu, zl);
            x[4 * j + 1] = minus(w[j] & 0x00f000f0u, zh);
            x[4 * j + 2] = minus(hi & 0x000f000fu, zl);
            x[4 * j + 3] = minus(hi & 0x00f000f0u, zh);
          }
          tc_st16(to + q * 16, x);
        }
        tc_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(unpacked(i));
          if (P::TEAMS == 2 || part == 1) mbar_arrive(c_empty(sg));
        }
      }
    } else {
      const int quarter = warp >> 2;                          // of the rows
      FeatureScales<G, FP32> rd;
      rd.s = (const uint8_t*)(m ? a.scales[1] : a.scales[0]) + f * (FP32 ? 4 : 2);
      if (stages > 0) rd.fetch(b0 * P::GPT, a.ng, aligned);
      int set = 0;
      uint32_t phase = 0;
      for (int sg = 0; sg < stages && ok; ++sg) {
        rd.turn();
        if (sg + 1 < stages) rd.fetch((b0 + sg + 1) * P::GPT, a.ng, aligned);
#pragma unroll
        for (int q = 0; q < P::GPT; ++q) {
          ok = __all_sync(0xffffffffu, mbar_wait(done(set), phase, s_abort));
          if (!ok) break;
          tc_fence_after();
          uint32_t d[HC];
#pragma unroll
          for (int c = 0; c < HC; c += 16) tc_ld16(tmem + lanes + P::D_COL + set * NP + quarter * HC + c, d + c);
          tc_wait_ld();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(added(set));
          if (++set == P::SETS) {
            set = 0;
            phase ^= 1;
          }
          const float sc = rd.get(q);
#pragma unroll
          for (int c = 0; c < HC; c += 2) fma2(acc + c, sc, d + c);
        }
      }
    }
    if (!ok && lane == 0) set_status(a.status, SL_DEV_GEMM_TIMEOUT);
  }

  // ---- sums of the cluster, epilogue ----
  tc_fence_before();
  __syncthreads();
  const bool good = *s_abort == 0;
  if (warp == P::MMA) {
    __syncwarp();
    tc_fence_after();
    tc_dealloc(tmem, 512);
  }
  if (warp < GT_ADDERS) {
    const int feature = (warp & 3) * 32 + lane, quarter = warp >> 2;
    if (!good) {                                              // an incomplete sum is NaN, for whichever CTA adds it
#pragma unroll
      for (int c = 0; c < HC; ++c) acc[c] = __uint_as_float(0x7fffffffu);
    }
#pragma unroll
    for (int c = 0; c < HC; ++c) sRed[(quarter * HC + c) * P::PITCH + feature] = acc[c];
  }
  if (S > 1) cluster_sync_all(); else __syncthreads();
  if (M > 0) {
    const int c0 = (int)(TO / 4 * rank / S), cols = (int)(TO / 4 * (rank + 1) / S) - c0;   // features in fours that this CTA finishes
    for (int i = threadIdx.x; i < min(M, NP) * cols; i += P::THREADS) {
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
int launch_gt(const CUtensorMap* w, const GqArgs& a, int epilogue, cudaStream_t st) {
  using P = GtPlan<G, NP>;
  constexpr int TO = DUAL ? 64 : 128;
  const int tiles = (a.n_out - 1) / TO + 1, nblk = (a.K - 1) / GQ_BK + 1;
  CUtensorMap rows;
  const int rc = gq_map(&rows, a.rows, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, a.max_rows, (long long)nblk * GQ_BK, NP, 64);
  if (rc != SL_OK) return rc;
  // the split of K with the least estimated time: rounds of CTAs (one per SM) times (stages of one + two stages' time to start and join)
  const long long work = (long long)tiles * ((a.max_rows + NP - 1) / NP);
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
  static std::atomic<uint64_t> allowed{0};
  SL_CUDA_TRY(allow_smem(kernel, P::SMEM, allowed));
  const dim3 grid(tiles * S, (a.max_rows + NP - 1) / NP);
  SL_CUDA_TRY(gq_launch(kernel, grid, P::THREADS, P::SMEM, S, st, w[0], w[1], rows, a, epilogue));
  return SL_OK;
}

// rows to a pass: with groups of 32 the accumulators of a step (four sets) leave room for 64
template <int G, bool DUAL, bool FP32>
int tc_rows(const CUtensorMap* w, const GqArgs& a, int epilogue, cudaStream_t st) {
  if constexpr (G != 32)
    if (a.max_rows > 64) return launch_gt<G, 128, DUAL, FP32>(w, a, epilogue, st);
  return launch_gt<G, 64, DUAL, FP32>(w, a, epilogue, st);
}
template <int G> int tc_kind(const CUtensorMap* w, const GqArgs& a, bool fp32, int epilogue, cudaStream_t st) {
  if (epilogue == EPI_SWIGLU) return fp32 ? tc_rows<G, true, true>(w, a, epilogue, st) : tc_rows<G, true, false>(w, a, epilogue, st);
  return fp32 ? tc_rows<G, false, true>(w, a, epilogue, st) : tc_rows<G, false, false>(w, a, epilogue, st);
}

}  // namespace

int launch_gemm_quantized_tc(const CUtensorMap* w, const GqArgs& a, int group, bool fp32, int epilogue, cudaStream_t st) {
  switch (group) {
    case 32: return tc_kind<32>(w, a, fp32, epilogue, st);
    case 64: return tc_kind<64>(w, a, fp32, epilogue, st);
    default: return tc_kind<128>(w, a, fp32, epilogue, st);
  }
}

}  // namespace sl
