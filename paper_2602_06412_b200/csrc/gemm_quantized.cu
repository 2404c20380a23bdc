// Products of a few packed rows with 4-bit weights (the projections of Algorithm 1 lines 10, 12, 15 for weights held in
// four bits):
//
//   C[r][n] = sum_k A[r][k] W[n][k],   W[n][k] = (u[n][k] - z[n][k / g]) * s[n][k / g],   u = 0 ... 15
//
// with the epilogues of surelock_gemm_fused.  What bounds it with few rows: the weights, K / 2 bytes per output feature and
// their scales, are streamed once; the instructions that make operands of the codes come next, 46 codes per clock and SM at
// the memory's rate.
//
// A 4-bit code alone in 16 bits IS an fp16 number: u 2^-24 (subnormal) in the lowest bits, u 2^-20 four bits up.  So eight
// codes become operands of 16-bit matrix instructions with four masks and one shift, (0,4) (1,5) of the word and (2,6) (3,7)
// of the word shifted by 8 (11 instructions to make bf16 numbers of them); the factor 16 between the pairs is taken out of the
// activations, which a small kernel in front rewrites once: a row as fp16 numbers a' = a 2^-e, the largest magnitude 2^14 ...
// 2^15, every other pair over 16.  fp16 has 11 bits to bf16's 8, so this is exact down to 2^-25 of the row's largest
// magnitude and off by at most 2^-35 of it below.  Per group
//   sum_k (u - z) a = 2^(e + 24) (D - z q),   D = sum_k (u 2^-24) a',   q = 2^-24 sum_k a',
// D from the products, q and e from the rewriting kernel; the bracket is formed in fp32 and multiplied by its group's scale
// in fp32, so a weight is never rounded.
//
// mma.sync m16n8k16 with 16 features as the rows and 8 packed rows as the columns: 970 multiply-adds per clock and SM
// measured, enough for some 20 rows at the memory's rate.  Warps work alone, each on its features, and many of them hide each
// other's steps.  (tcgen05 with the codes as the tensor-memory operand was built with bf16 and with e4m3 operands: unpack ->
// tensor memory -> product -> back per group is a chain of ~1000 clocks per 256 k that 16 warps per SM did not hide: 84 - 116
// us for 8 rows of the 4096 x 126464 head.  mma.sync with e4m3 operands converts them to fp16 on the way: 77 us.)
//   warps 0-7  16 features each (with SwiGLU half of the warps have the gate, half the up matrix), all k of the CTA's range
//   warp 8     one thread issues the copies: a stage is 256 k, 128 bytes of codes of 128 features by TMA (128-byte swizzle)
//              and the rewritten rows, already in the order of the MMA fragments, as one bulk copy
// The contraction index is permuted within 32 ... 128 k (a lane owns 16, 8 or 4 code bytes of a feature, for groups of 128,
// 64, 32), and the features within 8 (by bit reversal), so that the code loads touch all banks.
// The first codes are requested before the rewriting kernel has finished: it does not write them.  K is split over the CTAs
// of a cluster when the features alone do not fill the GPU; the sums meet through distributed shared memory in a fixed
// order: deterministic.  All waits are bounded.
// Measured in replayed graphs (calls made one by one take 6 - 7 us more, the host's part), 1 / 8 / 16 rows: 4096 x 4096
// 6.6 / 7.0 / 8.1 us, 4096 x 12288 12.5 / 12.9 / 15.9, gate and up 12288 x 4096 with SwiGLU 17.6 / 18.1 / 20.7 (23 rows 26.6),
// 126464 x 4096 55 / 55.5 / 70 (4.9 TB/s).  About 5 us of each are start, rewriting and join.
// 288 threads and three CTAs per SM leave 72 registers to a thread: every instance but those for 8 rows in groups of 32 without
// SwiGLU spills, 4 to 96 bytes (about 150 for 32 rows in groups of 32 with SwiGLU, 64 for the 23 rows above).  With four warps of 32
// features, which read every row fragment half as often, the 23 rows took 25.7 us, but one row of the same matrices 23.5.
#include "gemm_quantized.cuh"

namespace sl {

namespace {

constexpr int GQ_WARPS = 8, GQ_THREADS = 32 * GQ_WARPS + 32;
constexpr int GQ_ROWS = 8 * GQ_BK * 2;   // bytes of 8 rewritten rows in a stage

__device__ __forceinline__ void mma_f16(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}

// Scales and zero points of one feature for the groups of a stage, requested a stage ahead.  The four lanes that work on the
// feature have them all, or, with 8 groups to a stage, two each.
template <int G, bool FP32> struct GroupReader {
  static constexpr int GPT = GQ_BK / G, COUNT = GPT > 4 ? 2 : GPT, WORDS = COUNT * (FP32 ? 4 : 2) / 4;
  const uint8_t *s, *z;        // of the feature; z may be null
  uint32_t c[WORDS], n[WORDS], cz, nz;   // present and next stage

  __device__ __forceinline__ void fetch(int g0, int t, int ng, bool aligned) {   // of the stage whose first group is g0 -> n, nz
    const int g = g0 + (GPT > COUNT ? COUNT * t : 0);
    nz = 0x08080808u;
#pragma unroll
    for (int i = 0; i < WORDS; ++i) n[i] = 0;
    if (aligned) {
      if (g < ng) {
        const uint8_t* p = s + (size_t)g * (FP32 ? 4 : 2);
        if (WORDS == 1) {
          n[0] = __ldg(reinterpret_cast<const uint32_t*>(p));
        } else if (WORDS == 2) {
          const uint2 x = __ldg(reinterpret_cast<const uint2*>(p));
          n[0] = x.x; n[1 % WORDS] = x.y;
        } else {
          const uint4 x = __ldg(reinterpret_cast<const uint4*>(p));
          n[0] = x.x; n[1 % WORDS] = x.y; n[2 % WORDS] = x.z; n[3 % WORDS] = x.w;
        }
        if (z) nz = COUNT == 2 ? (uint32_t)__ldg(reinterpret_cast<const uint16_t*>(z + g)) : __ldg(reinterpret_cast<const uint32_t*>(z + g));
      }
    } else {
#pragma unroll
      for (int i = 0; i < COUNT; ++i)
        if (g + i < ng) {
          if (FP32) n[i % WORDS] = __ldg(reinterpret_cast<const uint32_t*>(s) + g + i);
          else n[i / 2 % WORDS] |= (uint32_t)__ldg(reinterpret_cast<const uint16_t*>(s) + g + i) << (16 * (i & 1));
          if (z) nz = (nz & ~(0xffu << (8 * i))) | (uint32_t)__ldg(z + g + i) << (8 * i);
        }
    }
  }
  __device__ __forceinline__ void turn() {
#pragma unroll
    for (int i = 0; i < WORDS; ++i) c[i] = n[i];
    cz = nz;
  }
  // group i of the stage: scale and minus the zero point (behind the feature's last group anything finite: its D and q are 0)
  __device__ __forceinline__ void get(int i, int lane, float& scale, float& minus_z) const {
    const int at = i % COUNT;
    uint32_t x = c[FP32 ? at % WORDS : at / 2 % WORDS], y = cz;
    if (GPT > COUNT) {
      x = __shfl_sync(0xffffffffu, x, (lane & 28) | (i / COUNT));
      y = __shfl_sync(0xffffffffu, y, (lane & 28) | (i / COUNT));
    }
    scale = __uint_as_float(FP32 ? x : at & 1 ? x & 0xffff0000u : x << 16);
    minus_z = 8388608.f - __uint_as_float(__byte_perm(y, 0x4b000000u, 0x7440 + at));   // 2^23 - (2^23 + z)
  }
};

template <int G, int NT> struct GqPlan {
  static constexpr int GPT = GQ_BK / G;                       // groups per stage
  static constexpr int CHUNK = GQ_ROWS + GPT * 32;           // 8 rewritten rows, then their q: [group][row]
  static constexpr int STAGE = GQ_CODES + (NT * CHUNK + 1023) / 1024 * 1024;
  static constexpr int OCC = 3;                               // CTAs per SM; two with more stages: 60 against 55 us (8 rows, 126464 x 4096); four: 26
                                                              // against 19 (gate and up 12288 x 4096)
  static constexpr int ROOM = 228 * 1024 / OCC - 1024 - 1024 - 256;
  static constexpr int STAGES = ROOM / STAGE > 4 ? 4 : ROOM / STAGE;
  static constexpr int PITCH = 132;                           // floats per packed row of the partial sums
  static constexpr int SMEM = 1024 + STAGES * STAGE + 256;
  static_assert(STAGES >= 2 && NT * 8 * PITCH * 4 <= STAGES * STAGE, "partial sums take the place of the stages");
};

// ---- the rewritten rows ----------------------------------------------------------------------------------------------
// One CTA per row, 8 k per thread at a time.  A row with an infinity or a NaN is NaN throughout.  Out: per (256 k, 8 rows) one
// chunk of GqPlan::CHUNK bytes, [word of a code fragment][lane] of 16 bytes: a' of the 8 k whose codes that word holds, in the
// order 0 4, 1 5 (over 16), 2 6, 3 7 (over 16), zeros behind K; then q of the groups, [group][row].  Or, not in FRAGMENTS, the
// same 16 bytes row by row, without q.  And e + 24 per row.
constexpr int GS_THREADS = 512;
constexpr int GS_KEPT = 4;              // eights of a row that a thread keeps in registers: 16384 k in all

template <int G, bool FRAGMENTS>
__global__ void __launch_bounds__(GS_THREADS)
gq_rewrite_rows_kernel(const bf16* __restrict__ A, const int32_t* __restrict__ n_active, int max_rows, int K, uint8_t* __restrict__ rows,
                       int32_t* __restrict__ row_exp) {
  __shared__ uint32_t sTop[GS_THREADS / 32];
  griddep_wait();
  griddep_launch();
  const int r = blockIdx.x;
  const uint4* row = reinterpret_cast<const uint4*>(A + (long long)r * K);
  constexpr uint32_t MAG = 0x7fff7fffu;
  uint4 first[GS_KEPT];                              // requested before the count is known: the row is there, if unused
#pragma unroll
  for (int j = 0; j < GS_KEPT; ++j) {
    const int i = threadIdx.x + j * GS_THREADS;
    first[j] = i < K / 8 ? __ldg(row + i) : make_uint4(0, 0, 0, 0);
  }
  if (r >= min(*n_active, max_rows)) return;
  uint32_t top = 0;
  auto largest = [&](const uint4& v) { top = __vmaxu2(top, __vmaxu2(__vmaxu2(v.x & MAG, v.y & MAG), __vmaxu2(v.z & MAG, v.w & MAG))); };
#pragma unroll
  for (int j = 0; j < GS_KEPT; ++j) largest(first[j]);
  for (int i = threadIdx.x + GS_KEPT * GS_THREADS; i < K / 8; i += GS_THREADS) largest(__ldg(row + i));
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = __vmaxu2(top, __shfl_xor_sync(0xffffffffu, top, o));
  if ((threadIdx.x & 31) == 0) sTop[threadIdx.x >> 5] = top;
  __syncthreads();
  top = sTop[threadIdx.x & (GS_THREADS / 32 - 1)];
#pragma unroll
  for (int o = GS_THREADS / 64; o > 0; o >>= 1) top = __vmaxu2(top, __shfl_xor_sync(0xffffffffu, top, o));
  top = max(top & 0xffffu, top >> 16);
  const bool bad = top >= 0x7f80u;
  int e = (int)(top >> 7) - 127 - 14;                // the largest magnitude becomes 2^14 ... 2^15
  if (top == 0 || bad) e = 0;
  e = max(e, -140);                                  // subnormal numbers
  if (threadIdx.x == 0) row_exp[r] = e + 24;
  const float d0 = gq_pow2(-e / 2), d1 = gq_pow2(-e - (-e / 2));
  const int blocks = (K + GQ_BK - 1) / GQ_BK, end = (blocks * 32 + GS_THREADS - 1) / GS_THREADS * GS_THREADS;   // whole warps: they shuffle
  auto rewrite = [&](int i, const uint4& v) __attribute__((always_inline)) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    float x[8], sum = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[2 * j] = __uint_as_float(w[j] << 16) * d0 * d1;
      x[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u) * d0 * d1;
    }
    uint32_t out[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float f = j & 1 ? 0.0625f : 1.f;
      const __half2 h = __floats2half2_rn(x[j] * f, x[j + 4] * f);
      const float2 back = __half22float2(h);         // what the products see
      sum += (back.x + back.y) * (j & 1 ? 16.f : 1.f);
      out[j] = bad ? 0x7fff7fffu : *reinterpret_cast<const uint32_t*>(&h);
    }
    if (FRAGMENTS) {
      if (bad) sum = __uint_as_float(0x7fffffffu);
#pragma unroll
      for (int o = 1; o < G / 8; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    }
    const int block = i / 32, k8 = i % 32, in = k8 % 16;
    if (block < blocks) {
      const uint4 y = make_uint4(out[0], out[1], out[2], out[3]);
      if (FRAGMENTS) {
        const int word = G == 128 ? in % 4 : G == 64 ? 2 * (in / 8) + in % 2 : in / 4;
        const int t = G == 128 ? in / 4 : G == 64 ? in % 8 / 2 : in % 4;
        uint8_t* chunk = rows + ((long long)block * ((max_rows + 7) / 8) + r / 8) * GqPlan<G, 1>::CHUNK;
        *reinterpret_cast<uint4*>(chunk + (((k8 / 16 * 4 + word) * 32 + (r % 8) * 4 + t) << 4)) = y;
        if (k8 % (G / 8) == 0) *reinterpret_cast<float*>(chunk + GQ_ROWS + k8 / (G / 8) * 32 + (r % 8) * 4) = sum * 5.9604644775390625e-8f;
      } else {
        *reinterpret_cast<uint4*>(rows + ((long long)r * blocks * 32 + i) * 16) = y;
      }
    }
  };
#pragma unroll
  for (int j = 0; j < GS_KEPT; ++j) {
    const int i = threadIdx.x + j * GS_THREADS;
    if (j * GS_THREADS < end) rewrite(i, first[j]);
  }
  for (int i = threadIdx.x + GS_KEPT * GS_THREADS; i < end; i += GS_THREADS) rewrite(i, i < K / 8 ? __ldg(row + i) : make_uint4(0, 0, 0, 0));
}

}  // namespace

// NT = number of eights of rows, max_rows / 8 rounded up
template <int G, int NT, bool DUAL, bool FP32>
__global__ void __launch_bounds__(GQ_THREADS, GqPlan<G, NT>::OCC)
gemm_quantized_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmW2, const GqArgs a, const int epilogue) {
  using P = GqPlan<G, NT>;
  constexpr int TO = DUAL ? 64 : 128;                         // output features of the CTA
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  float* sRed = reinterpret_cast<float*>(smem);               // [8 NT][PITCH] after the last stage
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + P::STAGES * P::STAGE);
  const uint32_t bar0 = smem_u32(bars);
  auto full = [&](int s) { return bar0 + 8u * s; };
  auto empty = [&](int s) { return bar0 + 8u * (P::STAGES + s); };
  volatile int* s_abort = reinterpret_cast<volatile int*>(bars + 2 * P::STAGES);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < P::STAGES; ++i) {
      mbar_init(full(i), 1);
      mbar_init(empty(i), GQ_WARPS);
    }
    *s_abort = 0;
    fence_mbar_init();
  }
  __syncthreads();

  uint32_t S, rank = 0;
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(S));
  if (S > 1) rank = cluster_ctarank();
  const int n0 = (int)(blockIdx.x / S) * TO;
  // *n_active, the weights and C were written before the rewriting kernel began; its rows come after griddep_wait()
  const int M = min(*a.n_active, a.max_rows);                 // none: the whole cluster leaves
  const int nblk = (a.K + GQ_BK - 1) / GQ_BK;
  const int b0 = (int)((long long)nblk * rank / S), b1 = (int)((long long)nblk * (rank + 1) / S);
  const int n = M > 0 ? b1 - b0 : 0;

  float acc[NT][4];
#pragma unroll
  for (int j = 0; j < NT; ++j) acc[j][0] = acc[j][1] = acc[j][2] = acc[j][3] = 0.f;

  if (warp == GQ_WARPS) {
    if (lane == 0) {
      const uint64_t once = l2_policy_evict_first();
      const int ahead = min(n, P::STAGES);
      auto codes = [&](int i) {
        const int st = i % P::STAGES;
        const uint32_t at = smem_u32(smem + st * P::STAGE);
        mbar_expect_tx(full(st), GQ_CODES + NT * P::CHUNK + (i == 0 && blockIdx.x == 0 ? a.lost : 0));
        tma_load_2d_hint(at, &tmW, (b0 + i) * (GQ_BK / 2), n0, full(st), once);
        if (DUAL) tma_load_2d_hint(at + GQ_CODES / 2, &tmW2, (b0 + i) * (GQ_BK / 2), n0, full(st), once);
      };
      for (int i = 0; i < ahead; ++i) codes(i);
      griddep_wait();
      griddep_launch();
      bool ok = true;
      int i = 0;
      for (; i < n; ++i) {
        const int st = i % P::STAGES;
        if (i >= ahead) {
          if (!(ok = mbar_wait(empty(st), ((i / P::STAGES) & 1) ^ 1, s_abort))) break;
          codes(i);
        }
        bulk_load(smem_u32(smem + st * P::STAGE) + GQ_CODES, a.rows + (long long)(b0 + i) * NT * P::CHUNK, NT * P::CHUNK, full(st));
      }
      // The copies in flight still write to this CTA's shared memory: they have landed (a bounded wait) before this thread goes
      // on, whichever warp's wait may have run out.
      const unsigned long long t0 = clock64();
      for (int k = max(0, i - P::STAGES); k < i; ++k)
        while (!mbar_try(full(k % P::STAGES), (k / P::STAGES) & 1) && clock64() - t0 < TC_WAIT_CYCLES) {}
      if (!ok) set_status(a.status, SL_DEV_GEMM_TIMEOUT);
    }
  } else {
    const int t = lane & 3, g = lane >> 2, rev = ((g & 1) << 2) | (g & 2) | (g >> 2);
    // feature rows of this lane in a stage: rows rev and 8 + rev of the warp's 16; with SwiGLU the first 64 of a
    // stage are the gate's, the others the up matrix's
    GroupReader<G, FP32> rd[2];
    const int mat = DUAL ? warp / (GQ_WARPS / 2) : 0;
    const uint32_t row0 = (uint32_t)(warp * 16 + rev) * 128;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int f = (DUAL ? warp % (GQ_WARPS / 2) : warp) * 16 + h * 8 + rev;
      const long long at = (long long)min(n0 + f, a.n_out - 1) * a.ng;   // features behind the last one: any scales, codes are 0
      rd[h].s = (const uint8_t*)(mat ? a.scales[1] : a.scales[0]) + at * (FP32 ? 4 : 2);
      const uint8_t* zeros = mat ? a.zeros[1] : a.zeros[0];
      rd[h].z = zeros ? zeros + at : nullptr;
    }
    auto fetch = [&](int i) {
#pragma unroll
      for (int h = 0; h < 2; ++h) rd[h].fetch((b0 + i) * P::GPT, t, a.ng, a.pairs != 0);
    };
    if (n > 0) fetch(0);
    bool ok = true;
    for (int i = 0; i < n; ++i) {
      const int st = i % P::STAGES;
      if (!(ok = __all_sync(0xffffffffu, mbar_wait(full(st), (i / P::STAGES) & 1, s_abort)))) break;
#pragma unroll
      for (int h = 0; h < 2; ++h) rd[h].turn();
      if (i + 1 < n) fetch(i + 1);
      const uint32_t base = smem_u32(smem + st * P::STAGE), tb = base + GQ_CODES + lane * 16;
      const uint32_t sw = (uint32_t)rev << 4;                 // swizzle: rows rev and 8 + rev of a tile have the same low bits
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        uint32_t cw[2][4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint32_t* c = cw[h];
          const uint32_t at = base + row0 + h * 8 * 128;
          if (G == 128) {
            const uint4 x = gq_lds128(at + (((hf * 4 + t) << 4) ^ sw));
            c[0] = x.x; c[1] = x.y; c[2] = x.z; c[3] = x.w;
          } else if (G == 64) {
#pragma unroll
            for (int q = 0; q < 2; ++q)
              asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(c[2 * q]), "=r"(c[2 * q + 1])
                           : "r"(at + (((hf * 4 + 2 * q + (t >> 1)) << 4) ^ sw) + (t & 1) * 8) : "memory");
          } else {
#pragma unroll
            for (int q = 0; q < 4; ++q)
              asm volatile("ld.shared.b32 %0, [%1];" : "=r"(c[q]) : "r"(at + (((hf * 4 + q) << 4) ^ sw) + t * 4) : "memory");
          }
        }
        float ga[NT][4];
        constexpr int WPG = G / 32;                           // words per group
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          if (w % WPG == 0) {
#pragma unroll
            for (int j = 0; j < NT; ++j) ga[j][0] = ga[j][1] = ga[j][2] = ga[j][3] = 0.f;
          }
          uint32_t x[2][4];                                   // codes 0 4 1 5 | 2 6 3 7
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint32_t lo = cw[h][w], hi = lo >> 8;
            x[0][h] = lo & 0x000f000fu;
            x[0][2 + h] = lo & 0x00f000f0u;
            x[1][h] = hi & 0x000f000fu;
            x[1][2 + h] = hi & 0x00f000f0u;
          }
#pragma unroll
          for (int j = 0; j < NT; ++j) {
            const uint4 b = gq_lds128(tb + j * P::CHUNK + (hf * 4 + w) * 512);
            mma_f16(ga[j], x[0], b.x, b.y);
            mma_f16(ga[j], x[1], b.z, b.w);
          }
          if (w % WPG == WPG - 1) {
            constexpr int HG = 4 / WPG;                       // groups per 128 k
            const int gi = hf * HG + w / WPG;
            float sc[2], mz[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) rd[h].get(gi, lane, sc[h], mz[h]);
#pragma unroll
            for (int j = 0; j < NT; ++j) {
              float q[2];                                     // of rows 2 t, 2 t + 1
              asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(q[0]), "=f"(q[1])
                           : "r"(base + GQ_CODES + j * P::CHUNK + GQ_ROWS + gi * 32 + t * 8) : "memory");
#pragma unroll
              for (int e = 0; e < 4; ++e)
                acc[j][e] = fmaf(sc[e >> 1], fmaf(mz[e >> 1], q[e & 1], ga[j][e]), acc[j][e]);
            }
          }
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(empty(st));
    }
    if (!ok && lane == 0) set_status(a.status, SL_DEV_GEMM_TIMEOUT);
  }

  // ---- sums of the cluster, epilogue ----
  __syncthreads();
  const bool good = *s_abort == 0;
  if (warp < GQ_WARPS) {
    const int t = lane & 3, g = lane >> 2, rev = ((g & 1) << 2) | (g & 2) | (g >> 2);
    if (!good) {                                              // an incomplete sum is NaN, for whichever CTA adds it
#pragma unroll
      for (int j = 0; j < NT; ++j) acc[j][0] = acc[j][1] = acc[j][2] = acc[j][3] = __uint_as_float(0x7fffffffu);
    }
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        sRed[(j * 8 + 2 * t + (e & 1)) * P::PITCH + warp * 16 + (e >> 1) * 8 + rev] = acc[j][e];
  }
  if (S > 1) cluster_sync_all(); else __syncthreads();
  if (M > 0) {
    const int c0 = (int)(TO / 4 * rank / S), cols = (int)(TO / 4 * (rank + 1) / S) - c0;   // features in fours that this CTA finishes
    for (int i = threadIdx.x; i < min(M, 8 * NT) * cols; i += GQ_THREADS) {
      const int r = i / cols, col = 4 * (c0 + i % cols);
      if (n0 + col >= a.n_out) continue;
      const float4 y = gq_total(sRed, S, r * P::PITCH + col);
      gq_store<DUAL>(a, epilogue, r, n0 + col, y, DUAL ? gq_total(sRed, S, r * P::PITCH + 64 + col) : y);
    }
  }
  if (S > 1) cluster_sync_all();                              // the others may still be reading this CTA's partial sums
}

namespace {

template <int G, int NT, bool DUAL, bool FP32>
int launch_gq(const CUtensorMap* w, const GqArgs& a, int epilogue, cudaStream_t st) {
  using P = GqPlan<G, NT>;
  constexpr int TO = DUAL ? 64 : 128;
  const int tiles = (a.n_out - 1) / TO + 1, nblk = (a.K - 1) / GQ_BK + 1;
  // K is split over S CTAs of a cluster while the CTAs still fit the GPU at once.  Unsplit / at most 4 / at most 8 / up to two rounds
  // of CTAs, 8 rows: 4096 x 4096 14.3 / 8.0 / 7.6 / 7.6 us, 4096 x 12288 35.8 / 14.1 / 13.0 / 12.9, gate and up 12288 x 4096 20.9 /
  // 19.3 / 19.3 / 24.2; 24 rows of these 34.2 / 28.5 / 28.3 / 34.0.
  const long long slots = (long long)sm_count() * P::OCC;
  int S = 1;
  while (S < 8 && S < nblk && (long long)tiles * (S + 1) <= slots) ++S;
  auto kernel = gemm_quantized_kernel<G, NT, DUAL, FP32>;
  static std::atomic<uint64_t> allowed{0};
  SL_CUDA_TRY(allow_smem(kernel, P::SMEM, allowed));
  SL_CUDA_TRY(gq_launch(kernel, dim3(tiles * S), GQ_THREADS, P::SMEM, S, st, w[0], w[1], a, epilogue));
  return SL_OK;
}

// Whether the kernel for few rows takes the call.  From 17 rows on its products bound it, where the weights are so few that the
// other kernel works on all of them at once, with a quarter of the k or less to a CTA (K = 12288, 4096 features: 25.0 against
// 21.5 us for 24 rows, 15.9 against 20.1 for 16); with more of them its fixed cost counts per round of CTAs (K = 4096, gate
// and up matrices of 12288 features: 28.5 against 42.4 us).  K = 4096, 17 / 24 / 32 rows, this kernel against the other:
//   1000 features 7.8 / 7.8 / 8.9 against 8.0 / 8.6 / 8.6     5120  11.7 / 12.1 / 15.8 against 12.9 / 13.0 / 13.1
//   2048          9.2 / 9.4 / 11.7 against 14.3 / 14.8 / 15.0  6144  12.1 / 12.5 / 21.9 against 22.1 / 22.3 / 22.5
//   4096          9.6 / 11.9 / 15.6 against 10.9 / 10.9 / 11.1 8192  13.9 / 15.4 / 19.7 against 15.4 / 15.2 / 15.4
//   4736          11.7 / 11.9 / 15.8 against 18.8 / 18.6 / 19.3 12288 16.6 / 17.0 / 20.9 against 33.4 / 33.8 / 33.4
// So the border is right on average; it loses where the other kernel's split of K comes out badly (2048 and 4736 features) and
// for 32 rows of 5120 or 8192.
constexpr int GQ_FEW = 32;             // most rows of the kernel for few rows
bool gq_few(int max_rows, int n_out, int epilogue) {
  const int tiles = (n_out - 1) / (epilogue == EPI_SWIGLU ? 64 : 128) + 1;
  return max_rows <= 16 || (max_rows <= GQ_FEW && 4ll * tiles > sm_count());
}

template <int G, bool DUAL, bool FP32> int by_rows(const CUtensorMap* w, const GqArgs& a, int epilogue, cudaStream_t st) {
  if (a.max_rows <= 8) return launch_gq<G, 1, DUAL, FP32>(w, a, epilogue, st);
  if (a.max_rows <= 16) return launch_gq<G, 2, DUAL, FP32>(w, a, epilogue, st);
  if (a.max_rows <= 24) return launch_gq<G, 3, DUAL, FP32>(w, a, epilogue, st);
  return launch_gq<G, 4, DUAL, FP32>(w, a, epilogue, st);
}
template <int G> int by_kind(const CUtensorMap* w, const void* A, const GqArgs& a, int epilogue, bool fp32, cudaStream_t st) {
  const bool few = gq_few(a.max_rows, a.n_out, epilogue);
  SL_CUDA_TRY(launch_pdl(few ? gq_rewrite_rows_kernel<G, true> : gq_rewrite_rows_kernel<G, false>, dim3(a.max_rows), dim3(GS_THREADS), 0, st,
                         (const bf16*)A, a.n_active, a.max_rows, a.K, (uint8_t*)a.rows, (int32_t*)a.row_exp));
  if (!few) return launch_gemm_quantized_tc(w, a, G, fp32, epilogue, st);
  if (epilogue == EPI_SWIGLU) return fp32 ? by_rows<G, true, true>(w, a, epilogue, st) : by_rows<G, true, false>(w, a, epilogue, st);
  return fp32 ? by_rows<G, false, true>(w, a, epilogue, st) : by_rows<G, false, false>(w, a, epilogue, st);
}

}  // namespace

int gq_map(CUtensorMap* out, const void* p, CUtensorMapDataType type, int elem, long long rows, long long cols, int box_rows, int box_cols) {
  TensorMapEncodeFn fn = tensor_map_encode_fn();
  if (!fn) return SL_ECUDA;
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)cols * elem};
  const cuuint32_t box[2] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows}, one[2] = {1, 1};
  const CUresult r = fn(out, type, 2, const_cast<void*>(p), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                        CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? SL_OK : SL_ECUDA;
}

// the workspace: the rewritten rows in either layout with room for the smallest groups (up to GQ_FEW rows the fragments take
// more), then their exponents
static size_t gq_rows_bytes(int max_rows, int K) {
  const size_t blocks = (K + GQ_BK - 1) / GQ_BK;
  if (max_rows <= GQ_FEW) return blocks * ((max_rows + 7) / 8) * GqPlan<32, 1>::CHUNK;
  return blocks * GQ_BK * 2 * max_rows;
}
size_t gemm_quantized_workspace_bytes(int max_rows, int K) { return gq_rows_bytes(max_rows, K) + (size_t)max_rows * sizeof(int32_t); }

int launch_gemm_quantized(const void* A, const surelock_w4* W, const surelock_w4* W2, void* C, const int32_t* n_active, int max_rows,
                          int n_out, int K, int epilogue, void* workspace, int32_t* status, cudaStream_t st) {
  if (max_rows > 65535) return SL_EUNSUPPORTED;
  GqArgs a{};
  CUtensorMap maps[2];
  a.ng = K / W->group;
  const bool fp32 = W->scale_dtype == SL_FP32, few = gq_few(max_rows, n_out, epilogue);
  a.pairs = a.ng % (few && W->group == 32 ? 2 : GQ_BK / W->group) == 0;
  for (int i = 0; i < 2; ++i) {
    const surelock_w4* w = i && W2 ? W2 : W;
    a.zeros[i] = (const uint8_t*)w->zeros;
    a.scales[i] = w->scales;
    if ((reinterpret_cast<uintptr_t>(w->scales) & 15) || (reinterpret_cast<uintptr_t>(w->zeros) & 7)) a.pairs = 0;
    const int rc = gq_map(&maps[i], w->codes, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, n_out, K / 2, epilogue == EPI_SWIGLU ? 64 : 128, GQ_BK / 2);
    if (rc != SL_OK) return rc;
  }
  a.rows = (const uint8_t*)workspace;
  a.row_exp = reinterpret_cast<const int32_t*>((const uint8_t*)workspace + gq_rows_bytes(max_rows, K));
  a.C = C;
  a.n_active = n_active;
  a.max_rows = max_rows;
  a.n_out = n_out;
  a.K = K;
  a.status = status;
  a.lost = take_lost_copy();
  switch (W->group) {
    case 32: return by_kind<32>(maps, A, a, epilogue, fp32, st);
    case 64: return by_kind<64>(maps, A, a, epilogue, fp32, st);
    default: return by_kind<128>(maps, A, a, epilogue, fp32, st);
  }
}

}  // namespace sl
