// Low-rank adapters, many rows to a sequence:  C[r] += scale B_a (A_a x_r)  on tcgen05.
//
// A cluster of CL CTAs takes 128 rows of one sequence.  Each CTA multiplies its share of K,  t = x A_a^T  (128 x rank, accumulated in tensor
// memory; x and A_a by TMA in 64 k at a time); the shares meet through distributed shared memory in a fixed order; t scale becomes the
// tensor-memory operand of the second product as three bf16 terms, all 24 bits of it; and each CTA adds  t B_a^T  to its share
// of the features, 64 at a time.  Whole tiles of a bf16 C come with the weights, in the ring's slots, are added to there and copied back; those of an fp32 C
// are added to by reductions of the L2, which the SM does not read.  A sequence's last rows, or a C off 16 bytes, are read when their product is there.
//
// Bound by x once and C twice (rank operations per byte are few for the tensor cores).  In a graph, K = n_out = 4096: 9216 rows of 8 ragged sequences, rank
// 32, fp32 C 96 - 98 us for 378 MB.  Stamps of that run: 225 CTAs in clusters of 3 lie on 142 SMs, 166 of them two to an SM; the tile is found at 2 us, x read
// by 18 (6 TB/s), t joined by 23, and the features take 28 us where a CTA has its SM alone and 54 where two share one, so that the former end at 51 -
// 58 us and the latter at 78 - 92.  12288 rows of rank 64, bf16 C 80 us (3.9 TB/s), of rank 128, fp32 145 us.  C moves in whole tiles because a bulk copy
// takes some 16 clocks however short it is (a row of 128 bytes at a time: 118 instead of 77 us; through registers, row by row of lanes: 240).
#include "gemm_adapters.cuh"

namespace sl {
namespace {

constexpr int AT_STAGES = 3, AT_THREADS = 192, AT_COPY = 4, AT_MMA = 5, AT_JOIN = 60;   // four warps own the 128 rows, one copies, one multiplies
constexpr int AT_X = 128 * 128, AT_W = 64 * 128;                          // bytes of 64 k of the rows; of 64 rows of weights

// NH: halves of 64 ranks
template <typename CT, int NH> struct AtPlan {
  static constexpr int SLOT = AT_X + NH * AT_W;
  static constexpr int PITCH = 68;                                        // floats of a staged row: 16-byte accesses of 8 rows miss one another's banks
  static constexpr int STAGE = 128 * PITCH * 4;
  static constexpr int BARS = 3 * AT_STAGES + 6;
  static constexpr int SMEM = 1024 + AT_STAGES * SLOT + STAGE + BARS * 8 + 16;
  // Tensor memory: terms of t (16 bits a number), then two accumulators of 64 features.  t itself is accumulated in ACC places from the first column on,
  // which take the blocks of k in turn and are added up in fp32 behind the products: a matrix instruction cuts off where an addition rounds, and one chain
  // of 85 of them left 8.9e-7 in a result where four chains leave 1.9e-7.  The terms come to lie where sums were that have been read: with two halves of
  // ranks, the second's sums wait in the last place meanwhile.
  static constexpr uint32_t T_COLS = 32 * NH, D_COL = TERMS * T_COLS, COLS = NH == 1 ? 256 : 512, KEPT_COL = COLS - 64;
  static constexpr int ACC = COLS / (64 * NH);
  static_assert(ACC == 4 && D_COL + 128 <= COLS && (NH == 1 || D_COL <= KEPT_COL), "tensor memory");
  static constexpr int CTAS = COLS == 256 && 2 * (SMEM + 1024) <= 227 * 1024 ? 2 : 1;
};

__device__ __forceinline__ void at_mma(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool accum) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"((uint32_t)accum)
      : "memory");
}
__device__ __forceinline__ bool one_lane() {
  uint32_t yes;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(yes));
  return yes != 0;
}
__device__ __forceinline__ float4 ld_cluster_f4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr));
  return v;
}

__device__ __forceinline__ void st_cluster_f4(uint32_t addr, float4 v) {
  asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}

template <typename CT, int NH>
__global__ void __launch_bounds__(AT_THREADS, AtPlan<CT, NH>::CTAS)
gemm_adapters_tc_kernel(const __grid_constant__ CUtensorMap tmX, const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
                        const __grid_constant__ CUtensorMap tmC, const __grid_constant__ AdapterArgs a) {
  using P = AtPlan<CT, NH>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  float* stage = reinterpret_cast<float*>(smem + AT_STAGES * P::SLOT);     // [128][PITCH]
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + AT_STAGES * P::SLOT + P::STAGE);
  const uint32_t ring = smem_u32(smem), bar0 = smem_u32(bars);
  auto full = [&](int i) { return bar0 + 8u * (i % AT_STAGES); };
  auto empty = [&](int i) { return bar0 + 8u * (AT_STAGES + i % AT_STAGES); };
  const uint32_t t_done = bar0 + 8u * (2 * AT_STAGES), t_ready = t_done + 8u;
  auto d_full = [&](int j) { return t_ready + 8u + 8u * (j & 1); };
  auto d_empty = [&](int j) { return t_ready + 24u + 8u * (j & 1); };
  auto c_empty = [&](int j) { return t_ready + 40u + 8u * (j % AT_STAGES); };
  uint32_t* s_tmem = reinterpret_cast<uint32_t*>(bars + P::BARS);
  volatile int* s_abort = reinterpret_cast<volatile int*>(s_tmem + 1);

  griddep_wait();
  uint32_t ctas;
  asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(ctas));
  const int CL = (int)ctas, cta = (int)cluster_ctarank();
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  int row0, rows, ad, rank;                          // the same in the whole cluster
  if (!find_tile(a, (int)(blockIdx.x / CL), (int)(gridDim.x / CL), 128, ad, row0, rows) || !find_rank(a, ad, rank)) return;
  const int ranks = (a.max_rank + 15) & ~15;         // rows of A_a in a copy: a whole number of 16
  constexpr int VEC = 16 / sizeof(CT);
  // C may be copied in tiles: a copy writes whole 16 bytes, also where the row ends inside them
  const bool wide = (reinterpret_cast<uintptr_t>(a.c) & 15) == 0 && (a.c_stride * sizeof(CT)) % 16 == 0 && a.n_out % VEC == 0;
  struct alignas(16) Vec { CT e[VEC]; };
  const int blocks = (a.K + 63) >> 6, b0 = (int)((long long)blocks * cta / CL), n1 = (int)((long long)blocks * (cta + 1) / CL) - b0;
  const int tiles = (a.n_out + 63) >> 6, f0 = (int)((long long)tiles * cta / CL), n2 = (int)((long long)tiles * (cta + 1) / CL) - f0;

  if (threadIdx.x == 0) {
    for (int i = 0; i < AT_STAGES; ++i) {
      mbar_init(full(i), 1);
      mbar_init(empty(i), 1);
    }
    mbar_init(t_done, 1);
    mbar_init(t_ready, 4);
    for (int j = 0; j < 2; ++j) {
      mbar_init(d_full(j), 1);
      mbar_init(d_empty(j), 4);
    }
    for (int i = 0; i < AT_STAGES; ++i) mbar_init(c_empty(i), 1);
    *s_abort = 0;
    fence_mbar_init();
  }
  if (warp == AT_MMA) tc_alloc(smem_u32(s_tmem), P::COLS);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *s_tmem;
  // Only now may the next kernel start beside this one: one that took the tensor memory that this CTA is still to get, and then waited for this grid
  // to end, would leave both waiting.
  griddep_launch();
  bool ok = true;

  if (warp == AT_COPY) {
    int i = 0;                                       // copies that were started: first the blocks of k, then the tiles of features
    auto load = [&](int n) {
      for (; i < n; ++i) {
        if (!(ok = mbar_wait(empty(i), ((i / AT_STAGES) & 1) ^ 1, s_abort))) break;
        const uint32_t at = ring + i % AT_STAGES * P::SLOT;
        if (i < n1) {
          mbar_expect_tx(full(i), AT_X + ranks * 128 + (i == 0 && blockIdx.x == 0 ? a.lost : 0));
          tma_load_2d(at, &tmX, (b0 + i) * 64, row0, full(i));
          tma_load_2d(at + AT_X, &tmA, (b0 + i) * 64, ad * a.max_rank, full(i));
        } else {
          const int halves = rank > 64 ? 2 : 1, f = (f0 + i - n1) * 64;
          const bool with_c = sizeof(CT) == 2 && wide && rows == 128;
          if (with_c && i - n1 >= AT_STAGES && !(ok = mbar_wait(c_empty(i - n1 - AT_STAGES), ((i - n1) / AT_STAGES - 1) & 1, s_abort))) break;
          mbar_expect_tx(full(i), halves * AT_W + (with_c ? AT_X : 0));
          for (int h = 0; h < halves; ++h) tma_load_2d(at + h * AT_W, &tmB, 64 * h, (int)((long long)ad * a.n_out + f), full(i));
          if (with_c) tma_load_2d(at + NH * AT_W, &tmC, f, row0, full(i));
        }
      }
    };
    if (lane == 0) load(n1 + min(n2, AT_STAGES));
    __syncwarp();
    if (CL > 1)
      for (int h = 0; h < 3 * NH; ++h) cluster_sync_all();
    if (lane == 0) {
      if (ok) load(n1 + n2);
      // the copies in flight have landed (a bounded wait) before this thread goes on, whichever warp's wait may have run out
      const unsigned long long t0 = clock64();
      for (int k = max(0, i - AT_STAGES); k < i; ++k)
        while (!mbar_try(full(k), (k / AT_STAGES) & 1) && clock64() - t0 < TC_WAIT_CYCLES) {}
    }
  } else if (warp == AT_MMA) {
    const uint32_t base = __shfl_sync(0xffffffffu, tmem, 0), slots = __shfl_sync(0xffffffffu, ring, 0);
    const uint32_t first = idesc_bf16_m128(ranks), later = idesc_bf16_m128(64);
    int i = 0;
    for (; i < n1 && ok; ++i) {
      ok = __all_sync(0xffffffffu, mbar_wait(full(i), (i / AT_STAGES) & 1, s_abort));
      if (!ok) break;
      tc_fence_after();
      const uint32_t at = slots + i % AT_STAGES * P::SLOT;
      if (one_lane()) {
#pragma unroll
        for (int k = 0; k < 4; ++k)
          tc_mma_bf16(base + i % P::ACC * (64 * NH), smem_desc_k_sw128(at + 32 * k), smem_desc_k_sw128(at + AT_X + 32 * k), first,
                      i >= P::ACC || k > 0);
        tc_commit(empty(i));
        if (i == n1 - 1) tc_commit(t_done);
      }
      __syncwarp();
    }
    if (CL > 1)
      for (int h = 0; h < 3 * NH; ++h) cluster_sync_all();
    ok = ok && __all_sync(0xffffffffu, mbar_wait(t_ready, 0, s_abort));
    tc_fence_after();
    const int steps = (rank + 15) >> 4;
    int j = 0;
    for (; j < n2 && ok; ++j) {
      i = n1 + j;
      ok = __all_sync(0xffffffffu, mbar_wait(full(i), (i / AT_STAGES) & 1, s_abort) && mbar_wait(d_empty(j), ((j >> 1) & 1) ^ 1, s_abort));
      if (!ok) break;
      const uint32_t at = slots + i % AT_STAGES * P::SLOT;
      if (rank & 15) {
        // what lies behind the adapter's own rank meets zeros in t, but may be anything: zero it up to the last step's end
        for (int f = lane; f < 64; f += 32)
          for (int k = rank; k < 16 * steps; ++k) {
            const uint32_t in = (uint32_t)f * 128 + (k & 63) * 2, to = at + (k >> 6) * AT_W + (in ^ ((in >> 3) & 0x70u));   // 128-byte swizzle
            asm volatile("st.shared.u16 [%0], %1;" ::"r"(to), "h"((unsigned short)0) : "memory");
          }
        fence_async_smem();
        __syncwarp();
      }
      tc_fence_after();
      const uint32_t d = base + P::D_COL + (j & 1) * 64;
      if (one_lane()) {
        bool more = false;
#pragma unroll
        for (int m = TERMS - 1; m >= 0; --m)      // the small terms first
          for (int s = 0; s < steps; ++s) {          // 16 ranks: 8 columns of the operand, 32 bytes of the weights' rows
            at_mma(d, base + m * P::T_COLS + 8 * s, smem_desc_k_sw128(at + (s >> 2) * AT_W + (s & 3) * 32), later, more);
            more = true;
          }
        tc_commit(empty(i));
        tc_commit(d_full(j));
      }
      __syncwarp();
    }
    // the tensor memory is freed behind the barrier below: this warp's products, which end in order, are through with it (a bounded wait)
    if (lane == 0) {
      const unsigned long long t0 = clock64();
      if (j > 0) while (!mbar_try(d_full(j - 1), ((j - 1) >> 1) & 1) && clock64() - t0 < TC_WAIT_CYCLES) {}
      else if (i > 0) while (!mbar_try(empty(i - 1), ((i - 1) / AT_STAGES) & 1) && clock64() - t0 < TC_WAIT_CYCLES) {}
    }
  } else {
    const uint32_t mine = tmem + ((uint32_t)warp << 21);                   // this warp's lanes of the tensor memory
    const int row = warp * 32 + lane;
    float* own = stage + row * P::PITCH;
    const float scale = a.scale[ad];
    ok = __all_sync(0xffffffffu, mbar_wait(t_done, 0, s_abort));
    tc_fence_after();
    auto sum = [&](int h, uint32_t* v) {               // a half of the ranks; what is behind the ranks of the product is not used
      tc_ld32(mine + 64 * h, v);
      tc_ld32(mine + 64 * h + 32, v + 32);
      tc_wait_ld();
      for (int c = 1; c < min(P::ACC, n1); ++c)
#pragma unroll
        for (int k = 0; k < 64; k += 32) {
          uint32_t u[32];
          tc_ld32(mine + 64 * NH * c + 64 * h + k, u);
          tc_wait_ld();
#pragma unroll
          for (int e = 0; e < 32; ++e) v[k + e] = __float_as_uint(__uint_as_float(v[k + e]) + __uint_as_float(u[e]));
        }
    };
    if (NH == 2) {
      uint32_t v[64];
      sum(1, v);
      tc_st32(mine + P::KEPT_COL, v);
      tc_st32(mine + P::KEPT_COL + 32, v + 32);
      tc_wait_st();
    }
#pragma unroll
    for (int h = 0; h < NH; ++h) {
      uint32_t v[64];
      if (h == 0) sum(0, v);
      else {
        tc_ld32(mine + P::KEPT_COL, v);
        tc_ld32(mine + P::KEPT_COL + 32, v + 32);
        tc_wait_ld();
      }
      if (!ok) {                                     // an incomplete sum is NaN, for whichever CTA uses it
#pragma unroll
        for (int k = 0; k < 64; ++k) v[k] = 0x7fffffffu;
      }
      if (CL > 1) {
        // each CTA sums its 1 / CL of the rows over the cluster, in the order of the CTAs, and gives every CTA the sums (all CTAs reading all
        // shares: CL times the traffic)
#pragma unroll
        for (int k = 0; k < 64; k += 4) *reinterpret_cast<uint4*>(own + k) = make_uint4(v[k], v[k + 1], v[k + 2], v[k + 3]);
        __syncwarp();
        cluster_sync_all();
        const int parts = (min(rank - 64 * h, 64) + 3) >> 2;               // 16 bytes each; none in a half behind the rank
        const int r0 = 128 * cta / CL, of_all = (128 * (cta + 1) / CL - r0) * max(parts, 0);
        float4 sums[8];                              // 128 / CL rows of 16 parts over 128 threads
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          const int w = threadIdx.x + 128 * u;
          if (w >= of_all) break;
          const uint32_t at = smem_u32(stage + (r0 + w / parts) * P::PITCH + 4 * (w % parts));
          float4 p[8];
#pragma unroll
          for (int c = 0; c < 8; ++c)
            if (c < CL) p[c] = ld_cluster_f4(mapa_u32(at, c));
          float4 t = p[0];
#pragma unroll
          for (int c = 1; c < 8; ++c)
            if (c < CL) {
              t.x += p[c].x;
              t.y += p[c].y;
              t.z += p[c].z;
              t.w += p[c].w;
            }
          sums[u] = t;
        }
        __syncwarp();
        cluster_sync_all();                          // all shares have been read
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          const int w = threadIdx.x + 128 * u;
          if (w >= of_all) break;
          const uint32_t at = smem_u32(stage + (r0 + w / parts) * P::PITCH + 4 * (w % parts));
          for (int c = 0; c < CL; ++c) st_cluster_f4(mapa_u32(at, c), sums[u]);
        }
        __syncwarp();
        cluster_sync_all();
#pragma unroll
        for (int k = 0; k < 64; k += 4) {
          const uint4 t = *reinterpret_cast<const uint4*>(own + k);
          v[k] = t.x;
          v[k + 1] = t.y;
          v[k + 2] = t.z;
          v[k + 3] = t.w;
        }
      }
#pragma unroll
      for (int k = 0; k < 64; ++k) v[k] = 64 * h + k < rank ? __float_as_uint(__uint_as_float(v[k]) * scale) : 0u;
#pragma unroll
      for (int m = 0; m < TERMS; ++m) {
        uint32_t w[32];
#pragma unroll
        for (int k = 0; k < 32; ++k) {
          float x = __uint_as_float(v[2 * k]), y = __uint_as_float(v[2 * k + 1]);
          const uint32_t a0 = m + 1 < TERMS ? next_term(x) : last_term(x), a1 = m + 1 < TERMS ? next_term(y) : last_term(y);
          w[k] = __byte_perm(a0, a1, 0x7632);
          v[2 * k] = __float_as_uint(x);
          v[2 * k + 1] = __float_as_uint(y);
        }
        tc_st32(mine + m * P::T_COLS + 32 * h, w);
      }
    }
    tc_wait_st();
    tc_fence_before();
    __syncwarp();
    if (lane == 0) mbar_arrive(t_ready);
    // The loop below has barriers of these four warps, and each came here by a wait of its own, which may have run out for some of them only:
    // all enter it, or none.  From here on `ok` is the same in all four at every turn.
    ok = epilogue_warps_agree(ok);

    const bool whole = wide && rows == 128, issues = threadIdx.x == 0, bulk = sizeof(CT) == 4 && wide;
    auto together = [] { asm volatile("bar.sync 1, 128;" ::: "memory"); };
    int j = 0;
    for (; j < n2 && ok; ++j) {
      const int f = (f0 + j) * 64, slot = (n1 + j) % AT_STAGES;
      ok = mbar_wait(d_full(j), (j >> 1) & 1, s_abort);
      if (sizeof(CT) == 2 && whole) ok = ok && mbar_wait(full(n1 + j), ((n1 + j) / AT_STAGES) & 1, s_abort);   // C's tile is here too
      ok = epilogue_warps_agree(ok);
      if (!ok) break;
      tc_fence_after();
      uint32_t v[64];
      tc_ld32(mine + P::D_COL + (j & 1) * 64, v);
      tc_ld32(mine + P::D_COL + (j & 1) * 64 + 32, v + 32);
      tc_wait_ld();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(d_empty(j));
      if (!whole) {
        // the last rows of a sequence, or a C that is not aligned: by ordinary accesses, a row's numbers side by side in the lanes
        if (bulk) bulk_wait_read0();
#pragma unroll
        for (int k = 0; k < 64; k += 4) *reinterpret_cast<uint4*>(own + k) = make_uint4(v[k], v[k + 1], v[k + 2], v[k + 3]);
        if constexpr (sizeof(CT) == 4)
          if (bulk) {                                // each row by a reduction of its own
            fence_async_smem();
            if (row < rows) bulk_reduce_add_f32(reinterpret_cast<float*>(a.c) + (long long)(row0 + row) * a.c_stride + f, smem_u32(own), 4 * min(64, a.n_out - f));
            bulk_commit();
            continue;
          }
        __syncwarp();
        constexpr int PER_ROW = 64 / VEC, LR = 32 / PER_ROW, STEPS = 32 / LR;
        const int lr = lane / PER_ROW, col = lane % PER_ROW * VEC, last = rows - warp * 32;
        const float* from = stage + (warp * 32 + lr) * P::PITCH + col;
        CT* to = reinterpret_cast<CT*>(a.c) + (long long)(row0 + warp * 32 + lr) * a.c_stride + f + col;
        if (wide && f + 64 <= a.n_out) {
          Vec o[STEPS];
#pragma unroll
          for (int s = 0; s < STEPS; ++s)
            if (s * LR + lr < last) o[s] = *reinterpret_cast<const Vec*>(to + (long long)s * LR * a.c_stride);
#pragma unroll
          for (int s = 0; s < STEPS; ++s)
            if (s * LR + lr < last) {
#pragma unroll
              for (int e = 0; e < VEC; ++e) o[s].e[e] = from_f<CT>(to_f(o[s].e[e]) + from[s * LR * P::PITCH + e]);
              *reinterpret_cast<Vec*>(to + (long long)s * LR * a.c_stride) = o[s];
            }
        } else {
          CT* c = reinterpret_cast<CT*>(a.c) + (long long)(row0 + warp * 32) * a.c_stride + f + lane;
          const bool in[2] = {f + lane < a.n_out, f + lane + 32 < a.n_out};
          for (int r0 = 0; r0 < min(last, 32); r0 += 4) {
            CT o[4][2];
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
              for (int h = 0; h < 2; ++h)
                if (in[h] && r0 + r < last) o[r][h] = c[(r0 + r) * a.c_stride + 32 * h];
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
              for (int h = 0; h < 2; ++h)
                if (in[h] && r0 + r < last) c[(r0 + r) * a.c_stride + 32 * h] = from_f<CT>(to_f(o[r][h]) + stage[(warp * 32 + r0 + r) * P::PITCH + lane + 32 * h]);
          }
        }
        __syncwarp();                                // the staged rows are written again
        continue;
      }
      if constexpr (sizeof(CT) == 4) {
        // fp32: 32 features at a time are staged and added to C by the L2, which the SM does not read
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          if (issues) asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");   // this half's last reduction has read its numbers
          together();
          uint8_t* to = reinterpret_cast<uint8_t*>(stage) + h * AT_X + row * 128;
#pragma unroll
          for (int k = 0; k < 8; ++k)
            *reinterpret_cast<uint4*>(to + ((k ^ (row & 7)) << 4)) = make_uint4(v[32 * h + 4 * k], v[32 * h + 4 * k + 1], v[32 * h + 4 * k + 2], v[32 * h + 4 * k + 3]);
          fence_async_smem();
          together();
          if (issues && f + 32 * h < a.n_out) {
            asm volatile("cp.reduce.async.bulk.tensor.2d.global.shared::cta.add.tile.bulk_group [%0, {%1, %2}], [%3];"
                         ::"l"(&tmC), "r"(f + 32 * h), "r"(row0), "r"(smem_u32(stage) + h * AT_X) : "memory");
          }
          if (issues) bulk_commit();
        }
      } else {
        // bf16: C's tile came with the weights'; it is added to in place and copied back
        uint8_t* at = smem + slot * P::SLOT + NH * AT_W + row * 128;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          uint4* p = reinterpret_cast<uint4*>(at + ((k ^ (row & 7)) << 4));
          const uint4 o = *p;
          const uint32_t w[4] = {o.x, o.y, o.z, o.w};
          uint32_t y[4];
#pragma unroll
          for (int e = 0; e < 4; ++e)
            y[e] = pack_bf16(__uint_as_float(w[e] << 16) + __uint_as_float(v[8 * k + 2 * e]), __uint_as_float(w[e] & 0xffff0000u) + __uint_as_float(v[8 * k + 2 * e + 1]));
          *p = make_uint4(y[0], y[1], y[2], y[3]);
        }
        fence_async_smem();
        together();
        if (issues) {
          asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];"
                       ::"l"(&tmC), "r"(f), "r"(row0), "r"(smem_u32(smem) + slot * P::SLOT + NH * AT_W) : "memory");
          bulk_commit();
          if (j > 0) {
            asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
            mbar_arrive(c_empty(j - 1));             // the last tile has been read
          }
        }
      }
    }
    bulk_wait0();
    if (!ok && row < rows)                           // what this CTA did not get to is NaN
      for (int f = (f0 + j) * 64; f < min((f0 + n2) * 64, a.n_out); ++f)
        reinterpret_cast<CT*>(a.c)[(long long)(row0 + row) * a.c_stride + f] = from_f<CT>(__uint_as_float(0x7fffffffu));
  }
  if (!ok && lane == 0) set_status(a.status, SL_DEV_GEMM_TIMEOUT);
  tc_fence_before();
  __syncthreads();
  if (warp == AT_MMA) {
    tc_fence_after();
    tc_dealloc(tmem, P::COLS);
  }
}

template <typename CT, int NH> int launch_at(const AdapterArgs& a, cudaStream_t st) {
  using P = AtPlan<CT, NH>;
  CUtensorMap x, wa, wb, c;
  const int ranks = (a.max_rank + 15) & ~15;
  int rc = get_tensor_map_2d(a.x, a.max_rows, a.K, 128, &x);
  if (rc == SL_OK) rc = get_tensor_map_2d(a.a, (long long)a.n_adapters * a.max_rank, a.K, ranks, &wa);
  if (rc == SL_OK) rc = get_tensor_map_2d(a.b, (long long)a.n_adapters * a.n_out, a.max_rank, 64, &wb);
  if (rc != SL_OK) return rc;
  if ((reinterpret_cast<uintptr_t>(a.c) & 15) == 0 && (a.c_stride * sizeof(CT)) % 16 == 0) {
    TensorMapEncodeFn fn = tensor_map_encode_fn();
    const cuuint64_t dims[2] = {(cuuint64_t)a.n_out, (cuuint64_t)a.max_rows}, strides[1] = {(cuuint64_t)a.c_stride * sizeof(CT)};
    const cuuint32_t box[2] = {128 / sizeof(CT), 128}, each[2] = {1, 1};
    if (!fn || fn(&c, sizeof(CT) == 2 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 2, a.c, dims, strides, box, each,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
      return SL_ECUDA;
  } else {
    c = x;                                           // not used
  }
  auto kernel = gemm_adapters_tc_kernel<CT, NH>;
  static std::atomic<uint64_t> done{0};
  SL_CUDA_TRY(allow_smem(kernel, P::SMEM, done));
  const long long groups = a.max_rows / 128 + (a.max_rows < a.B ? a.max_rows : a.B);   // every sequence may end in a tile that is not full
  // The number of CTAs to a tile with the least estimated time: rounds of CTAs on the GPU, times a CTA's share of the work and what it spends
  // on starting and joining.  Half of the sequences are taken to end in a tile of their own.
  const long long likely = a.max_rows / 128 + (a.max_rows < a.B ? a.max_rows : a.B) / 2 + 1, room = (long long)P::CTAS * sm_count();
  int CL = 1;
  long long best = 0;
  for (int n = 1; n <= 8 && n <= (a.K + 63) / 64; ++n) {
    const long long t = (likely * n + room - 1) / room * (1000 / n + AT_JOIN);
    if (n == 1 || t < best) {
      best = t;
      CL = n;
    }
  }
  if (groups * CL > 0x7fffffffll) return SL_EUNSUPPORTED;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(groups * CL));
  cfg.blockDim = dim3(AT_THREADS);
  cfg.dynamicSmemBytes = P::SMEM;
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = CL;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = pdl_enabled() ? 2 : 1;
  SL_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, x, wa, wb, c, a));
  return SL_OK;
}

}  // namespace

int launch_gemm_adapters_tc(const AdapterArgs& a, int dtype, cudaStream_t st) {
  if (dtype == SL_BF16) return a.max_rank <= 64 ? launch_at<bf16, 1>(a, st) : launch_at<bf16, 2>(a, st);
  return a.max_rank <= 64 ? launch_at<float, 1>(a, st) : launch_at<float, 2>(a, st);
}

}  // namespace sl
