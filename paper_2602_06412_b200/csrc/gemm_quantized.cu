// Products of a few packed rows with 4-bit weights (the projections of Algorithm 1 lines 10, 12, 15 for weights held in
// four bits):
//
//   C[r][n] = sum_k A[r][k] W[n][k],   W[n][k] = (u[n][k] - z[n][k / g]) * s[n][k / g],   u = 0 ... 15
//
// with the epilogues of surelock_gemm_fused.  What bounds it with few rows: the weights, K / 2 bytes per output feature and
// their scales, are streamed once; every 4-bit code takes part in one multiply-add per row.
//
// mma.sync m16n8k16 with the WEIGHTS as the 16-row operand and the packed rows, padded to 8 NT, as its columns: with up to
// 16 rows an eighth of a tcgen05 tile would be used, and codes would have to travel through shared or tensor memory; here
// they go from global memory to registers and become bf16 there: (code & 15) | 0x4300 is the bf16 number 128 + u, minus
// (128 + z) is u - z, both exact.  The scale multiplies the fp32 sum of a whole group, so a weight is never rounded.
// The contraction index is permuted (the same way for both operands): a lane owns 16 consecutive code bytes per 128 weights
// of a row (8 or 4 with groups of 64 or 32, so that one MMA stays inside a group), and the codes of a 32-bit word pair up as
// (0,4) (1,5) (2,6) (3,7), which is what a shift and one logic operation give.  The rows' slice is brought into shared memory
// once per CTA in exactly that order, as the B fragments of the MMAs.
// A CTA has WN x WK warps: WN share the features (16 MTL each), WK the blocks of 128 k; the CTAs of a cluster share K
// further, so that few features still fill the GPU.  Sums meet in shared memory, then through distributed shared memory, in
// a fixed order: deterministic, no workspace.
#include <mutex>

#include "tc_common.cuh"

namespace sl {

namespace {

constexpr int GQ_THREADS = 256;

struct GqArgs {
  const bf16* A;
  const uint8_t *codes[2], *zeros[2];
  const void* scales[2];
  void* C;
  const int32_t* n_active;
  int max_rows, n_out, K, slice_blocks;   // slice: blocks of 128 k whose rows are in shared memory at a time
  int scale_fp32;
};

__device__ __forceinline__ void mma_bf16(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t sub_bf16x2(uint32_t a, uint32_t b) {
  const __nv_bfloat162 r = __hsub2(*reinterpret_cast<__nv_bfloat162*>(&a), *reinterpret_cast<__nv_bfloat162*>(&b));
  return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint4 ldg_stream(const void* p) {
  uint4 r;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p));
  return r;
}
__device__ __forceinline__ float ld_cluster_f32(uint32_t a) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(a) : "memory");
  return v;
}

// the codes, scales and zero points that a lane needs of 128 k of its 2 MTL feature rows
template <int G, int MTL> struct Codes {
  uint32_t w[MTL][2][4];
  float s[MTL][2][128 / G];
  uint32_t z[MTL][2][128 / G];   // 128 + z as two bf16
};

}  // namespace

template <int G, int NT, int MTL, int WN, bool DUAL, bool ZEROS>
__global__ void __launch_bounds__(GQ_THREADS, NT > 4 ? 1 : 2) gemm_quantized_kernel(const GqArgs a, const int epilogue) {
  constexpr int WK = GQ_THREADS / 32 / WN, TN = 16 * MTL * WN, GPB = 128 / G;
  constexpr int TO = DUAL ? TN / 2 : TN;          // output features of the CTA
  constexpr int PITCH = TN + 4;                   // floats per packed row of the reduction buffer
  extern __shared__ __align__(16) uint8_t smem[];
  uint4* sA = reinterpret_cast<uint4*>(smem);                  // [block][word][NT][32]
  float* sRed = reinterpret_cast<float*>(smem);                // [WK][8 NT][PITCH], after the last block

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int wn = warp % WN, wk = warp / WN;
  uint32_t S, rank = 0;
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(S));
  if (S > 1) rank = cluster_ctarank();
  const int n0 = (int)(blockIdx.x / S) * TO, r0 = blockIdx.y * 8 * NT;

  griddep_wait();
  griddep_launch();
  const int M = min(*a.n_active, a.max_rows) - r0;             // rows of this tile
  if (M <= 0) return;                                          // the whole cluster

  const int nblk = (a.K + 127) / 128, ng = a.K / G;
  const int b0 = (int)((long long)nblk * rank / S), b1 = (int)((long long)nblk * (rank + 1) / S);

  // feature rows of this lane; rows behind the last one read the last one's codes, their sums are dropped
  const uint8_t* code[MTL][2];
  long long srow[MTL][2];
#pragma unroll
  for (int mt = 0; mt < MTL; ++mt)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int tile = DUAL ? wn * (MTL / 2) + mt / 2 : wn * MTL + mt;
      const int n = min(n0 + tile * 16 + g + 8 * h, a.n_out - 1);
      code[mt][h] = a.codes[DUAL ? mt & 1 : 0] + (long long)n * (a.K / 2) + t * (G / 8);
      srow[mt][h] = (long long)n * ng;
    }

  auto load = [&](Codes<G, MTL>& c, int blk) {
#pragma unroll
    for (int mt = 0; mt < MTL; ++mt)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint8_t* p = code[mt][h] + (long long)blk * 64;
#pragma unroll
        for (int q = 0; q < GPB; ++q) {
          const int grp = blk * GPB + q;
          const bool in = G == 128 || grp < ng;
          if (G == 128) {
            const uint4 x = ldg_stream(p);
            c.w[mt][h][0] = x.x; c.w[mt][h][1] = x.y; c.w[mt][h][2] = x.z; c.w[mt][h][3] = x.w;
          } else if (G == 64) {
            const uint2 x = in ? __ldg(reinterpret_cast<const uint2*>(p + q * 32)) : make_uint2(0, 0);
            c.w[mt][h][(2 * q) & 3] = x.x;
            c.w[mt][h][(2 * q + 1) & 3] = x.y;
          } else {
            c.w[mt][h][q & 3] = in ? __ldg(reinterpret_cast<const uint32_t*>(p + q * 16)) : 0u;
          }
          const int m = DUAL ? mt & 1 : 0;
          const long long at = srow[mt][h] + grp;
          float s = 0.f;
          if (in) s = a.scale_fp32 ? __ldg((const float*)a.scales[m] + at) : __bfloat162float(((const bf16*)a.scales[m])[at]);
          c.s[mt][h][q] = s;
          if (ZEROS) c.z[mt][h][q] = in ? a.zeros[m][at] : 0;
        }
      }
  };

  float acc[MTL][NT][4];
#pragma unroll
  for (int mt = 0; mt < MTL; ++mt)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[mt][j][0] = acc[mt][j][1] = acc[mt][j][2] = acc[mt][j][3] = 0.f;

  auto compute = [&](const Codes<G, MTL>& c, const uint4* fr) {   // fr: the block's fragments, + lane
    float ga[MTL][NT][4];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      constexpr int WPG = 4 / GPB;                                // words per group
      const int q = w / WPG;
      if (w % WPG == 0) {
#pragma unroll
        for (int mt = 0; mt < MTL; ++mt)
#pragma unroll
          for (int j = 0; j < NT; ++j) ga[mt][j][0] = ga[mt][j][1] = ga[mt][j][2] = ga[mt][j][3] = 0.f;
      }
      uint32_t x[MTL][2][4];                                      // pairs (0,4) (1,5) (2,6) (3,7) of the two feature rows
#pragma unroll
      for (int mt = 0; mt < MTL; ++mt)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint32_t zz = 0x43084308u;                              // 136 = 128 + 8
          if (ZEROS) zz = 0x43004300u + c.z[mt][h][q] * 0x10001u;
#pragma unroll
          for (int i = 0; i < 4; ++i) x[mt][h][i] = sub_bf16x2(((c.w[mt][h][w] >> (4 * i)) & 0x000f000fu) | 0x43004300u, zz);
        }
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        const uint4 b = fr[(w * NT + j) * 32];
#pragma unroll
        for (int mt = 0; mt < MTL; ++mt) {
          const uint32_t a0[4] = {x[mt][0][0], x[mt][1][0], x[mt][0][1], x[mt][1][1]};
          const uint32_t a1[4] = {x[mt][0][2], x[mt][1][2], x[mt][0][3], x[mt][1][3]};
          mma_bf16(ga[mt][j], a0, b.x, b.y);
          mma_bf16(ga[mt][j], a1, b.z, b.w);
        }
      }
      if (w % WPG == WPG - 1) {
#pragma unroll
        for (int mt = 0; mt < MTL; ++mt)
#pragma unroll
          for (int j = 0; j < NT; ++j) {
            acc[mt][j][0] += c.s[mt][0][q] * ga[mt][j][0];
            acc[mt][j][1] += c.s[mt][0][q] * ga[mt][j][1];
            acc[mt][j][2] += c.s[mt][1][q] * ga[mt][j][2];
            acc[mt][j][3] += c.s[mt][1][q] * ga[mt][j][3];
          }
      }
    }
  };

  Codes<G, MTL> c0, c1;
  int blk = b0 + wk;
  if (blk < b1) load(c0, blk);
  for (int s0 = b0; s0 < b1; s0 += a.slice_blocks) {
    const int s1 = min(b1, s0 + a.slice_blocks);
    if (s0 > b0) __syncthreads();
    // rows of this slice, 8 consecutive k to a 16-byte fragment
    for (int i = threadIdx.x; i < (s1 - s0) * 4 * NT * 32; i += GQ_THREADS) {
      const int l = i & 31, j = (i >> 5) % NT, w = (i >> 5) / NT & 3, bl = (i >> 5) / NT >> 2;
      const int row = j * 8 + (l >> 2), tt = l & 3;
      const int k = (s0 + bl) * 128 + (G == 128 ? 32 * tt + 8 * w : G == 64 ? 64 * (w >> 1) + 16 * tt + 8 * (w & 1) : 32 * w + 8 * tt);
      uint4 v = make_uint4(0, 0, 0, 0);
      if (row < M && k < a.K) v = __ldg(reinterpret_cast<const uint4*>(a.A + (long long)(r0 + row) * a.K + k));
      sA[i] = make_uint4(__byte_perm(v.x, v.z, 0x5410), __byte_perm(v.x, v.z, 0x7632), __byte_perm(v.y, v.w, 0x5410),
                         __byte_perm(v.y, v.w, 0x7632));
    }
    __syncthreads();
    for (; blk < s1; blk += 2 * WK) {
      const bool two = blk + WK < b1;
      if (two) load(c1, blk + WK);
      compute(c0, sA + (blk - s0) * 4 * NT * 32 + lane);
      if (!two) { blk += WK; break; }
      if (blk + WK >= s1) {                                    // the next block belongs to the next slice
        c0 = c1;
        blk += WK;
        break;
      }
      if (blk + 2 * WK < b1) load(c0, blk + 2 * WK);
      compute(c1, sA + (blk + WK - s0) * 4 * NT * 32 + lane);
    }
  }

  // ---- reduction and epilogue ----
  __syncthreads();
  float* red = sRed + wk * (8 * NT * PITCH);
#pragma unroll
  for (int mt = 0; mt < MTL; ++mt)
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        red[(j * 8 + 2 * t + (i & 1)) * PITCH + (wn * MTL + mt) * 16 + g + 8 * (i >> 1)] = acc[mt][j][i];
  __syncthreads();
  if (WK > 1 && S > 1) {                                       // one partial result per CTA
    for (int i = threadIdx.x; i < min(M, 8 * NT) * TN; i += GQ_THREADS) {
      const int at = (i / TN) * PITCH + i % TN;
      float x = 0.f;
#pragma unroll
      for (int w = 0; w < WK; ++w) x += sRed[w * (8 * NT * PITCH) + at];
      sRed[at] = x;
    }
  }
  if (S > 1) cluster_sync_all();
  const uint32_t sred = smem_u32(sRed);
  auto total = [&](int at) {
    float x = 0.f;
    if (S > 1) {
      for (uint32_t s = 0; s < S; ++s) x += ld_cluster_f32(mapa_u32(sred + 4 * at, s));
    } else {
#pragma unroll
      for (int w = 0; w < WK; ++w) x += sRed[w * (8 * NT * PITCH) + at];
    }
    return x;
  };
  const int cols = TO / S;                                     // features that this CTA finishes
  for (int i = threadIdx.x; i < min(M, 8 * NT) * cols; i += GQ_THREADS) {
    const int r = i / cols, col = (int)rank * cols + i % cols, n = n0 + col;
    if (n >= a.n_out) continue;
    const long long at = (long long)(r0 + r) * a.n_out + n;
    if (DUAL) {
      const int p = r * PITCH + (col >> 4) * 32 + (col & 15);
      const float gate = total(p), up = total(p + 16);
      reinterpret_cast<bf16*>(a.C)[at] = __float2bfloat16_rn(gate / (1.f + __expf(-gate)) * up);
    } else {
      const float x = total(r * PITCH + col);
      if (epilogue == EPI_RESIDUAL) reinterpret_cast<float*>(a.C)[at] += x;
      else reinterpret_cast<bf16*>(a.C)[at] = __float2bfloat16_rn(x);
    }
  }
  if (S > 1) cluster_sync_all();                               // the others may still be reading this CTA's partial sums
}

namespace {

template <int G, int NT, int MTL, int WN, bool DUAL, bool ZEROS>
int launch_gq(const GqArgs& args, int epilogue, cudaStream_t st) {
  constexpr int WK = GQ_THREADS / 32 / WN, TN = 16 * MTL * WN, TO = DUAL ? TN / 2 : TN;
  GqArgs a = args;
  const int tiles = (a.n_out + TO - 1) / TO, nblk = (a.K + 127) / 128;
  const int row_tiles = (a.max_rows + 8 * NT - 1) / (8 * NT);
  const int slots = sm_count() * (NT > 4 ? 1 : 2);
  // K is shared by a cluster while the CTAs still fit the GPU at once and every warp keeps a block
  int S = 1;
  while (S < 8 && (long long)tiles * row_tiles * S * 2 <= slots && nblk >= 2 * S * WK) S *= 2;
  const int red = WK * 8 * NT * (TN + 4) * 4, cap = (NT > 4 ? 200 : 100) * 1024;
  const int per = (nblk + S - 1) / S, block_bytes = NT * 2048;
  a.slice_blocks = per * block_bytes <= cap ? per : cap / block_bytes;
  if (a.slice_blocks < per) a.slice_blocks -= a.slice_blocks % WK;   // a slice's blocks are dealt to the warps evenly
  const int smem = a.slice_blocks * block_bytes > red ? a.slice_blocks * block_bytes : red;
  auto kernel = gemm_quantized_kernel<G, NT, MTL, WN, DUAL, ZEROS>;
  static std::once_flag once;
  static cudaError_t attr;
  std::call_once(once, [&] { attr = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 200 * 1024); });
  SL_CUDA_TRY(attr);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(tiles * S, row_tiles);
  cfg.blockDim = dim3(GQ_THREADS);
  cfg.dynamicSmemBytes = (size_t)smem;
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
  SL_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, a, epilogue));
  return SL_OK;
}

template <int G, bool DUAL, bool ZEROS> int by_rows(const GqArgs& a, int epilogue, cudaStream_t st) {
  if (a.max_rows <= 8) return launch_gq<G, 1, 2, 4, DUAL, ZEROS>(a, epilogue, st);
  if (a.max_rows <= 16) return launch_gq<G, 2, 2, 4, DUAL, ZEROS>(a, epilogue, st);
  if (a.max_rows <= 32) return launch_gq<G, 4, 2, 4, DUAL, ZEROS>(a, epilogue, st);
  return launch_gq<G, 8, 2, 4, DUAL, ZEROS>(a, epilogue, st);
}
template <int G> int by_kind(const GqArgs& a, int epilogue, bool zeros, cudaStream_t st) {
  if (epilogue == EPI_SWIGLU) return zeros ? by_rows<G, true, true>(a, epilogue, st) : by_rows<G, true, false>(a, epilogue, st);
  return zeros ? by_rows<G, false, true>(a, epilogue, st) : by_rows<G, false, false>(a, epilogue, st);
}

}  // namespace

int launch_gemm_quantized(const void* A, const surelock_w4* W, const surelock_w4* W2, void* C, const int32_t* n_active, int max_rows,
                          int n_out, int K, int epilogue, cudaStream_t st) {
  GqArgs a{};
  a.A = (const bf16*)A;
  for (int i = 0; i < 2; ++i) {
    const surelock_w4* w = i && W2 ? W2 : W;
    a.codes[i] = (const uint8_t*)w->codes;
    a.zeros[i] = (const uint8_t*)w->zeros;
    a.scales[i] = w->scales;
  }
  a.C = C;
  a.n_active = n_active;
  a.max_rows = max_rows;
  a.n_out = n_out;
  a.K = K;
  a.scale_fp32 = W->scale_dtype == SL_FP32;
  switch (W->group) {
    case 32: return by_kind<32>(a, epilogue, W->zeros != nullptr, st);
    case 64: return by_kind<64>(a, epilogue, W->zeros != nullptr, st);
    default: return by_kind<128>(a, epilogue, W->zeros != nullptr, st);
  }
}

}  // namespace sl
