// Low-rank adapters of many requests beside a shared projection: for the rows r of a sequence that uses adapter a,
//   C[r] += scale_a B_a (A_a x_r),   A_a [rank][K], B_a [n_out][rank].
//
// One launch, no workspace: a cluster of CL CTAs takes 16 rows of one sequence (its adapter's weights are read once for
// them).  Each CTA multiplies its 1 / CL of K, the partial t = A_a x of all CTAs meet through distributed shared memory in a
// fixed order, and each CTA then adds its 1 / CL of the features to C.  Both products are mma.sync m16n8k16 with the rows on the
// 16 side: they are far from the tensor cores' rate (rank operations per byte), and their operands come straight from global
// memory in 16- and 8-byte loads, since any order of k serves as long as both operands keep it.
//
// x and the weights are bf16, so the first product's terms are exact and summed in fp32.  t scale stays an fp32 number: it enters
// the second product as three bf16 terms, all of its 24 bits.
//
// Bounded by latency for one row (6.4 us in a graph, K = n_out = 4096, rank 16: finding the sequence 1.2, each product about 1, joining t 1.2 us) and by
// round trips to the L2 for many adapters (64 rows of 48 adapters of rank 64, 4096 x 12288: 29 us for 74 MB, of 64: 31; of rank 16: 16.5 us): 16 warps of
// 128 registers to an SM, with the next 32 features' operands on their way.  Clusters as large as one round of the SMs' CTAs allows (two rounds, 64 adapters
// of rank 64, 32, 16: 35, 24.5, 20.5 instead of 31, 20.5, 16.5 us; of rank 128 with n_out = 4096: 41 instead of 35 us).
#include "gemm_adapters.cuh"

namespace sl {
namespace {

constexpr int AD_WARPS = 8, AD_THREADS = 32 * AD_WARPS, AD_CLUSTER = 8, AD_CHAIN = 8;

__device__ __forceinline__ void mma_16816(float* d, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float ld_cluster(uint32_t addr) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr));
  return v;
}

// two numbers of ranks k and k + 1: those from `rank` on become zeros
__device__ __forceinline__ uint32_t only(uint32_t two, int k, int rank) {
  return k >= rank ? 0u : k + 1 >= rank ? two & 0xffffu : two;
}

template <int NT, typename CT> struct AdapterTile {
  // times 32 features of weights and C in registers: as many as leave 128 registers to a thread and so two CTAs to an SM.  64 rows, n_out = 12288, with
  // twice as many and one CTA: rank 64 41 instead of 31 us, 32 26.5 instead of 20.5 with either C, 16 with fp32 C 22.5 instead of 16.5.  More than 64 ranks
  // take 252 registers.
  static constexpr bool FP32 = sizeof(CT) == 4;
  static constexpr int AHEAD = NT > 4 ? 1 : NT == 4 ? (FP32 ? 1 : 2) : (FP32 ? 2 : 3);
  static constexpr int CTAS = NT <= 8 ? 2 : 1;
  static constexpr int ROWS = 16, KS = AD_WARPS;
  static constexpr int TP = 8 * NT + 4;                               // pitch of t in floats: rows 4 banks apart
  // ranks to a load of weights: a quad's four lanes take 32 or 64 bytes of a feature, which costs the L1 half as many lines (64 ranks 35 -> 29 us)
  static constexpr int WK = NT <= 2 ? 16 : 32;
  static constexpr int SP = NT <= 2 ? 24 : NT == 4 ? 32 : 8 * NT + 32;  // pitch of its bf16 terms: neighbouring rows' WK miss one another's banks
  static constexpr int T_BYTES = KS * ROWS * TP * 4, BYTES = T_BYTES + TERMS * ROWS * SP * 2;
};

template <int NT, typename CT>
__global__ void __launch_bounds__(AD_THREADS, AdapterTile<NT, CT>::CTAS) gemm_adapters_kernel(AdapterArgs a) {
  using L = AdapterTile<NT, CT>;
  constexpr int ROWS = L::ROWS, KS = L::KS, TP = L::TP, SP = L::SP, WK = L::WK, KS2 = (8 * NT + WK - 1) / WK;
  extern __shared__ __align__(16) unsigned char smem[];
  float* part = reinterpret_cast<float*>(smem);
  bf16* terms = reinterpret_cast<bf16*>(smem + L::T_BYTES);
  griddep_wait();
  griddep_launch();
  uint32_t ctas;
  asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(ctas));
  const int CL = (int)ctas, rank_cta = (int)cluster_ctarank();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  int ad, row0, rows, rank;
  if (!find_tile(a, (int)(blockIdx.x / CL), (int)(gridDim.x / CL), ROWS, ad, row0, rows) || !find_rank(a, ad, rank)) return;
  const bf16* wa = a.a + (long long)ad * a.max_rank * a.K;
  const bf16* wb = a.b + (long long)ad * a.n_out * a.max_rank;
  // Up to 8 rows leave the lower half of the matrix instruction's 16 empty: it takes the rows' middle terms beside the first ones, and half of the last one
  // beside the other half; what comes of it is added to the upper half's.  So the third term costs those tiles no instruction (64 x 1 rows of rank 64, bf16
  // C: 29 us, by three instructions for every tile 33; fp32 C: 29 and 33).
  const bool half = rows <= 8;
  const int fgs = (a.n_out + 31) >> 5, fg0 = (int)((long long)fgs * rank_cta / CL), fg1 = (int)((long long)fgs * (rank_cta + 1) / CL);

  // ---- t = A_a x over this warp's k
  float acc[NT][4];
#pragma unroll
  for (int j = 0; j < NT; ++j) acc[j][0] = acc[j][1] = acc[j][2] = acc[j][3] = 0.f;
  {
    const int chunks = (a.K + 31) >> 5, splits = CL * KS, s = rank_cta * KS + warp;
    const int c0 = (int)((long long)chunks * s / splits), c1 = (int)((long long)chunks * (s + 1) / splits);
    const int ra = g, rb = g + 8;
    const bf16 *xa = a.x + (long long)(row0 + ra) * a.K, *xb = a.x + (long long)(row0 + rb) * a.K;
    const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
    // A matrix instruction may cut off where an addition would round, so long chains are joined outside: the sums so far go to shared memory
    float* to = part + (warp * ROWS + g) * TP + 2 * t;
    auto flush = [&](bool first) {
#pragma unroll
      for (int j = 0; j < NT; ++j) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float2* p = reinterpret_cast<float2*>(to + 8 * h * TP + 8 * j);
          float2 v = make_float2(acc[j][2 * h], acc[j][2 * h + 1]);
          if (!first) {
            const float2 o = *p;
            v.x += o.x;
            v.y += o.y;
          }
          *p = v;
        }
        acc[j][0] = acc[j][1] = acc[j][2] = acc[j][3] = 0.f;
      }
    };
#pragma unroll 2
    for (int ch = c0; ch < c1; ++ch) {
      if (ch > c0 && (ch - c0) % AD_CHAIN == 0) flush(ch - c0 == AD_CHAIN);
      const int k = ch * 32 + t * 8;
      const bool in = k < a.K;
      const uint4 u = in && ra < rows ? *reinterpret_cast<const uint4*>(xa + k) : zero;
      const uint4 v = in && rb < rows ? *reinterpret_cast<const uint4*>(xb + k) : zero;
      uint4 w[NT];
#pragma unroll
      for (int j = 0; j < NT; ++j) w[j] = in && 8 * j + g < rank ? __ldg(reinterpret_cast<const uint4*>(wa + (long long)(8 * j + g) * a.K + k)) : zero;
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        if (8 * j >= rank) break;
        mma_16816(acc[j], u.x, v.x, u.y, v.y, w[j].x, w[j].y);
        mma_16816(acc[j], u.z, v.z, u.w, v.w, w[j].z, w[j].w);
      }
    }
    flush(c1 - c0 <= AD_CHAIN);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < ROWS * 8 * NT; i += AD_THREADS) {
    const int at = (i / (8 * NT)) * TP + i % (8 * NT);
    float v = part[at];
#pragma unroll
    for (int w = 1; w < KS; ++w) v += part[w * ROWS * TP + at];
    part[at] = v;
  }
  cluster_sync_all();
  {
    const float scale = a.scale[ad];
    const uint32_t base = smem_u32(part);
    for (int i = threadIdx.x; i < ROWS * WK * KS2; i += AD_THREADS) {
      const int r = i / (WK * KS2), j = i % (WK * KS2);
      float v = 0.f;
      if (j < rank && r < rows) {
        const uint32_t at = base + 4 * (r * TP + j);
        float w[AD_CLUSTER];
#pragma unroll
        for (int c = 0; c < AD_CLUSTER; ++c) w[c] = c < CL ? ld_cluster(mapa_u32(at, c)) : 0.f;
#pragma unroll
        for (int c = 0; c < AD_CLUSTER; ++c) v += w[c];
        v *= scale;
      }
#pragma unroll
      for (int m = 0; m < TERMS; ++m)
        terms[m * ROWS * SP + r * SP + j] = __ushort_as_bfloat16((unsigned short)((m + 1 < TERMS ? next_term(v) : last_term(half ? 0.5f * v : v)) >> 16));
    }
  }
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");   // this CTA has read the others' t
  __syncthreads();

  // ---- C += B_a t over this CTA's features, 32 at a time to a warp: lane t of a quad ends up with 8 neighbours.  The weights and C of the
  // next times are on their way while these are multiplied.
  CT* c = reinterpret_cast<CT*>(a.c);
  const bool wide = (reinterpret_cast<uintptr_t>(c) & 15) == 0 && (a.c_stride * sizeof(CT)) % 16 == 0;
  const int ra = g, rb = g + 8;
  constexpr int LK = WK / 4;                          // ranks to a lane
  using Word = std::conditional_t<LK == 8, uint4, uint2>;
  const bf16* mine = terms + g * SP + LK * t;
  CT* const row_a = c + (row0 + ra) * a.c_stride + 8 * t;
  CT* const row_b = c + (row0 + rb) * a.c_stride + 8 * t;
  constexpr int WORDS = sizeof(CT) / 2;
  struct alignas(16) Eight { CT e[8]; };
  constexpr int AHEAD = L::AHEAD;
  Eight old[AHEAD][2];
  Word w[AHEAD][KS2][4];
  const bf16* const my_w = wb + (long long)(8 * (g >> 1) + (g & 1)) * a.max_rank + LK * t;
  auto load_w = [&](int fg, Word* to, int s) {
    const bf16* p = my_w + (long long)fg * 32 * a.max_rank + WK * s;
    const bool in = WK * s + LK * t < rank;
    if (fg * 32 + 32 <= a.n_out) {                   // the same for the whole warp
#pragma unroll
      for (int j = 0; j < 4; ++j) to[j] = in ? __ldg(reinterpret_cast<const Word*>(p + 2 * j * a.max_rank)) : Word{};
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        to[j] = in && fg * 32 + 8 * (g >> 1) + 2 * j + (g & 1) < a.n_out ? __ldg(reinterpret_cast<const Word*>(p + 2 * j * a.max_rank)) : Word{};
    }
  };
  auto load_c = [&](int fg, Eight* to) {
    const int f0 = fg * 32 + 8 * t;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const CT* p = (h ? row_b : row_a) + fg * 32;
      if ((h ? rb : ra) >= rows) continue;
      if (wide && f0 + 8 <= a.n_out) {
#pragma unroll
        for (int i = 0; i < WORDS; ++i) reinterpret_cast<uint4*>(&to[h])[i] = reinterpret_cast<const uint4*>(p)[i];
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (f0 + i < a.n_out) to[h].e[i] = p[i];
      }
    }
  };
#pragma unroll
  for (int u = 0; u < AHEAD; ++u)
    if (fg0 + warp + u * KS < fg1) {
      load_c(fg0 + warp + u * KS, old[u]);
#pragma unroll
      for (int s = 0; s < KS2; ++s) load_w(fg0 + warp + u * KS, w[u][s], s);
    }
  for (int fg_u = fg0 + warp; fg_u < fg1; fg_u += AHEAD * KS)
#pragma unroll
    for (int q = 0; q < AHEAD; ++q) {
      const int fg = fg_u + q * KS, next = fg + AHEAD * KS, f0 = fg * 32 + 8 * t;
      if (fg >= fg1) break;
      float d[4][4];
#pragma unroll
      for (int j = 0; j < 4; ++j) d[j][0] = d[j][1] = d[j][2] = d[j][3] = 0.f;
#pragma unroll
      for (int s = 0; s < KS2; ++s) {
        if (WK * s >= rank) break;
        const int k = WK * s + LK * t;
        Word* x = w[q][s];
        if (WK * s + WK > rank && k + LK > rank) {   // what lies behind the adapter's own rank is not read into the sum
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if constexpr (LK == 8) {
              x[j].w = only(x[j].w, k + 6, rank);
              x[j].z = only(x[j].z, k + 4, rank);
            }
            if (k + 3 >= rank) x[j].y &= 0xffffu;
            if (k + 2 >= rank) x[j].y = 0u;
            if (k + 1 >= rank) x[j].x &= 0xffffu;
          }
        }
#pragma unroll
        for (int m = TERMS - 1; m >= 0; --m) {       // the small terms first
          if (m == 1 && half) continue;
          const Word u = *reinterpret_cast<const Word*>(mine + m * ROWS * SP + WK * s);
          const Word v = *reinterpret_cast<const Word*>(mine + m * ROWS * SP + (!half ? 8 * SP : m == 0 ? ROWS * SP : 0) + WK * s);
#pragma unroll
          for (int j = 0; j < 4; ++j) mma_16816(d[j], u.x, v.x, u.y, v.y, x[j].x, x[j].y);
          if constexpr (LK == 8)
#pragma unroll
            for (int j = 0; j < 4; ++j) mma_16816(d[j], u.z, v.z, u.w, v.w, x[j].z, x[j].w);
        }
        if (next < fg1) load_w(next, x, s);
      }
      if (half)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          d[j][0] += d[j][2];
          d[j][1] += d[j][3];
        }
#pragma unroll
      for (int h = 0; h < 2; ++h)
        if ((h ? rb : ra) < rows) {
          CT* p = (h ? row_b : row_a) + fg * 32;
          Eight out;
#pragma unroll
          for (int i = 0; i < 8; ++i) out.e[i] = from_f<CT>(to_f(old[q][h].e[i]) + d[i >> 1][2 * h + (i & 1)]);
          if (wide && f0 + 8 <= a.n_out) {
#pragma unroll
            for (int i = 0; i < WORDS; ++i) reinterpret_cast<uint4*>(p)[i] = reinterpret_cast<const uint4*>(&out)[i];
          } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
              if (f0 + i < a.n_out) p[i] = out.e[i];
          }
        }
      if (next < fg1) load_c(next, old[q]);
    }
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");      // nobody reads this CTA's t any more
}

template <int NT, typename CT>
int launch_tile(const AdapterArgs& a, int groups, cudaStream_t st) {
  using L = AdapterTile<NT, CT>;
  // As large as one round allows, where half of the sequences of 16 rows and more are taken to end in whole tiles (16 x 24 rows of rank 128: 24.5 us, by
  // the bound alone 37)
  const int likely = groups - (a.max_rows >= 16ll * a.B ? a.B / 2 : 0);
  int CL = AD_CLUSTER;
  while (CL > 1 && (long long)likely * CL > (long long)L::CTAS * sm_count()) CL >>= 1;
  static std::atomic<uint64_t> done{0};
  SL_CUDA_TRY(allow_smem(gemm_adapters_kernel<NT, CT>, L::BYTES, done));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)groups * CL);
  cfg.blockDim = dim3(AD_THREADS);
  cfg.dynamicSmemBytes = L::BYTES;
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = CL;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = pdl_enabled() ? 2 : 1;
  SL_CUDA_TRY(cudaLaunchKernelEx(&cfg, gemm_adapters_kernel<NT, CT>, a));
  return SL_OK;
}

template <typename CT>
int launch_few(const AdapterArgs& a, cudaStream_t st) {
  // every sequence may end in a tile that is not full
  const long long groups = a.max_rows / 16 + (a.max_rows < a.B ? a.max_rows : a.B);
  if (groups > (1 << 27)) return SL_EUNSUPPORTED;
  if (a.max_rank <= 16) return launch_tile<2, CT>(a, (int)groups, st);
  if (a.max_rank <= 32) return launch_tile<4, CT>(a, (int)groups, st);
  if (a.max_rank <= 64) return launch_tile<8, CT>(a, (int)groups, st);
  return launch_tile<16, CT>(a, (int)groups, st);
}

}  // namespace

int launch_gemm_adapters(const void* A, const surelock_adapters& w, const int32_t* adapter_of_seq, const int32_t* row_offsets, int B,
                         void* C, long long c_stride, int max_rows, int n_out, int K, int dtype, int32_t* status, cudaStream_t st) {
  AdapterArgs a = {(const bf16*)A, (const bf16*)w.a, (const bf16*)w.b, w.scale, w.ranks, adapter_of_seq, row_offsets, C, status,
                         c_stride, w.n_adapters, w.max_rank, B, max_rows, n_out, K, 0};
  // The kernel for many rows takes 128 of a sequence at a time and 19 us at least; this one's time grows with rows x rank.  K = n_out = 4096, bf16, few
  // / many, us: 1 x 512 rows of rank 64 16.5 / 20.5, of rank 128 25 / 29; 1 x 1536 of rank 64 32 / 22.5; 8 x 64 rows of rank 64 16.5 / 25, of rank 128 24.5 /
  // 32.5; 8 x 128 rows of rank 16 12.5 / 20.5, 64 20.5 / 22.5, 128 37 / 29; 8 x 512 of rank 16 27 / 23.5, fp32 34.5 / 27; 32 x 64 of rank 64 33 / 31, fp32 35 /
  // 30, of rank 128 70 / 53.  So the border costs up to 8 us at a few hundred rows of the highest ranks (they lie just above it: 1 x 512 and 8 x 64 rows of
  // rank 128, where this kernel would be the faster one), and would cost as much at many rows of low ranks if it were twice as high.  (Its copies count the
  // pool's rows in 32 bits.)
  const bool many = max_rows >= 64ll * B && (long long)max_rows * w.max_rank >= 49152;
  if (many && (long long)w.n_adapters * (n_out > w.max_rank ? n_out : w.max_rank) < 0x7fffff00ll) {
    a.lost = take_lost_copy();
    return launch_gemm_adapters_tc(a, dtype, st);
  }
  return dtype == SL_BF16 ? launch_few<bf16>(a, st) : launch_few<float>(a, st);
}

}  // namespace sl
