// Products with 4-bit weights: what the kernel for few rows (gemm_quantized.cu) and the one for more (gemm_quantized_tc.cu)
// share.
#pragma once
#include <cuda_fp16.h>

#include "tc_common.cuh"

namespace sl {

constexpr int GQ_BK = 256;             // k per stage: 128 bytes of a feature's codes (64-byte rows stream at two thirds of the rate)
constexpr int GQ_CODES = 128 * GQ_BK / 2;   // bytes of the codes of 128 features

struct GqArgs {
  const uint8_t *zeros[2], *rows;
  const void* scales[2];
  void* C;
  const int32_t* n_active;
  const int32_t* row_exp;              // e + 24 of every row
  int max_rows, n_out, K, ng;
  int pairs;                           // scales and zero points of a few neighbouring groups lie on aligned addresses
  int32_t* status;
  int lost;                            // bytes that CTA 0's first stage waits for in vain: 0, but for the diagnostic
};

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
__device__ __forceinline__ float gq_pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }   // -126 <= e <= 127

// four neighbouring features of one row, summed over the CTAs of the cluster in order: partial sums at float index `at` of each
__device__ __forceinline__ float4 gq_total(const float* red, uint32_t S, int at) {
  if (S == 1) return *reinterpret_cast<const float4*>(red + at);
  const uint32_t base = smem_u32(red) + 4 * at;
  float4 p[8], x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
  for (uint32_t s = 0; s < 8; ++s)
    if (s < S) p[s] = ld_cluster_f4(mapa_u32(base, s));
#pragma unroll
  for (uint32_t s = 0; s < 8; ++s)
    if (s < S) {
      x.x += p[s].x; x.y += p[s].y; x.z += p[s].z; x.w += p[s].w;
    }
  return x;
}
// result of features n ... n + 3 of row r: sum (and, with SwiGLU, the up matrix's), times the row's power of two
template <bool DUAL> __device__ __forceinline__ void gq_store(const GqArgs& a, int epilogue, int r, int n, const float4& y, const float4& u) {
  const int ex = __ldcg(a.row_exp + r);              // in two factors, which are normal numbers
  const float p0 = gq_pow2(ex / 2), p1 = gq_pow2(ex - ex / 2);
  float x[4] = {y.x * p0 * p1, y.y * p0 * p1, y.z * p0 * p1, y.w * p0 * p1};
  if (DUAL) {
    const float up[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = x[e] / (1.f + __expf(-x[e])) * (up[e] * p0 * p1);
  }
  const long long out = (long long)r * a.n_out + n;
  if (epilogue == EPI_RESIDUAL && !DUAL) {
    float* c = reinterpret_cast<float*>(a.C) + out;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (n + e < a.n_out) c[e] += x[e];
  } else {
    bf16* c = reinterpret_cast<bf16*>(a.C) + out;
    if ((a.n_out & 3) == 0) {
      *reinterpret_cast<uint2*>(c) = make_uint2(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]));
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (n + e < a.n_out) c[e] = __float2bfloat16_rn(x[e]);
    }
  }
}

// 2-D row-major tensor map, zeros out of bounds, in boxes of 128-byte rows under the 128-byte swizzle
int gq_map(CUtensorMap* out, const void* p, CUtensorMapDataType type, int elem, long long rows, long long cols, int box_rows, int box_cols);
// launch with a cluster of S CTAs along x and programmatic dependent launch
template <typename... KArgs, typename... Args>
inline cudaError_t gq_launch(void (*kernel)(KArgs...), dim3 grid, int threads, size_t smem, int S, cudaStream_t st, Args&&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = S;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = pdl_enabled() ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...);
}

// the product for more rows (gemm_quantized_tc.cu); rows rewritten as [max_rows][K up to GQ_BK] fp16
int launch_gemm_quantized_tc(const CUtensorMap* w, const GqArgs& a, int group, bool fp32, int epilogue, cudaStream_t st);

}  // namespace sl
