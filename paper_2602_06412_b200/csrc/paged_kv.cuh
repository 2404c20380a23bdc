// Paged K/V cache held in few bits: element types and conversions shared by the kernels that write it, read it back and
// attend to it (the layout is described at surelock_paged_kv in include/surelock.h).
#pragma once
#include <cuda_fp16.h>

#include "common.cuh"

namespace sl {

// what can be checked on the host; SL_OK, SL_EINVAL or SL_EUNSUPPORTED
int check_paged_kv(const surelock_paged_kv* c);

int launch_kv_scatter_paged(const surelock_paged_kv& c, const void* k, const void* v, long long row_stride, const int32_t* idx,
                            const int32_t* n_active, int max_rows, int B, int N, int dtype, int32_t* status, cudaStream_t st);
int launch_kv_gather_paged(const surelock_paged_kv& c, const int32_t* idx, const int32_t* n_active, int max_rows, int B, int N,
                           void* k, void* v, long long row_stride, int dtype, int32_t* status, cudaStream_t st);

size_t attention_paged_workspace_bytes(int head_dim);
int launch_attention_paged(const surelock_paged_kv& c, const void* q, long long q_stride, const int32_t* row_offsets,
                           const int32_t* seq_lens, int max_rows, int B, int H, void* o, long long o_stride, void* workspace,
                           int32_t* status, cudaStream_t st);

template <int KIND> struct KvKind;
template <> struct KvKind<SL_BF16> { static constexpr int BYTES = 2; static constexpr float QMAX = 0.f; };
template <> struct KvKind<SL_E4M3> { static constexpr int BYTES = 1; static constexpr float QMAX = 448.f; };
template <> struct KvKind<SL_INT8> { static constexpr int BYTES = 1; static constexpr float QMAX = 127.f; };

// two codes (the low and the high byte of the lower 16 bits) as two fp16 values; exact for both types
__device__ __forceinline__ uint32_t e4m3x2_to_f16x2(uint16_t two) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"(two));
  return r;
}

}  // namespace sl
