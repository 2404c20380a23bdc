// Low-rank adapters of many requests: what the two kernels share (the few rows' in gemm_adapters.cu, the many rows' in
// gemm_adapters_tc.cu).
#pragma once
#include "tc_common.cuh"

namespace sl {

struct AdapterArgs {
  const bf16 *x, *a, *b;
  const float* scale;
  const int32_t *ranks, *adapter_of_seq, *row_offsets;
  void* c;
  int32_t* status;
  long long c_stride;
  int n_adapters, max_rank, B, max_rows, n_out, K;
  int lost;                         // bytes of a copy that is waited for and never made (a diagnostic), or 0
};

// The group-th tile, of at most `groups`, of `tile` rows of one sequence: its adapter's number, first row and rows; every lane of a warp gets the same.
__device__ __forceinline__ bool find_tile(const AdapterArgs& a, int group, int groups, int tile, int& ad, int& row0, int& rows) {
  const int lane = threadIdx.x & 31;
  int before = 0;                                    // tiles of the sequences before this round's 32
  bool bad = false;
  for (int b0 = 0; b0 < a.B; b0 += 32) {
    const int b = b0 + lane;
    // offsets are clamped, so that no row is outside C
    int from = b < a.B ? a.row_offsets[b] : 0, to = b < a.B ? a.row_offsets[b + 1] : 0;
    const int its = b < a.B ? a.adapter_of_seq[b] : -1;    // for every sequence, so that its load does not wait for the search
    if (b < a.B) bad |= from < 0 || to < from || to > a.max_rows;
    from = min(max(from, 0), a.max_rows);
    to = min(max(to, from), a.max_rows);
    const int mine = (int)(((long long)to - from + tile - 1) / tile);
    int sum = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, sum, o);
      if (lane >= o) sum += v;
    }
    const unsigned hit = __ballot_sync(0xffffffffu, group - before < sum);
    if (hit) {
      const int l = __ffs(hit) - 1;
      const int first = group - before - __shfl_sync(0xffffffffu, sum - mine, l);
      ad = __shfl_sync(0xffffffffu, its, l);
      row0 = __shfl_sync(0xffffffffu, from, l) + first * tile;
      rows = min(tile, __shfl_sync(0xffffffffu, to, l) - row0);
      if (group + 1 == groups)                       // nobody else looks at the offsets behind these
        for (int i = b0 + 32 + lane; i < a.B; i += 32) bad |= a.row_offsets[i] < 0 || a.row_offsets[i + 1] < a.row_offsets[i] || a.row_offsets[i + 1] > a.max_rows;
      if (bad) set_status(a.status, SL_DEV_BAD_INDEX);
      return true;
    }
    before += __shfl_sync(0xffffffffu, sum, 31);
  }
  if (bad) set_status(a.status, SL_DEV_BAD_INDEX);
  return false;
}

// The rank of an adapter; false where there is nothing to add.
__device__ __forceinline__ bool find_rank(const AdapterArgs& a, int ad, int& rank) {
  if (ad < 0 || ad >= a.n_adapters) {
    if (ad >= a.n_adapters) set_status(a.status, SL_DEV_BAD_INDEX);
    return false;
  }
  rank = a.max_rank;
  if (a.ranks) {
    const int given = a.ranks[ad];
    if (given < 0 || given > a.max_rank) set_status(a.status, SL_DEV_BAD_INDEX);
    rank = min(max(given, 0), a.max_rank);
  }
  return rank > 0;
}

// t enters the second product as a sum of TERMS bf16 numbers.  next_term gives the first of what is left of v and takes it away: the upper 8 bits or, where
// these are all of it, its half; last_term the rest.  So the terms of a number have its sign and none is zero: with an infinite weight their products have one
// sign too, and sum up to the infinity that the number's product is (a term of zero, or of the other sign, would make it NaN); and no term of a
// number next to the end of fp32 is rounded to an infinity.  Their last bit is a quarter of the number's own last bit at least (an
// eighth, where the last term is halved once more), so sums that fp32 holds with three bits to spare stay exact.  The three are v itself where |v| >= 2^-108,
// and off by 2^-132 below.  Zero gives zeros, an infinity or a NaN itself.
constexpr int TERMS = 3;
__device__ __forceinline__ uint32_t next_term(float& v) {        // in the word's upper half
  float a = __uint_as_float(__float_as_uint(v) & 0xffff0000u);
  if (a == v) a = 0.5f * v;
  v = isinf(v) ? v : v - a;
  return __float_as_uint(a);
}
__device__ __forceinline__ uint32_t last_term(float v) { return __float_as_uint(v); }

int launch_gemm_adapters_tc(const AdapterArgs& a, int dtype, cudaStream_t st);

}  // namespace sl
