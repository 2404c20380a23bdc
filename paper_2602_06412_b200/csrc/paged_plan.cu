// Page tables, row offsets and flat positions of a paged cache from the lengths of its sequences: the integer work in front
// of a served step (surelock_paged_extend) and after one whose tokens are given up (surelock_paged_truncate).
//
// With P tokens to a page, sequence b of length L_b gets n_b tokens and needs  ceil((L_b + n_b) / P) - ceil(L_b / P)  pages
// of the free list.  Two prefix sums over the sequences say who is served (first come, first served) and where everyone's
// pages and rows begin; then every row and every page finds its sequence by bisection in shared memory, so that ragged
// lengths cost nothing.  One thread per sequence in every CTA: each CTA does the sums by itself and writes its share of rows.
//
// Bounded by latency: start, one round of loads, the sums, one round of stores.  In a graph, the replay's 4.1 us among it: 32 sequences of one
// token 4.2 us, 8 prompts of up to 1536 tokens 6.3, 32 sequences cut 4.1, 900 cut 8.4.  One CTA or a cluster of 8, us: 1 x 4096 tokens 4.3 / 6.3, 32 x
// 128 6.3 / 6.3, 64 x 128 12.4 / 6.3; cut: 32 sequences of 64 places 4.2 / 4.3, 64 of 65 6.2 / 4.2, 900 of 127 31 / 8.4.  So a cluster beyond 4096.
#include "paged_kv.cuh"
#include "tc_common.cuh"

namespace sl {
namespace {

constexpr int PLAN_THREADS = 1024, PLAN_CLUSTER = 8;

struct PlanArgs {
  int32_t* table;
  const int32_t *seq_lens, *want, *n_free;
  int32_t *free_pages, *row_offsets, *active_idx, *n_active, *seq_lens_out, *n_free_out, *status;
  int B, page_shift, max_pages, n_pages, max_rows;
};

__device__ __forceinline__ int pages_of(long long tokens, int shift) { return (int)((tokens + (1 << shift) - 1) >> shift); }

// inclusive sums of two values over the block's threads in one go; `part`: 64 words
__device__ __forceinline__ void scan2(long long& a, long long& b, long long* part) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long x = __shfl_up_sync(0xffffffffu, a, o), y = __shfl_up_sync(0xffffffffu, b, o);
    if (lane >= o) {
      a += x;
      b += y;
    }
  }
  if (lane == 31) {
    part[warp] = a;
    part[32 + warp] = b;
  }
  __syncthreads();
  if (warp == 0) {
    long long x = lane < (int)(blockDim.x >> 5) ? part[lane] : 0, y = lane < (int)(blockDim.x >> 5) ? part[32 + lane] : 0;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long u = __shfl_up_sync(0xffffffffu, x, o), v = __shfl_up_sync(0xffffffffu, y, o);
      if (lane >= o) {
        x += u;
        y += v;
      }
    }
    part[lane] = x;
    part[32 + lane] = y;
  }
  __syncthreads();
  if (warp) {
    a += part[warp - 1];
    b += part[32 + warp - 1];
  }
}

// the sequence whose share of [0, first[n]) holds i: the last one that begins at or before i
__device__ __forceinline__ int share_of(const int* first, int n, int i) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int m = (lo + hi) >> 1;
    if (first[m] <= i) lo = m; else hi = m;
  }
  return lo;
}

// CTAS > 1: one cluster of that many CTAs, which all read before any of them writes (lengths may be updated in place)
template <int CTAS> __device__ __forceinline__ void everyone_has_read() {
  if (CTAS > 1) cluster_sync_all(); else __syncthreads();
}

template <int CTAS>
__global__ void __launch_bounds__(PLAN_THREADS) paged_extend_kernel(PlanArgs a) {
  __shared__ long long part[64];
  __shared__ int s_row[PLAN_THREADS + 1], s_page[PLAN_THREADS + 1], s_len[PLAN_THREADS], s_have[PLAN_THREADS];
  griddep_wait();
  griddep_launch();
  const int t = threadIdx.x, cta = CTAS > 1 ? (int)blockIdx.x : 0, threads = (int)blockDim.x;
  const long long N = (long long)a.max_pages << a.page_shift;
  int n_free = *a.n_free, len = 0, fresh = 0;
  bool bad = n_free < 0 || n_free > a.n_pages;
  n_free = min(max(n_free, 0), a.n_pages);
  if (t < a.B) {
    len = a.seq_lens[t];
    fresh = a.want[t];
    bad |= len < 0 || len > N || fresh < 0;
    len = (int)min(max((long long)len, 0ll), N);
    fresh = max(fresh, 0);
  }
  const bool fits = (long long)len + fresh <= N;
  const int have = pages_of(len, a.page_shift), need = fits ? pages_of((long long)len + fresh, a.page_shift) - have : 0;
  // who is served: sums that stop counting just above what there is
  long long pages = min((long long)need, n_free + 1ll), rows = fits ? min((long long)fresh, a.max_rows + 1ll) : 0;
  scan2(pages, rows, part);
  const bool ok = fits && (need == 0 || pages <= n_free) && rows <= a.max_rows;
  __syncthreads();                                   // part is used again
  pages = ok ? need : 0;
  rows = ok ? fresh : 0;
  scan2(pages, rows, part);
  if (t == 0) s_row[0] = s_page[0] = 0;
  s_row[t + 1] = (int)rows;
  s_page[t + 1] = (int)pages;
  s_len[t] = len;
  s_have[t] = have;
  everyone_has_read<CTAS>();
  const int M = s_row[threads], taken = s_page[threads];
  if (bad) set_status(a.status, SL_DEV_BAD_INDEX);
  if (cta == 0) {
    if (t < a.B) {
      a.seq_lens_out[t] = len + (ok ? fresh : 0);
      a.row_offsets[t + 1] = (int)rows;
    }
    if (t == 0) {
      a.row_offsets[0] = 0;
      *a.n_active = M;
      *a.n_free_out = n_free - taken;
    }
  }
  for (int j = cta * threads + t; j < taken; j += CTAS * threads) {
    const int b = share_of(s_page, a.B, j), page = a.free_pages[n_free - 1 - j];
    if ((unsigned)page >= (unsigned)a.n_pages) set_status(a.status, SL_DEV_BAD_INDEX);
    a.table[(long long)b * a.max_pages + s_have[b] + j - s_page[b]] = page;
  }
  for (int r = cta * threads + t; r < M; r += CTAS * threads) {
    const int b = share_of(s_row, a.B, r);
    a.active_idx[r] = b * (int)N + s_len[b] + r - s_row[b];
  }
}

template <int CTAS>
__global__ void __launch_bounds__(PLAN_THREADS) paged_truncate_kernel(PlanArgs a) {
  __shared__ long long part[64];
  __shared__ long long s_page[PLAN_THREADS + 1];
  __shared__ int s_first[PLAN_THREADS];
  griddep_wait();
  griddep_launch();
  const int t = threadIdx.x, cta = CTAS > 1 ? (int)blockIdx.x : 0, threads = (int)blockDim.x;
  const long long N = (long long)a.max_pages << a.page_shift;
  int n_free = *a.n_free, len = 0, keep = 0;
  bool bad = n_free < 0 || n_free > a.n_pages;
  n_free = min(max(n_free, 0), a.n_pages);
  if (t < a.B) {
    len = a.seq_lens[t];
    keep = a.want[t];
    bad |= len < 0 || len > N || keep < 0;
    len = (int)min(max((long long)len, 0ll), N);
    keep = min(max(keep, 0), len);
  }
  const int first = pages_of(keep, a.page_shift);
  long long pages = pages_of(len, a.page_shift) - first, none = 0;
  scan2(pages, none, part);
  if (t == 0) s_page[0] = 0;
  s_page[t + 1] = pages;
  s_first[t] = first;
  everyone_has_read<CTAS>();
  const long long all = s_page[threads], room = a.n_pages - n_free;
  const int given = (int)min(all, room);             // more than there is room for: a page is on two tables
  bad |= all > room;
  if (bad) set_status(a.status, SL_DEV_BAD_INDEX);
  if (cta == 0) {
    if (t < a.B) a.seq_lens_out[t] = keep;
    if (t == 0) *a.n_free_out = n_free + given;
  }
  for (int j = cta * threads + t; j < given; j += CTAS * threads) {
    int lo = 0, hi = a.B;
    while (hi - lo > 1) {
      const int m = (lo + hi) >> 1;
      if (s_page[m] <= j) lo = m; else hi = m;
    }
    const int page = a.table[(long long)lo * a.max_pages + s_first[lo] + (int)(j - s_page[lo])];
    if ((unsigned)page >= (unsigned)a.n_pages) set_status(a.status, SL_DEV_BAD_INDEX);
    a.free_pages[n_free + j] = page;
  }
}

template <typename Kernel>
int launch_plan(Kernel kernel, int ctas, const PlanArgs& a, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(ctas);
  cfg.blockDim = dim3(ctas > 1 ? PLAN_THREADS : a.B <= 128 ? 256 : PLAN_THREADS);
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = ctas;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = pdl_enabled() ? 2 : 1;
  SL_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, a));
  return SL_OK;
}

}  // namespace

int launch_paged_extend(int32_t* table, int B, int page_size, int max_pages, int n_pages, const int32_t* seq_lens, const int32_t* want,
                        const int32_t* free_pages, const int32_t* n_free, int32_t* row_offsets, int32_t* active_idx, int32_t* n_active,
                        int max_rows, int32_t* seq_lens_out, int32_t* n_free_out, int32_t* status, cudaStream_t st) {
  PlanArgs a = {table, seq_lens, want, n_free, const_cast<int32_t*>(free_pages), row_offsets, active_idx, n_active, seq_lens_out,
                n_free_out, status, B, 0, max_pages, n_pages, max_rows};
  while ((1 << a.page_shift) < page_size) ++a.page_shift;
  return max_rows <= 4 * PLAN_THREADS ? launch_plan(paged_extend_kernel<1>, 1, a, st)
                                      : launch_plan(paged_extend_kernel<PLAN_CLUSTER>, PLAN_CLUSTER, a, st);
}

int launch_paged_truncate(const int32_t* table, int B, int page_size, int max_pages, int n_pages, const int32_t* seq_lens,
                          const int32_t* keep, int32_t* free_pages, const int32_t* n_free, int32_t* seq_lens_out, int32_t* n_free_out,
                          int32_t* status, cudaStream_t st) {
  PlanArgs a = {const_cast<int32_t*>(table), seq_lens, keep, n_free, free_pages, nullptr, nullptr, nullptr, seq_lens_out, n_free_out,
                status, B, 0, max_pages, n_pages, 0};
  while ((1 << a.page_shift) < page_size) ++a.page_shift;
  return (long long)B * max_pages <= 4 * PLAN_THREADS ? launch_plan(paged_truncate_kernel<1>, 1, a, st)
                                                       : launch_plan(paged_truncate_kernel<PLAN_CLUSTER>, PLAN_CLUSTER, a, st);
}

}  // namespace sl
