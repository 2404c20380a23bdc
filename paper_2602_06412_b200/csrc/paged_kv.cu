// Writing K/V rows into a paged cache, quantised on the way, and reading them back (the cache scatter of Algorithm 1
// line 11 and its inverse, for a cache in pages of 8-bit codes).
//
// One (row, head) of K or V has its own scale:  s = fp32(max_d |x_d| / Q)  (Q = 448 for e4m3, 127 for int8), and its codes
// are c_d = x_d / s rounded ONCE, to nearest even, from the exact quotient by the stored s.  Read back: c_d s, rounded
// once to 32 bits and, for a bf16 output, once more.  s = 0 (all zero) gives codes 0; a row with an infinity or a NaN gets
// s = NaN, so that everything read back of it is NaN.
//
// Exact rounding without a division per element: y = x * (1 / s) is within 2^-22 of the quotient (two roundings), so when
// y (1 + 2^-21) and y (1 - 2^-21) round to the same code, that is the code of the exact quotient too.  Otherwise (about one
// value in 10^5) the quotient is formed truncated with its lowest bit set when it is inexact ("round to odd"), whose
// rounding to a code's few bits is that of the exact value.  Rows below 2^-64 are first multiplied by 2^64 (exactly), so
// that 1 / s stays finite and the remainder in the odd rounding stays representable.
//
// Memory-bound: DH / 8 lanes take one (row, head) of K and of V, 8 elements a lane in 16-byte loads, all loads issued before
// the first use; the 8-byte stores of a half-warp (DH = 128) fill one 128-byte line, as one head's places in a page are
// contiguous.  Index chain (position -> page table -> slot) runs under the data loads.
#include "paged_kv.cuh"

namespace sl {

int check_paged_kv(const surelock_paged_kv* c) {
  if (!c || !c->k || !c->v || !c->page_table || c->n_pages <= 0 || c->max_pages <= 0 || c->n_kv_heads <= 0) return SL_EINVAL;
  if (c->dtype != SL_BF16 && c->dtype != SL_E4M3 && c->dtype != SL_INT8) return SL_EINVAL;
  if (c->dtype != SL_BF16 && (!c->k_scale || !c->v_scale)) return SL_EINVAL;
  if (c->page_size != 16 && c->page_size != 32 && c->page_size != 64 && c->page_size != 128 && c->page_size != 256)
    return SL_EUNSUPPORTED;
  if (c->head_dim != 64 && c->head_dim != 128) return SL_EUNSUPPORTED;
  if ((long long)c->max_pages * c->page_size > 0x7fffff00ll) return SL_EUNSUPPORTED;
  uintptr_t a = reinterpret_cast<uintptr_t>(c->k) | reinterpret_cast<uintptr_t>(c->v);
  if (c->dtype != SL_BF16) a |= reinterpret_cast<uintptr_t>(c->k_scale) | reinterpret_cast<uintptr_t>(c->v_scale);
  return (a & 15) ? SL_EUNSUPPORTED : SL_OK;
}

namespace {

constexpr int PK_THREADS = 256;

struct PagedArgs {
  void *k, *v;
  float *ks, *vs;
  const int32_t *table, *idx, *n_active;
  int n_pages, page_shift, max_pages, Hkv, B, N, max_rows;
  long long row_stride;
  int32_t* status;
};

// slot index ((page * Hkv + h) * page_size + place) of flat position f, or -1
__device__ __forceinline__ long long paged_slot(const PagedArgs& a, int f, int h) {
  if (f < 0) return -1;
  const int b = f / a.N, i = f - b * a.N;
  if (b >= a.B || (i >> a.page_shift) >= a.max_pages) return -1;
  const int page = __ldg(a.table + (long long)b * a.max_pages + (i >> a.page_shift));
  if ((unsigned)page >= (unsigned)a.n_pages) return -1;
  return ((((long long)page * a.Hkv + h)) << a.page_shift) + (i & ((1 << a.page_shift) - 1));
}

// 8 consecutive elements, widened
__device__ __forceinline__ void load8(const bf16* p, float* x) {
  const uint4 u = *reinterpret_cast<const uint4*>(p);
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void load8(const float* p, float* x) {
  const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
  x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
  x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
__device__ __forceinline__ uint32_t two_bf16(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ void store8(bf16* p, const float* x) {
  *reinterpret_cast<uint4*>(p) =
      make_uint4(two_bf16(x[0], x[1]), two_bf16(x[2], x[3]), two_bf16(x[4], x[5]), two_bf16(x[6], x[7]));
}
__device__ __forceinline__ void store8(float* p, const float* x) {
  *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
  *reinterpret_cast<float4*>(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
}

// four values -> four codes, lowest byte first; values beyond the largest code become it
template <int KIND> __device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d) {
  if (KIND == SL_E4M3) {
    uint16_t lo, hi;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
    return (uint32_t)lo | ((uint32_t)hi << 16);
  } else {
    auto one = [](float v) { return (uint32_t)(__float2int_rn(fminf(fmaxf(v, -127.f), 127.f)) & 0xff); };
    return one(a) | (one(b) << 8) | (one(c) << 16) | (one(d) << 24);
  }
}
// x / s truncated, lowest bit set when inexact: rounds to a shorter format as the exact quotient does
__device__ __noinline__ float quotient_to_odd(float x, float s) {
  const float q = __fdiv_rz(x, s);
  return __fmaf_rn(-q, s, x) != 0.f ? __uint_as_float(__float_as_uint(q) | 1u) : q;
}

// quantise the 8 elements of this lane; all LANES lanes of the (row, head) take part.  Returns the scale.
template <int KIND, int LANES> __device__ __forceinline__ float quantise8(float* x, uint2& out) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);   // orders like the magnitude, NaN above all
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
  out = make_uint2(0u, 0u);
  if (top >= 0x7f800000u) return __uint_as_float(0x7fffffffu);
  const float amax = __uint_as_float(top);
  const float scale = __fdiv_rn(amax, KvKind<KIND>::QMAX);
  if (scale == 0.f) return 0.f;
  float s = scale;
  if (amax < 5.421010862427522e-20f) {   // 2^-64
    s *= 18446744073709551616.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] *= 18446744073709551616.f;
  }
  const float inv = __fdiv_rn(1.f, s);
  constexpr float UP = 1.f + 4.76837158e-7f, DOWN = 1.f - 4.76837158e-7f;   // 1 +- 2^-21
  uint32_t c[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    float* p = x + 4 * h;
    const float y[4] = {p[0] * inv, p[1] * inv, p[2] * inv, p[3] * inv};
    c[h] = codes4<KIND>(y[0] * UP, y[1] * UP, y[2] * UP, y[3] * UP);
    if (c[h] != codes4<KIND>(y[0] * DOWN, y[1] * DOWN, y[2] * DOWN, y[3] * DOWN))
      c[h] = codes4<KIND>(quotient_to_odd(p[0], s), quotient_to_odd(p[1], s), quotient_to_odd(p[2], s), quotient_to_odd(p[3], s));
  }
  out = make_uint2(c[0], c[1]);
  return scale;
}

template <int KIND, int DH, typename T>
__global__ void __launch_bounds__(PK_THREADS)
kv_scatter_paged_kernel(PagedArgs a, const T* __restrict__ k, const T* __restrict__ v) {
  constexpr int LANES = DH / 8;
  griddep_wait();
  griddep_launch();
  const int M = min(*a.n_active, a.max_rows);
  const int lane = threadIdx.x % LANES;
  const long long items = (long long)M * a.Hkv, step = (long long)gridDim.x * (PK_THREADS / LANES);
  // the lanes of a warp stay together (they shuffle): the loop bound is taken for the warp's first item
  for (long long it = (long long)blockIdx.x * (PK_THREADS / LANES) + threadIdx.x / LANES;; it += step) {
    const long long first = it - (threadIdx.x % 32) / LANES;
    if (first >= items) return;
    const bool live = it < items;
    const long long w = live ? it : items - 1;
    const int r = (int)(w / a.Hkv), h = (int)(w - (long long)r * a.Hkv);
    const long long src = (long long)r * a.row_stride + (long long)h * DH + lane * 8;
    float xk[8], xv[8];
    load8(k + src, xk);
    load8(v + src, xv);
    const long long slot = paged_slot(a, __ldg(a.idx + r), h);
    if (live && slot < 0 && lane == 0 && h == 0) set_status(a.status, SL_DEV_BAD_INDEX);
    const bool put = live && slot >= 0;
    if (KIND == SL_BF16) {
      if (put) {
        store8((bf16*)a.k + slot * DH + lane * 8, xk);
        store8((bf16*)a.v + slot * DH + lane * 8, xv);
      }
    } else {
      uint2 ck, cv;
      const float sk = quantise8<KIND == SL_BF16 ? SL_E4M3 : KIND, LANES>(xk, ck);
      const float sv = quantise8<KIND == SL_BF16 ? SL_E4M3 : KIND, LANES>(xv, cv);
      if (put) {
        *reinterpret_cast<uint2*>((uint8_t*)a.k + slot * DH + lane * 8) = ck;
        *reinterpret_cast<uint2*>((uint8_t*)a.v + slot * DH + lane * 8) = cv;
        if (lane == 0) {
          a.ks[slot] = sk;
          a.vs[slot] = sv;
        }
      }
    }
  }
}

template <int KIND> __device__ __forceinline__ void dequantise8(uint2 c, float s, float* x) {
  const uint32_t w[2] = {c.x, c.y};
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if (KIND == SL_E4M3) {
      const uint32_t lo = e4m3x2_to_f16x2((uint16_t)(w[h] & 0xffffu)), hi = e4m3x2_to_f16x2((uint16_t)(w[h] >> 16));
      const float2 f0 = __half22float2(*reinterpret_cast<const __half2*>(&lo)), f1 = __half22float2(*reinterpret_cast<const __half2*>(&hi));
      x[4 * h] = f0.x * s; x[4 * h + 1] = f0.y * s; x[4 * h + 2] = f1.x * s; x[4 * h + 3] = f1.y * s;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) x[4 * h + i] = (float)(int8_t)(w[h] >> (8 * i)) * s;
    }
  }
}

template <int KIND, int DH, typename T>
__global__ void __launch_bounds__(PK_THREADS) kv_gather_paged_kernel(PagedArgs a, T* __restrict__ k, T* __restrict__ v) {
  constexpr int LANES = DH / 8;
  griddep_wait();
  griddep_launch();
  const int M = min(*a.n_active, a.max_rows);
  const int lane = threadIdx.x % LANES;
  const long long items = (long long)M * a.Hkv, step = (long long)gridDim.x * (PK_THREADS / LANES);
  for (long long it = (long long)blockIdx.x * (PK_THREADS / LANES) + threadIdx.x / LANES; it < items; it += step) {
    const int r = (int)(it / a.Hkv), h = (int)(it - (long long)r * a.Hkv);
    const long long slot = paged_slot(a, __ldg(a.idx + r), h);
    float xk[8] = {}, xv[8] = {};
    if (slot < 0) {
      if (lane == 0 && h == 0) set_status(a.status, SL_DEV_BAD_INDEX);
    } else if (KIND == SL_BF16) {
      load8((const bf16*)a.k + slot * DH + lane * 8, xk);
      load8((const bf16*)a.v + slot * DH + lane * 8, xv);
    } else {
      const uint2 ck = *reinterpret_cast<const uint2*>((const uint8_t*)a.k + slot * DH + lane * 8);
      const uint2 cv = *reinterpret_cast<const uint2*>((const uint8_t*)a.v + slot * DH + lane * 8);
      const float sk = a.ks[slot], sv = a.vs[slot];
      dequantise8<KIND == SL_BF16 ? SL_E4M3 : KIND>(ck, sk, xk);
      dequantise8<KIND == SL_BF16 ? SL_E4M3 : KIND>(cv, sv, xv);
    }
    const long long dst = (long long)r * a.row_stride + (long long)h * DH + lane * 8;
    store8(k + dst, xk);
    store8(v + dst, xv);
  }
}

PagedArgs paged_args(const surelock_paged_kv& c, const int32_t* idx, const int32_t* n_active, int max_rows, int B, int N,
                     long long row_stride, int32_t* status) {
  PagedArgs a;
  a.k = c.k; a.v = c.v; a.ks = c.k_scale; a.vs = c.v_scale;
  a.table = c.page_table; a.idx = idx; a.n_active = n_active;
  a.n_pages = c.n_pages; a.max_pages = c.max_pages; a.Hkv = c.n_kv_heads;
  a.page_shift = 0;
  while ((1 << a.page_shift) < c.page_size) ++a.page_shift;
  a.B = B; a.N = N; a.max_rows = max_rows; a.row_stride = row_stride; a.status = status;
  return a;
}

int paged_grid(const surelock_paged_kv& c, int max_rows) {
  const long long groups = PK_THREADS / (c.head_dim / 8);
  const long long want = ((long long)max_rows * c.n_kv_heads + groups - 1) / groups;
  const long long cap = (long long)sm_count() * 16;
  return (int)(want < 1 ? 1 : want > cap ? cap : want);
}

template <int KIND, int DH>
int scatter_kind(const surelock_paged_kv& c, const PagedArgs& a, const void* k, const void* v, int dtype, cudaStream_t st) {
  const dim3 g(paged_grid(c, a.max_rows));
  if (dtype == SL_BF16)
    SL_CUDA_TRY(launch_pdl(kv_scatter_paged_kernel<KIND, DH, bf16>, g, dim3(PK_THREADS), 0, st, a, (const bf16*)k, (const bf16*)v));
  else
    SL_CUDA_TRY(launch_pdl(kv_scatter_paged_kernel<KIND, DH, float>, g, dim3(PK_THREADS), 0, st, a, (const float*)k, (const float*)v));
  return SL_OK;
}

template <int KIND, int DH>
int gather_kind(const surelock_paged_kv& c, const PagedArgs& a, void* k, void* v, int dtype, cudaStream_t st) {
  const dim3 g(paged_grid(c, a.max_rows));
  if (dtype == SL_BF16)
    SL_CUDA_TRY(launch_pdl(kv_gather_paged_kernel<KIND, DH, bf16>, g, dim3(PK_THREADS), 0, st, a, (bf16*)k, (bf16*)v));
  else
    SL_CUDA_TRY(launch_pdl(kv_gather_paged_kernel<KIND, DH, float>, g, dim3(PK_THREADS), 0, st, a, (float*)k, (float*)v));
  return SL_OK;
}

}  // namespace

#define SL_BY_KIND(F, ...)                                                                                    \
  (c.dtype == SL_BF16   ? (c.head_dim == 128 ? F<SL_BF16, 128>(__VA_ARGS__) : F<SL_BF16, 64>(__VA_ARGS__))    \
   : c.dtype == SL_E4M3 ? (c.head_dim == 128 ? F<SL_E4M3, 128>(__VA_ARGS__) : F<SL_E4M3, 64>(__VA_ARGS__))    \
                        : (c.head_dim == 128 ? F<SL_INT8, 128>(__VA_ARGS__) : F<SL_INT8, 64>(__VA_ARGS__)))

int launch_kv_scatter_paged(const surelock_paged_kv& c, const void* k, const void* v, long long row_stride, const int32_t* idx,
                            const int32_t* n_active, int max_rows, int B, int N, int dtype, int32_t* status, cudaStream_t st) {
  const PagedArgs a = paged_args(c, idx, n_active, max_rows, B, N, row_stride, status);
  return SL_BY_KIND(scatter_kind, c, a, k, v, dtype, st);
}

int launch_kv_gather_paged(const surelock_paged_kv& c, const int32_t* idx, const int32_t* n_active, int max_rows, int B, int N,
                           void* k, void* v, long long row_stride, int dtype, int32_t* status, cudaStream_t st) {
  const PagedArgs a = paged_args(c, idx, n_active, max_rows, B, N, row_stride, status);
  return SL_BY_KIND(gather_kind, c, a, k, v, dtype, st);
}

}  // namespace sl
