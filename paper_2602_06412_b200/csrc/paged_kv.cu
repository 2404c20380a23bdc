// Writing K/V rows into a paged cache, quantised on the way, and reading them back (the cache scatter of Algorithm 1
// line 11 and its inverse, for a cache in pages of 8-bit codes).
//
// One (row, head) of K or V has its own scale:  s = fp32(max_d |x_d| / Q)  (Q = 448 for e4m3, 127 for int8), and its codes
// are c_d = x_d / s rounded ONCE, to nearest even, from the exact quotient by the stored s.  Read back: c_d s, rounded
// once to 32 bits and, for a bf16 output, once more.  s = 0 (all zero) gives codes 0; a row with an infinity or a NaN gets
// s = NaN, so that everything read back of it is NaN.
//
// Exact rounding without a division per element.  For fp32 inputs: x times an approximate 1 / s (2^-23) is within 2^-22 of
// the quotient, so when the products by (1 + 2^-21) / s and (1 - 2^-21) / s round to the same code, that is the code of the
// exact quotient too.  Otherwise the sign of x - b s, b the border between the two codes, settles it: one fma, so the sign is
// exact.  Rows below 2^-64 are first multiplied by 2^64 (exactly), so that 1 / s is a normal number and x - b s does not
// underflow.
// For bf16 inputs the sign is the same for a whole (row, head).  With significands m of 8 bits, x Q / amax is a border b (odd
// significand below 2^5 for e4m3, 2^8 for int8) or at least 1 / (m_amax m_b) > 2^-16 away from it, relatively; and x / s =
// (x Q / amax) (1 + rho / (Q s)) with rho = amax - Q s, which one fma gives.  So x times (1 + sign(rho) 2^-18) / s rounds like
// the quotient; where rho = 0 a residual step makes x / s exact where it is a border.  (12288 rows of 32 heads, e4m3: 77 us
// with the two products for bf16 too, as borders are common there: where amax has a factor 7, one value in 16.)
//
// Memory-bound: DH / 8 lanes take one (row, head) of K and of V, 8 elements a lane in 16-byte loads, all loads issued before
// the first use; the 8-byte stores of a half-warp (DH = 128) fill one 128-byte line, as one head's places in a page are
// contiguous.  Index chain (position -> page table -> slot) runs under the data loads.
// Measured in replayed graphs, 32 heads of 128: 12288 rows written from bf16 to e4m3 / int8 / bf16 pages 52 / 53 / 62 us (5.9 / 5.7 / 6.5
// TB/s), from fp32 82 / 84 / 89 us (6.2 / 6.0 / 6.8 TB/s); 6144 rows read back to bf16 27 / 29 / 33 us (5.6 / 5.2 / 6.0 TB/s), to fp32 56 / 58 /
// 59 us (4.5 / 4.3 / 5.2 TB/s).  Calls made one by one take 5 - 6 us more.
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
constexpr int PK_SCATTER_BLOCKS = 6, PK_GATHER_BLOCKS = 8;   // per SM

struct PagedArgs {
  void *k, *v;
  float *ks, *vs;
  const int32_t *table, *idx, *n_active;
  int n_pages, page_shift, max_pages, Hkv, B, N, max_rows;
  int parts;                    // parts of a row, U heads each
  uint32_t div_parts, div_n;    // ceil(2^32 / parts), ceil(2^32 / N): see fast_div
  long long row_stride;
  int32_t* status;
};

// x / d by the reciprocal m = ceil(2^32 / d) (0 for d = 1): the product is the quotient or one more
__device__ __forceinline__ unsigned fast_div(unsigned x, unsigned d, unsigned m) {
  if (m == 0) return x;
  const unsigned q = __umulhi(x, m);
  return q * d > x ? q - 1 : q;
}
// slot index ((page * Hkv + h) * page_size + place) of flat position f, or -1
__device__ __forceinline__ long long paged_slot(const PagedArgs& a, int f, int h) {
  if (f < 0) return -1;
  const int b = (int)fast_div((unsigned)f, (unsigned)a.N, a.div_n), i = f - b * a.N;
  if (b >= a.B || (i >> a.page_shift) >= a.max_pages) return -1;
  const int page = __ldg(a.table + (long long)b * a.max_pages + (i >> a.page_shift));
  if ((unsigned)page >= (unsigned)a.n_pages) return -1;
  return ((((long long)page * a.Hkv + h)) << a.page_shift) + (i & ((1 << a.page_shift) - 1));
}

// 8 consecutive elements as they are stored
template <typename T> struct Raw8;
template <> struct Raw8<bf16> { uint4 u; };
template <> struct Raw8<float> { uint4 u, w; };
__device__ __forceinline__ void load8(const bf16* p, Raw8<bf16>& r) { r.u = *reinterpret_cast<const uint4*>(p); }
__device__ __forceinline__ void load8(const float* p, Raw8<float>& r) {
  r.u = *reinterpret_cast<const uint4*>(p);
  r.w = *reinterpret_cast<const uint4*>(p + 4);
}
__device__ __forceinline__ void widen8(const Raw8<bf16>& r, float* x) {
  const uint32_t w[4] = {r.u.x, r.u.y, r.u.z, r.u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void widen8(const Raw8<float>& r, float* x) {
  const uint32_t w[8] = {r.u.x, r.u.y, r.u.z, r.u.w, r.w.x, r.w.y, r.w.z, r.w.w};
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(w[i]);
}
// bits of the largest magnitudes of K's and of V's elements over the lanes of a (row, head) (magnitudes order like their
// bits, NaN above all); bf16 pairs are compared two at a time, and K's and V's go through the shuffles together
template <int LANES> __device__ __forceinline__ void tops(const Raw8<bf16>& k, const Raw8<bf16>& v, uint32_t& tk, uint32_t& tv) {
  auto top = [](uint32_t x, uint32_t y) {            // of magnitudes, two at a time; a NaN stays one
    const __nv_bfloat162 m = __hmax2_nan(*reinterpret_cast<__nv_bfloat162*>(&x), *reinterpret_cast<__nv_bfloat162*>(&y));
    return *reinterpret_cast<const uint32_t*>(&m);
  };
  constexpr uint32_t A = 0x7fff7fffu;
  const uint32_t a = top(top(k.u.x & A, k.u.y & A), top(k.u.z & A, k.u.w & A));
  const uint32_t b = top(top(v.u.x & A, v.u.y & A), top(v.u.z & A, v.u.w & A));
  uint32_t both = top(__byte_perm(a, b, 0x5410), __byte_perm(a, b, 0x7632));
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) both = top(both, __shfl_xor_sync(0xffffffffu, both, o));
  tk = both << 16;
  tv = both & 0xffff0000u;
}
template <int LANES> __device__ __forceinline__ void tops(const Raw8<float>& k, const Raw8<float>& v, uint32_t& tk, uint32_t& tv) {
  constexpr uint32_t A = 0x7fffffffu;
  tk = max(max(max(k.u.x & A, k.u.y & A), max(k.u.z & A, k.u.w & A)), max(max(k.w.x & A, k.w.y & A), max(k.w.z & A, k.w.w & A)));
  tv = max(max(max(v.u.x & A, v.u.y & A), max(v.u.z & A, v.u.w & A)), max(max(v.w.x & A, v.w.y & A), max(v.w.z & A, v.w.w & A)));
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) {
    tk = max(tk, __shfl_xor_sync(0xffffffffu, tk, o));
    tv = max(tv, __shfl_xor_sync(0xffffffffu, tv, o));
  }
}
// x[0..3] * f, two products to an instruction
__device__ __forceinline__ void mul4(const float* x, float f, float* y) {
#pragma unroll
  for (int i = 0; i < 4; i += 2)
    asm("{\n\t.reg .b64 a, b, c;\n\t"
        "mov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %4};\n\t"
        "mul.rn.f32x2 c, a, b;\n\tmov.b64 {%0, %1}, c;\n\t}"
        : "=f"(y[i]), "=f"(y[i + 1]) : "f"(x[i]), "f"(x[i + 1]), "f"(f));
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

// four values -> four codes, lowest byte first.  e4m3: values beyond the largest code become it.  int8: |value| < 127.5; adding
// 1.5 x 2^23 rounds to a whole number, to nearest even, and leaves it in the low byte.
template <int KIND> __device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d) {
  if (KIND == SL_E4M3) {
    uint16_t lo, hi;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
    return (uint32_t)lo | ((uint32_t)hi << 16);
  } else {
    constexpr float R = 12582912.f;
    const uint32_t lo = __byte_perm(__float_as_uint(a + R), __float_as_uint(b + R), 0x0040);
    const uint32_t hi = __byte_perm(__float_as_uint(c + R), __float_as_uint(d + R), 0x0040);
    return __byte_perm(lo, hi, 0x5410);
  }
}
// the numbers that four codes stand for
template <int KIND> __device__ __forceinline__ void values4(uint32_t c, float* v) {
  if (KIND == SL_E4M3) {
    const uint32_t lo = e4m3x2_to_f16x2((uint16_t)(c & 0xffffu)), hi = e4m3x2_to_f16x2((uint16_t)(c >> 16));
    const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&lo)), b = __half22float2(*reinterpret_cast<const __half2*>(&hi));
    v[0] = a.x; v[1] = a.y; v[2] = b.x; v[3] = b.y;
  } else {
    // code + 128 as the low byte of 2^23 + (code + 128)
    const uint32_t u = c ^ 0x80808080u;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(__byte_perm(u, 0x4b000000u, 0x7440 + i)) - 8388736.f;
  }
}
// the codes of the exact quotients x / s, which lie between those of `low` and `high` (neighbours or the same): on which side
// of the border b between the two is told by the sign of x - b s, which one fma gives exactly; on the border the conversion
// takes the even one
template <int KIND> __device__ __forceinline__ uint32_t settle4(const float* x, float s, uint32_t low, uint32_t high) {
  float a[4], b[4];
  values4<KIND>(low, a);
  values4<KIND>(high, b);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    b[i] = 0.5f * (a[i] + b[i]);
    const float r = fmaf(-b[i], s, x[i]), step = fabsf(b[i]) * 9.5367431640625e-7f;   // 2^-20
    b[i] += r > 0.f ? step : r < 0.f ? -step : 0.f;
  }
  return codes4<KIND>(b[0], b[1], b[2], b[3]);
}

// amax / Q, correctly rounded, for amax >= 2^-64: one residual step from amax * RN(1 / Q) (Markstein's theorem; nothing
// underflows there)
template <int KIND> __device__ __forceinline__ float scale_of(float amax) {
  constexpr float Q = KvKind<KIND>::QMAX, RQ = 1.f / Q;
  const float q = amax * RQ;
  return __fmaf_rn(__fmaf_rn(-q, Q, amax), RQ, q);
}
__device__ __forceinline__ float about_inverse(float s) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(s));
  return r;
}

// quantise the 8 elements of this lane; top = bits of the largest magnitude of the whole (row, head).  Returns the scale.
template <int KIND> __device__ __forceinline__ float quantise8(float* x, uint32_t top, uint2& out) {
  constexpr float Q = KvKind<KIND>::QMAX;
  out = make_uint2(0u, 0u);
  if (top >= 0x7f800000u) return __uint_as_float(0x7fffffffu);
  const float amax = __uint_as_float(top);
  float scale, s;
  if (top >= 0x1f800000u) {   // 2^-64
    scale = s = scale_of<KIND>(amax);
  } else {
    scale = __fdiv_rn(amax, Q);
    if (scale == 0.f) return 0.f;
    s = scale * 18446744073709551616.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = fminf(fmaxf(x[i] * 18446744073709551616.f, -Q * s), Q * s);   // a subnormal scale may be far from amax / Q
  }
  const float inv = about_inverse(s);
  const float up = inv * (1.f + 4.76837158e-7f), down = inv * (1.f - 4.76837158e-7f);   // 1 +- 2^-21
  uint32_t c[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const float* p = x + 4 * h;
    float y[4], z[4];
    mul4(p, up, y);
    mul4(p, down, z);
    c[h] = codes4<KIND>(y[0], y[1], y[2], y[3]);
    const uint32_t other = codes4<KIND>(z[0], z[1], z[2], z[3]);
    if (c[h] != other) c[h] = settle4<KIND>(p, s, other, c[h]);
  }
  out = make_uint2(c[0], c[1]);
  return scale;
}
template <int KIND> __device__ __forceinline__ float quantise8(const Raw8<float>& r, uint32_t top, uint2& out) {
  float x[8];
  widen8(r, x);
  return quantise8<KIND>(x, top, out);
}
template <int KIND> __device__ __forceinline__ float quantise8(const Raw8<bf16>& r, uint32_t top, uint2& out) {
  float x[8], y[8];
  widen8(r, x);
  if (top < 0x1f800000u || top >= 0x7f800000u) return quantise8<KIND>(x, top, out);
  const float s = scale_of<KIND>(__uint_as_float(top)), rho = __fmaf_rn(-s, KvKind<KIND>::QMAX, __uint_as_float(top));
  const float inv = about_inverse(s), f = rho > 0.f ? inv * (1.f + 3.81469727e-6f) : rho < 0.f ? inv * (1.f - 3.81469727e-6f) : inv;   // 1 +- 2^-18
  mul4(x, f, y);
  mul4(x + 4, f, y + 4);
  if (rho == 0.f) {
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = fmaf(fmaf(-y[i], s, x[i]), inv, y[i]);
  }
  out = make_uint2(codes4<KIND>(y[0], y[1], y[2], y[3]), codes4<KIND>(y[4], y[5], y[6], y[7]));
  return s;
}

template <int KIND, int DH, int U, typename T>
__global__ void __launch_bounds__(PK_THREADS, sizeof(T) == 2 ? PK_SCATTER_BLOCKS : 1)
kv_scatter_paged_kernel(PagedArgs a, const T* __restrict__ k, const T* __restrict__ v) {
  constexpr int LANES = DH / 8;
  constexpr int QK = KIND == SL_BF16 ? SL_E4M3 : KIND;
  griddep_wait();
  griddep_launch();
  const int M = min(*a.n_active, a.max_rows);
  const int lane = threadIdx.x % LANES;
  const unsigned items = (unsigned)max(M, 0) * a.parts, step = gridDim.x * (PK_THREADS / LANES);
  // the lanes of a warp stay together (they shuffle): the loop bound is taken for the warp's first item
  for (unsigned it = blockIdx.x * (PK_THREADS / LANES) + threadIdx.x / LANES;; it += step) {
    if (it - (threadIdx.x % 32) / LANES >= items) return;
    const bool live = it < items;
    const unsigned w = live ? it : items - 1, r = fast_div(w, a.parts, a.div_parts), h = (w - r * a.parts) * U;
    const int heads = min(U, a.Hkv - (int)h);
    const long long src = r * a.row_stride + (long long)h * DH + lane * 8;
    Raw8<T> rk[U], rv[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long long from = src + (u < heads ? u * DH : 0);
      load8(k + from, rk[u]);
      load8(v + from, rv[u]);
    }
    const long long slot = paged_slot(a, __ldg(a.idx + r), h);
    if (live && slot < 0 && lane == 0 && h == 0) set_status(a.status, SL_DEV_BAD_INDEX);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool put = live && slot >= 0 && u < heads;
      const long long to = slot + ((long long)u << a.page_shift);
      if (KIND == SL_BF16) {
        if (put) {
          float xk[8], xv[8];
          widen8(rk[u], xk);
          widen8(rv[u], xv);
          store8((bf16*)a.k + to * DH + lane * 8, xk);
          store8((bf16*)a.v + to * DH + lane * 8, xv);
        }
      } else {
        uint32_t tk, tv;
        tops<LANES>(rk[u], rv[u], tk, tv);
        uint2 ck, cv;
        const float sk = quantise8<QK>(rk[u], tk, ck), sv = quantise8<QK>(rv[u], tv, cv);
        if (put) {
          *reinterpret_cast<uint2*>((uint8_t*)a.k + to * DH + lane * 8) = ck;
          *reinterpret_cast<uint2*>((uint8_t*)a.v + to * DH + lane * 8) = cv;
          if (lane == 0) {
            a.ks[to] = sk;
            a.vs[to] = sv;
          }
        }
      }
    }
  }
}

template <int KIND> __device__ __forceinline__ void dequantise8(uint2 c, float s, float* x) {
  values4<KIND>(c.x, x);
  values4<KIND>(c.y, x + 4);
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] *= s;
}

template <int KIND, int DH, int U, typename T>
__global__ void __launch_bounds__(PK_THREADS, PK_GATHER_BLOCKS) kv_gather_paged_kernel(PagedArgs a, T* __restrict__ k, T* __restrict__ v) {
  constexpr int LANES = DH / 8;
  constexpr int QK = KIND == SL_BF16 ? SL_E4M3 : KIND;
  griddep_wait();
  griddep_launch();
  const int M = min(*a.n_active, a.max_rows);
  const int lane = threadIdx.x % LANES;
  const unsigned items = (unsigned)max(M, 0) * a.parts, step = gridDim.x * (PK_THREADS / LANES);
  for (unsigned it = blockIdx.x * (PK_THREADS / LANES) + threadIdx.x / LANES; it < items; it += step) {
    const unsigned r = fast_div(it, a.parts, a.div_parts), h = (it - r * a.parts) * U;
    const int heads = min(U, a.Hkv - (int)h);
    const long long slot = paged_slot(a, __ldg(a.idx + r), h), dst = r * a.row_stride + (long long)h * DH + lane * 8;
    if (slot < 0 && lane == 0 && h == 0) set_status(a.status, SL_DEV_BAD_INDEX);
    if (KIND == SL_BF16) {
      Raw8<bf16> rk[U], rv[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        rk[u].u = rv[u].u = make_uint4(0u, 0u, 0u, 0u);
        if (slot >= 0 && u < heads) {
          const long long from = (slot + ((long long)u << a.page_shift)) * DH + lane * 8;
          load8((const bf16*)a.k + from, rk[u]);
          load8((const bf16*)a.v + from, rv[u]);
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (u < heads) {
          float x[8];
          widen8(rk[u], x);
          store8(k + dst + u * DH, x);
          widen8(rv[u], x);
          store8(v + dst + u * DH, x);
        }
    } else {
      uint2 ck[U], cv[U];
      float sk[U], sv[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        ck[u] = cv[u] = make_uint2(0u, 0u);
        sk[u] = sv[u] = 0.f;
        if (slot >= 0 && u < heads) {
          const long long from = slot + ((long long)u << a.page_shift);
          ck[u] = *reinterpret_cast<const uint2*>((const uint8_t*)a.k + from * DH + lane * 8);
          cv[u] = *reinterpret_cast<const uint2*>((const uint8_t*)a.v + from * DH + lane * 8);
          sk[u] = a.ks[from];
          sv[u] = a.vs[from];
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (u < heads) {
          float x[8];
          dequantise8<QK>(ck[u], sk[u], x);
          store8(k + dst + u * DH, x);
          dequantise8<QK>(cv[u], sv[u], x);
          store8(v + dst + u * DH, x);
        }
    }
  }
}

// ceil(2^32 / d), 0 for d = 1
uint32_t fast_div_by(int d) { return d == 1 ? 0u : (uint32_t)(0x100000000ull / d + (0x100000000ull % d != 0)); }

PagedArgs paged_args(const surelock_paged_kv& c, const int32_t* idx, const int32_t* n_active, int max_rows, int B, int N,
                     long long row_stride, int32_t* status, int heads) {
  PagedArgs a;
  a.k = c.k; a.v = c.v; a.ks = c.k_scale; a.vs = c.v_scale;
  a.table = c.page_table; a.idx = idx; a.n_active = n_active;
  a.n_pages = c.n_pages; a.max_pages = c.max_pages; a.Hkv = c.n_kv_heads;
  a.page_shift = 0;
  while ((1 << a.page_shift) < c.page_size) ++a.page_shift;
  a.parts = (c.n_kv_heads + heads - 1) / heads;
  a.div_parts = fast_div_by(a.parts);
  a.div_n = fast_div_by(N);
  a.B = B; a.N = N; a.max_rows = max_rows; a.row_stride = row_stride; a.status = status;
  return a;
}

// A lane group takes two heads of a row, so that the chain position -> page table -> slot is walked once for both (12288 rows
// of 32 heads written: 59 us with one head, 51 with two, 57 with four; 6144 read back: 32.7, 29.1, 31.3), unless one head each
// fits the SMs at once: then the shortest chain wins (23 rows written: 2.0 us with one head, 2.3 with two).
int heads_at_once(const surelock_paged_kv& c, int max_rows) {
  return (long long)max_rows * c.n_kv_heads <= (long long)sm_count() * PK_SCATTER_BLOCKS * (PK_THREADS / (c.head_dim / 8)) ? 1 : 2;
}
// a grid with a lane group per item; the kernels still loop should it be cut
int paged_grid(const PagedArgs& a, int head_dim) {
  const long long items = (long long)a.max_rows * a.parts, groups = PK_THREADS / (head_dim / 8);
  if (items > 0x7fffffffll) return -1;   // the kernels count items in 32 bits
  const long long want = (items + groups - 1) / groups;
  return (int)(want < 1 ? 1 : want > (1 << 20) ? 1 << 20 : want);
}

template <int KIND, int DH, int U>
int scatter_kind(const PagedArgs& a, const void* k, const void* v, int dtype, cudaStream_t st) {
  const int grid = paged_grid(a, DH);
  if (grid < 0) return SL_EUNSUPPORTED;
  const dim3 g(grid);
  if (dtype == SL_BF16)
    SL_CUDA_TRY(launch_pdl(kv_scatter_paged_kernel<KIND, DH, U, bf16>, g, dim3(PK_THREADS), 0, st, a, (const bf16*)k, (const bf16*)v));
  else
    SL_CUDA_TRY(launch_pdl(kv_scatter_paged_kernel<KIND, DH, U, float>, g, dim3(PK_THREADS), 0, st, a, (const float*)k, (const float*)v));
  return SL_OK;
}

template <int KIND, int DH, int U>
int gather_kind(const PagedArgs& a, void* k, void* v, int dtype, cudaStream_t st) {
  const int grid = paged_grid(a, DH);
  if (grid < 0) return SL_EUNSUPPORTED;
  const dim3 g(grid);
  if (dtype == SL_BF16)
    SL_CUDA_TRY(launch_pdl(kv_gather_paged_kernel<KIND, DH, U, bf16>, g, dim3(PK_THREADS), 0, st, a, (bf16*)k, (bf16*)v));
  else
    SL_CUDA_TRY(launch_pdl(kv_gather_paged_kernel<KIND, DH, U, float>, g, dim3(PK_THREADS), 0, st, a, (float*)k, (float*)v));
  return SL_OK;
}

}  // namespace

#define SL_BY_HEAD(F, KIND, ...)                                                            \
  (c.head_dim == 128 ? (heads == 2 ? F<KIND, 128, 2>(__VA_ARGS__) : F<KIND, 128, 1>(__VA_ARGS__)) \
                     : (heads == 2 ? F<KIND, 64, 2>(__VA_ARGS__) : F<KIND, 64, 1>(__VA_ARGS__)))
#define SL_BY_KIND(F, ...)                                          \
  (c.dtype == SL_BF16   ? SL_BY_HEAD(F, SL_BF16, __VA_ARGS__)       \
   : c.dtype == SL_E4M3 ? SL_BY_HEAD(F, SL_E4M3, __VA_ARGS__)       \
                        : SL_BY_HEAD(F, SL_INT8, __VA_ARGS__))

int launch_kv_scatter_paged(const surelock_paged_kv& c, const void* k, const void* v, long long row_stride, const int32_t* idx,
                            const int32_t* n_active, int max_rows, int B, int N, int dtype, int32_t* status, cudaStream_t st) {
  const int heads = heads_at_once(c, max_rows);
  const PagedArgs a = paged_args(c, idx, n_active, max_rows, B, N, row_stride, status, heads);
  return SL_BY_KIND(scatter_kind, a, k, v, dtype, st);
}

int launch_kv_gather_paged(const surelock_paged_kv& c, const int32_t* idx, const int32_t* n_active, int max_rows, int B, int N,
                           void* k, void* v, long long row_stride, int dtype, int32_t* status, cudaStream_t st) {
  const int heads = heads_at_once(c, max_rows);
  const PagedArgs a = paged_args(c, idx, n_active, max_rows, B, N, row_stride, status, heads);
  return SL_BY_KIND(gather_kind, a, k, v, dtype, st);
}

}  // namespace sl
