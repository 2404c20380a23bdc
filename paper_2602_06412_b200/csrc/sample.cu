// A token per row of logits from one given uniform number, with temperature, top-k, top-p and min-p.
//
// With m the row's largest logit and w_v = exp((x_v - m) / T), put the tokens in order of falling x (ties: the lowest index first;
// tokens of -inf do not count).  Each filter keeps a prefix of that order:
//   top-k   the first k;   top-p  of those, the shortest prefix whose weights sum to at least top_p of theirs;
//   min-p   the tokens with w_v >= min_p;
// the token drawn is the first one of the shortest prefix whose running sum of weights exceeds u times the prefix's.  So nothing
// needs sorting: all that is asked of the row is "which token has rank n" and "at which token does the running sum reach s", and
// both are answered by sums over values.  Sums are held in 64 bits: with 100000 tokens in the prefix, 32 would draw a neighbour of
// the right token in one row of a hundred.
//
// bf16 rows (WindowSums): a bf16 number is its own histogram bin.  One pass counts the row's values in shared memory, 6144 bins
// to a sign for magnitudes in [2^-32, 2^16), which leaves the sums to the few thousand distinct values: one exponential each instead of
// one per token, and a sum is exact but for 2^-53 roundings.  The occupied range of bins is then walked in order, a few bins to
// a thread.  The token's index is found by a second pass that counts the tokens of the value that was drawn, out of the L2.  A row with a
// finite value outside the window (not zero) is done by the other method.
//
// fp32 rows (BinnedSums): 2048 bins of equal width over the values that weigh anything.  One pass adds every token's weight, as four limbs of
// a fixed-point number (exact sums in any order), to its bin; a bin that is asked for is opened by another pass over the row's tokens
// in it: a few are ranked against one another, more of them are binned once more by their keys.
//
// A row is one CTA's work, or with few rows that of a cluster of CTAs, whose shares meet through distributed shared memory.
#include "tc_common.cuh"

namespace sl {
namespace {

constexpr int SM_THREADS = 512, SM_WARPS = SM_THREADS / 32;

struct SampleArgs {
  const void* logits;
  long long row_stride;
  surelock_sampling sets;
  const int32_t *set_of_row, *n_active;
  const float* u;
  int32_t *token, *n_kept, *status;
  float* conf;
  int max_rows, vocab;
};

__device__ __forceinline__ uint32_t ld_cluster_u32(uint32_t addr) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ double ld_cluster_f64(uint32_t addr) {
  double v;
  asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(v) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ void add_shared(uint32_t addr, uint32_t v) {
  asm volatile("red.shared.add.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}

// of two 16-bit numbers at a time
__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.u16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t add_u16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("add.u16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t min_u16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("min.u16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

// all threads of the row: one CTA's, or a cluster's
template <bool CLUSTER> __device__ __forceinline__ void row_sync() {
  if (CLUSTER) cluster_sync_all(); else __syncthreads();
}

// Ordered keys: a larger number has a larger key; both zeros have the same.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key); }

// This CTA's share of a row: whole 16-byte words, the first CTA also what lies before the first of them, the last what is left.
template <typename T> struct Share {
  static constexpr int V = 16 / sizeof(T);
  const T* row;
  int head, tail0, vocab;           // tokens before the first word, first token behind the last
  int v0, v1;                       // this CTA's words
  bool first, last;
  __device__ Share(const T* p, int n, int cta, int ctas) : row(p), vocab(n) {
    head = min(n, (int)(((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / sizeof(T)));
    const int words = (n - head) / V;
    tail0 = head + words * V;
    v0 = (int)((long long)words * cta / ctas);
    v1 = (int)((long long)words * (cta + 1) / ctas);
    first = cta == 0;
    last = cta == ctas - 1;
  }
  __device__ const uint4* words() const { return reinterpret_cast<const uint4*>(row + head); }
  // f(x) for every token of this CTA's share, in no particular order
  template <typename F> __device__ void each(F f) const {
    const uint4* w = words();
    for (int v = v0 + (int)threadIdx.x; v < v1; v += SM_THREADS) {
      const uint4 u = w[v];
      const T* e = reinterpret_cast<const T*>(&u);
#pragma unroll
      for (int i = 0; i < V; ++i) f(to_f(e[i]));
    }
    if (first && (int)threadIdx.x < head) f(to_f(row[threadIdx.x]));
    if (last && tail0 + (int)threadIdx.x < vocab) f(to_f(row[tail0 + threadIdx.x]));
  }
};

// a token by its place in the order: its rank (0 = the largest), the sum of weights up to and with it, its value (or bin) and which of
// the tokens of that value it is; for a bin also its tokens and what lies before it
struct Found {
  double mass, before_w;
  uint32_t rank, key, nth, before_n, tokens, valid;
};

struct Shared {                     // beside the bins
  double part_w[SM_WARPS], part_m[SM_WARPS], part_raw[SM_WARPS];
  uint32_t part_n[SM_WARPS], part_nm[SM_WARPS], matches[SM_WARPS];
  double powers[32];                // 2^(i / 32)
  double cta_w, cta_m, cta_raw;     // this CTA's sums, read by the cluster
  uint32_t cta_n, cta_nm, cta_matches;
  uint32_t top, lo, hi, flags, zeros, list_n, owner;
  Found found[2], here;             // found: by turns, so that none is overwritten while the cluster reads it
};

enum { ROW_UNDEFINED = 1, ROW_OUTSIDE = 2 };

// the settings of a row
struct Settings {
  double T, top_p, min_p;
  float u;
  int top_k;
  bool greedy, ok;
};

// e^z for z <= 0, by a table of 2^(i/32) and the Taylor polynomial of what is left (Tang's table-driven method): |r| <= ln 2 / 64, so that
// r^6 / 720 is 2^-48 of the result at most.  Below e^-700 it stays e^-700, which no sum notices.
__device__ __forceinline__ double exp_falling(double z, const double* table) {
  z = fmax(z, -700.0);
  const double n = rint(z * 46.16624130844683);                     // 32 / ln 2
  const double r = fma(-n, 5.9631716539705866e-12, fma(-n, 0.02166084938653512, z));   // ln 2 / 32 in two terms, the first of 32 bits
  const int k = (int)n;
  double p = fma(r, 1.0 / 120, 1.0 / 24);
  p = fma(p, r, 1.0 / 6);
  p = fma(p, r, 0.5);
  p = fma(p * r, r, r);
  const double t = table[k & 31];
  const double v = fma(t, p, t);
  return __hiloint2double(__double2hiint(v) + ((k >> 5) << 20), __double2loint(v));
}

// What both methods leave in registers: every thread has a run of values in falling order, the runs in order of threads (and
// CTAs).  n, w: tokens of the run and their weights, incl_*: running sums up to and with it.
struct Runs {
  uint32_t n, incl_n, excl_n;
  double w, incl_w, excl_w;
  uint32_t total_n, total_nm;
  double total_w, total_m, total_raw;
};

__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ uint32_t warp_sum(uint32_t v) { return __reduce_add_sync(0xffffffffu, v); }

// Running sums of the runs over the row.  nm, m: tokens and weights that min-p keeps; raw: weights at T = 1.
template <bool CLUSTER>
__device__ void sum_runs(Shared& s, Runs& q, uint32_t nm, double m, double raw, int ctas, int cta) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint32_t n = q.n;
  double w = q.w;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t a = __shfl_up_sync(0xffffffffu, n, o);
    const double b = __shfl_up_sync(0xffffffffu, w, o);
    if (lane >= o) {
      n += a;
      w += b;
    }
  }
  nm = warp_sum(nm);
  m = warp_sum(m);
  raw = warp_sum(raw);
  if (lane == 31) {
    s.part_n[warp] = n;
    s.part_w[warp] = w;
    s.part_nm[warp] = nm;
    s.part_m[warp] = m;
    s.part_raw[warp] = raw;
  }
  __syncthreads();
  uint32_t n0 = 0, nn = 0, nnm = 0;
  double w0 = 0, ww = 0, mm = 0, rr = 0;
#pragma unroll
  for (int i = 0; i < SM_WARPS; ++i) {
    if (i == warp) {
      n0 = nn;
      w0 = ww;
    }
    nn += s.part_n[i];
    ww += s.part_w[i];
    nnm += s.part_nm[i];
    mm += s.part_m[i];
    rr += s.part_raw[i];
  }
  double before_w = 0;
  uint32_t before_n = 0;
  if (CLUSTER) {
    if (threadIdx.x == 0) {
      s.cta_n = nn;
      s.cta_w = ww;
      s.cta_nm = nnm;
      s.cta_m = mm;
      s.cta_raw = rr;
    }
    cluster_sync_all();
    nn = nnm = 0;
    ww = mm = rr = 0;
    for (int c = 0; c < ctas; ++c) {
      if (c == cta) {
        before_n = nn;
        before_w = ww;
      }
      nn += ld_cluster_u32(mapa_u32(smem_u32(&s.cta_n), c));
      nnm += ld_cluster_u32(mapa_u32(smem_u32(&s.cta_nm), c));
      ww += ld_cluster_f64(mapa_u32(smem_u32(&s.cta_w), c));
      mm += ld_cluster_f64(mapa_u32(smem_u32(&s.cta_m), c));
      rr += ld_cluster_f64(mapa_u32(smem_u32(&s.cta_raw), c));
    }
  }
  q.total_n = nn; q.total_nm = nnm; q.total_w = ww; q.total_m = mm; q.total_raw = rr;
  q.incl_n = before_n + n0 + n;
  q.incl_w = before_w + (w0 + w);
  q.excl_n = q.incl_n - q.n;
  const double up = __shfl_up_sync(0xffffffffu, q.incl_w, 1);
  q.excl_w = lane ? up : before_w + w0;
}

// The number of tokens of weight w, 1 ... c, after which cum reaches the target (strict: exceeds it); c if none does.
__device__ __forceinline__ bool reaches(double cum, double target, bool strict) { return strict ? cum > target : cum >= target; }
__device__ __forceinline__ uint32_t tokens_until(double cum, double w, uint32_t c, double target, bool strict) {
  const double about = ceil((target - cum) / w);
  uint32_t j = about >= 1.0 ? (about <= (double)c ? (uint32_t)about : c) : 1u;   // also where w = 0
  while (j > 1 && reaches(cum + (j - 1) * w, target, strict)) --j;
  while (j < c && !reaches(cum + j * w, target, strict)) ++j;
  return j;
}

// What a find asks for: the token of a rank, or the first token at which the running sum of weights reaches a target.
struct Ask {
  bool by_rank, strict;
  uint32_t rank;
  double target;
  __device__ bool in(const Runs& q) const {
    return q.n && (by_rank ? rank < q.incl_n : reaches(q.incl_w, target, strict));
  }
};
__device__ __forceinline__ Ask ask_rank(uint32_t rank) { return {true, false, rank, 0.0}; }
__device__ __forceinline__ Ask ask_mass(double target, bool strict) { return {false, strict, 0u, target}; }

// A walk down a run, value by value; true once the token is found.  `last`: the place to take should roundings leave none.
struct Walk {
  double cum;
  uint32_t n;
  Found f;
  __device__ bool step(const Ask& a, uint32_t c, double w, uint32_t key) {
    if (!c) return false;
    const bool here = a.by_rank ? a.rank < n + c : reaches(cum + c * w, a.target, a.strict);
    const uint32_t j = !here ? c : a.by_rank ? a.rank - n + 1 : tokens_until(cum, w, c, a.target, a.strict);
    f.mass = cum + j * w;
    f.rank = n + j - 1;
    f.key = key;
    f.nth = j - 1;
    f.before_w = cum;
    f.before_n = n;
    f.tokens = c;
    cum += c * w;
    n += c;
    return here;
  }
};

// The first thread of this CTA whose run holds what is asked for, SM_THREADS if none does.
__device__ __forceinline__ uint32_t first_thread(Shared& s, bool in) {
  if (threadIdx.x == 0) s.owner = SM_THREADS;
  __syncthreads();
  const unsigned b = __ballot_sync(0xffffffffu, in);
  if (b && (threadIdx.x & 31) == 0) atomicMin(&s.owner, threadIdx.x + __ffs(b) - 1);
  __syncthreads();
  const uint32_t o = s.owner;
  __syncthreads();
  return o;
}

// What both methods share: whose run holds what is asked for, its walk there, and the answer for all threads of the row.
template <bool CLUSTER> struct Finder {
  Shared& s;
  int cta, ctas, turn = 0;
  Runs q;
  double inv_T;                     // (x - max) / T as a product: off by 2^-52 of itself
  __device__ Finder(Shared& sh, int c, int n) : s(sh), cta(c), ctas(n) {}
  template <typename F> __device__ Found search(const Ask& ask, const Runs& r, F walk) {
    const uint32_t o = first_thread(s, ask.in(r));
    Found& mine = s.found[turn];
    turn ^= 1;
    if (threadIdx.x == 0 && o == SM_THREADS) mine.valid = 0u;
    if (threadIdx.x == o) {
      Walk k;
      k.cum = r.excl_w;
      k.n = r.excl_n;
      walk(k);
      k.f.valid = 1u;
      mine = k.f;
    }
    row_sync<CLUSTER>();
    if (!CLUSTER) return mine;
    Found f;
    f.valid = 0u;
    for (int c = 0; c < ctas && !f.valid; ++c) {
      const uint32_t a = mapa_u32(smem_u32(&mine), c);
      f.valid = ld_cluster_u32(a + offsetof(Found, valid));
      if (!f.valid) continue;
      f.mass = ld_cluster_f64(a + offsetof(Found, mass));
      f.before_w = ld_cluster_f64(a + offsetof(Found, before_w));
      f.rank = ld_cluster_u32(a + offsetof(Found, rank));
      f.key = ld_cluster_u32(a + offsetof(Found, key));
      f.nth = ld_cluster_u32(a + offsetof(Found, nth));
      f.before_n = ld_cluster_u32(a + offsetof(Found, before_n));
      f.tokens = ld_cluster_u32(a + offsetof(Found, tokens));
    }
    return f;
  }
  // no run reached the target, by roundings: it is behind the last token
  __device__ static Found behind_all(double mass) {
    Found f = {};
    f.mass = mass;
    f.rank = 0xffffffffu;
    return f;
  }
};

// ---- bf16: counts of values -----------------------------------------------------------------------------------------------
constexpr uint32_t WIN_LO = (127 - 32) << 7, WIN_HI = (127 + 16) << 7, WIN_BINS = WIN_HI - WIN_LO;   // magnitudes' bits

template <bool CLUSTER> struct WindowSums : Finder<CLUSTER> {
  typedef Finder<CLUSTER> F;
  using F::s; using F::cta; using F::ctas; using F::q; using F::inv_T;
  static constexpr int SMEM = (2 * WIN_BINS + 32) * 4 + (CLUSTER ? (WIN_BINS + 8) * 4 : 0);
  uint32_t* bins;                   // [magnitude][sign], and 32 that nobody reads
  uint32_t* merged;                 // this CTA's run of places, summed over the cluster
  uint32_t hi, R, zeros, lo, p0, p1;    // places: positive values from magnitude hi of the window down, zero at R, negative ones from lo up
  uint32_t base;                    // first place of this CTA
  double top;

  __device__ WindowSums(Shared& sh, void* smem, int c, int n) : F(sh, c, n) {
    bins = reinterpret_cast<uint32_t*>(smem);
    merged = bins + 2 * WIN_BINS + 32;
  }
  // Counts the row.  0, ROW_UNDEFINED (a NaN, +inf, or nothing finite) or ROW_OUTSIDE (values outside the window).
  __device__ uint32_t count(const Share<bf16>& row) {
    uint4* b4 = reinterpret_cast<uint4*>(bins);
    for (int i = threadIdx.x; i < (int)(2 * WIN_BINS / 4); i += SM_THREADS) b4[i] = make_uint4(0u, 0u, 0u, 0u);
    if (threadIdx.x == 0) {
      s.top = s.hi = s.flags = s.zeros = 0u;
      s.lo = 0xffffu;
    }
    __syncthreads();
    // a bf16 number turned left by a bit is its magnitude and then its sign; less the window's start, the number of its bin
    constexpr uint32_t SHIFT = (0x10000u - 2 * WIN_LO) * 0x10001u, LIMIT = (0x8000u - 2 * WIN_BINS) * 0x10001u;
    uint32_t most = 0u, least = 0xffffffffu, zero = 0u, flags = 0u;   // bins, two at a time
    __nv_bfloat162 top2 = __float2bfloat162_rn(-INFINITY);
    const uint32_t aside = (2 * WIN_BINS + (threadIdx.x & 31)) * 0x10001u;   // a bin per lane for what is outside
    // what makes a word have bins outside: zeros are counted apart, -inf is left out, and the rest is for the row to know
    auto explain = [&](uint32_t w, uint32_t b) {
      const __nv_bfloat162 x = *reinterpret_cast<const __nv_bfloat162*>(&w);
      const uint32_t zeros2 = __heq2_mask(x, __float2bfloat162_rn(0.f)), none2 = __heq2_mask(x, __float2bfloat162_rn(-INFINITY));
      zero += __popc(zeros2 & 0x10001u);
#pragma unroll
      for (int h = 0; h < 32; h += 16) {
        const uint32_t bin = (b >> h) & 0xffffu;
        if (bin < 2 * WIN_BINS) most = max_u16x2(most, bin);
        else if (!(((zeros2 | none2) >> h) & 1u)) flags |= ((w >> h) & 0x7fffu) >= 0x7f80u ? ROW_UNDEFINED : ROW_OUTSIDE;
      }
    };
    auto eight = [&](const uint4& u) {
      const uint32_t w[4] = {u.x, u.y, u.z, u.w};
      uint32_t b[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        b[i] = min_u16x2(add_u16x2(((w[i] << 1) & 0xfffefffeu) | ((w[i] >> 15) & 0x00010001u), SHIFT), aside);
        atomicAdd(bins + (b[i] & 0xffffu), 1u);
        atomicAdd(bins + (b[i] >> 16), 1u);
        top2 = __hmax2(top2, *reinterpret_cast<const __nv_bfloat162*>(&w[i]));
      }
      const uint32_t mx = max_u16x2(max_u16x2(b[0], b[1]), max_u16x2(b[2], b[3]));
      least = min_u16x2(least, min_u16x2(min_u16x2(b[0], b[1]), min_u16x2(b[2], b[3])));
      if (((mx + LIMIT) & 0x80008000u) == 0u) most = max_u16x2(most, mx);   // all inside
      else
#pragma unroll
        for (int i = 0; i < 4; ++i) explain(w[i], b[i]);
    };
    auto one = [&](uint32_t h) {                     // with a -inf beside it
      const uint32_t w = h | 0xff800000u;
      const uint32_t b = min_u16x2(add_u16x2(((w << 1) & 0xfffefffeu) | ((w >> 15) & 0x00010001u), SHIFT), aside);
      atomicAdd(bins + (b & 0xffffu), 1u);
      least = min_u16x2(least, b);
      explain(w, b);
      top2 = __hmax2(top2, *reinterpret_cast<const __nv_bfloat162*>(&w));
    };
    const uint4* w = row.words();
    int v = row.v0 + (int)threadIdx.x;
    for (; v + 3 * SM_THREADS < row.v1; v += 4 * SM_THREADS) {
      uint4 u[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) u[i] = w[v + i * SM_THREADS];
#pragma unroll
      for (int i = 0; i < 4; ++i) eight(u[i]);
    }
    for (; v < row.v1; v += SM_THREADS) eight(w[v]);
    const uint16_t* raw = reinterpret_cast<const uint16_t*>(row.row);
    if (row.first && (int)threadIdx.x < row.head) one(raw[threadIdx.x]);
    if (row.last && row.tail0 + (int)threadIdx.x < row.vocab) one(raw[row.tail0 + threadIdx.x]);

    const uint32_t hi1 = __reduce_max_sync(0xffffffffu, max(most & 0xffffu, most >> 16));
    const uint32_t lo1 = __reduce_min_sync(0xffffffffu, min(least & 0xffffu, least >> 16));   // behind the window where there are none
    const uint32_t top1 = __reduce_max_sync(0xffffffffu, key_of(fmaxf(__low2float(top2), __high2float(top2))));
    const uint32_t zero1 = warp_sum(zero);
    flags = __reduce_or_sync(0xffffffffu, flags);
    if ((threadIdx.x & 31) == 0) {
      atomicMax(&s.hi, hi1);
      atomicMin(&s.lo, lo1);
      atomicMax(&s.top, top1);
      atomicAdd(&s.zeros, zero1);
      atomicOr(&s.flags, flags);
    }
    row_sync<CLUSTER>();
    uint32_t t = s.top, f = s.flags;
    hi = s.hi; lo = s.lo; zeros = s.zeros;
    if (CLUSTER) {
      hi = t = f = zeros = 0u;
      lo = 0xffffu;
      for (int c = 0; c < ctas; ++c) {
        hi = max(hi, ld_cluster_u32(mapa_u32(smem_u32(&s.hi), c)));
        lo = min(lo, ld_cluster_u32(mapa_u32(smem_u32(&s.lo), c)));
        t = max(t, ld_cluster_u32(mapa_u32(smem_u32(&s.top), c)));
        f |= ld_cluster_u32(mapa_u32(smem_u32(&s.flags), c));
        zeros += ld_cluster_u32(mapa_u32(smem_u32(&s.zeros), c));
      }
    }
    hi >>= 1;
    lo >>= 1;
    top = (double)value_of(t);
    if ((f & ROW_UNDEFINED) || t == key_of(-INFINITY)) return ROW_UNDEFINED;
    return f & ROW_OUTSIDE;
  }
  // bin and value of a place
  __device__ uint32_t bin_of(uint32_t p) const { return p < R ? 2 * (hi - p) : 2 * (lo + (p - R - 1)) + 1; }
  __device__ float value(uint32_t p) const {
    return p == R ? 0.f : __uint_as_float(p < R ? (WIN_LO + hi - p) << 16 : 0x80000000u | (WIN_LO + lo + (p - R - 1)) << 16);
  }
  __device__ uint32_t tokens(uint32_t p) const { return CLUSTER ? merged[p - base] : p == R ? zeros : bins[bin_of(p)]; }
  __device__ double largest_value() const { return top; }
  __device__ double weight(uint32_t p) const { return exp_falling(((double)value(p) - top) * inv_T, s.powers); }

  __device__ void sum(const Settings& set) {
    inv_T = set.greedy ? 1.0 : 1.0 / set.T;
    R = hi >= lo ? hi - lo + 1 : 0u;
    // the place of the largest logit: those before it are empty
    const uint32_t mag = (__float_as_uint((float)top) & 0x7fffffffu) >> 16;
    const uint32_t p_top = top > 0.0 ? hi - (mag - WIN_LO) : top == 0.0 ? R : R + 1 + (mag - WIN_LO - lo), places = 2 * R + 1 - p_top;
    base = p_top + places * cta / ctas;
    const uint32_t end = p_top + places * (cta + 1) / ctas;
    if (CLUSTER) {
      for (uint32_t p = base + threadIdx.x; p < end; p += SM_THREADS) {
        uint32_t c = zeros;
        if (p != R) {
          const uint32_t a = smem_u32(bins + bin_of(p));
          c = 0u;
          for (int i = 0; i < ctas; ++i) c += ld_cluster_u32(mapa_u32(a, i));
        }
        merged[p - base] = c;
      }
      __syncthreads();
    }
    const uint32_t each = (end - base + SM_THREADS - 1) / SM_THREADS;
    p0 = min(end, base + each * threadIdx.x);
    p1 = min(end, p0 + each);
    q.n = 0u;
    q.w = 0.0;
    uint32_t nm = 0u;
    double m = 0.0, raw = 0.0;
    const bool plain = inv_T == 1.0;
#pragma unroll 2
    for (uint32_t p = p0; p < p1; ++p) {              // no branch on empty bins: a warp has hardly a step without a full one
      const uint32_t c = tokens(p);
      const double w = weight(p), cw = c * w;
      q.n += c;
      q.w += cw;
      raw += plain ? cw : (double)((float)c * expf((float)((double)value(p) - top)));
      const bool keeps = w >= set.min_p;
      nm += keeps ? c : 0u;
      m += keeps ? cw : 0.0;
    }
    sum_runs<CLUSTER>(s, q, nm, m, raw, ctas, cta);
  }
  __device__ Found find(const Share<bf16>&, const Ask& ask) {
    const Found f = F::search(ask, q, [&](Walk& k) {
      for (uint32_t p = p0; p < p1; ++p) {
        const uint32_t c = tokens(p);
        if (c && k.step(ask, c, weight(p), key_of(value(p)))) break;
      }
    });
    return f.valid ? f : F::behind_all(q.total_w);
  }
};

// ---- any type: bins with exact sums of weights ---------------------------------------------------------------------------------
constexpr int BINS = 2048, LIMBS = 4, LIMB_BITS = 14;   // of a weight in units of 2^-54; 2^17 tokens to a CTA fit a 32-bit sum of limbs
constexpr double WEIGHT_UNIT = 18014398509481984.0;     // 2^54
constexpr int LIST = 256;                               // tokens that are ranked against one another

template <typename T, bool CLUSTER> struct BinnedSums : Finder<CLUSTER> {
  typedef Finder<CLUSTER> F;
  using F::s; using F::cta; using F::ctas; using F::q; using F::inv_T;
  static constexpr int SMEM = BINS * (1 + LIMBS) * 4 + LIST * 16;
  static constexpr int EACH = BINS / SM_THREADS;        // bins to a thread; in a cluster the CTAs share them out
  uint32_t* bins;                   // [1 + LIMBS][BINS]: tokens, limbs
  unsigned long long* weights;      // [LIST]
  uint32_t *list, *keys;            // [LIST]: this CTA's tokens of a bin, and those of the whole row
  float topf, step;                 // bins to a unit of the logits
  uint32_t c0[EACH];                // this thread's bins, from the top
  double w0[EACH];

  __device__ BinnedSums(Shared& sh, void* smem, int c, int n) : F(sh, c, n) {
    bins = reinterpret_cast<uint32_t*>(smem);
    weights = reinterpret_cast<unsigned long long*>(bins + BINS * (1 + LIMBS));
    list = reinterpret_cast<uint32_t*>(weights + LIST);
    keys = list + LIST;
  }
  // the row's largest and smallest finite logits; 0 or ROW_UNDEFINED
  __device__ uint32_t range(const Share<T>& row, float& least) {
    row_sync<CLUSTER>();                            // nobody reads what these words held before
    if (threadIdx.x == 0) {
      s.top = s.flags = 0u;
      s.lo = 0xffffffffu;
    }
    __syncthreads();
    uint32_t t = 0u, lo = 0xffffffffu, flags = 0u;
    row.each([&](float x) {
      if (!(x < INFINITY)) flags |= ROW_UNDEFINED;   // NaN or +inf
      const uint32_t k = key_of(x);
      t = max(t, k);
      if (x != -INFINITY) lo = min(lo, k);
    });
    t = __reduce_max_sync(0xffffffffu, t);
    lo = __reduce_min_sync(0xffffffffu, lo);
    flags = __reduce_or_sync(0xffffffffu, flags);
    if ((threadIdx.x & 31) == 0) {
      atomicMax(&s.top, t);
      atomicMin(&s.lo, lo);
      atomicOr(&s.flags, flags);
    }
    row_sync<CLUSTER>();
    t = s.top;
    lo = s.lo;
    flags = s.flags;
    for (int c = 0; CLUSTER && c < ctas; ++c) {
      t = max(t, ld_cluster_u32(mapa_u32(smem_u32(&s.top), c)));
      lo = min(lo, ld_cluster_u32(mapa_u32(smem_u32(&s.lo), c)));
      flags |= ld_cluster_u32(mapa_u32(smem_u32(&s.flags), c));
    }
    if (flags || lo == 0xffffffffu) return ROW_UNDEFINED;
    topf = value_of(t);
    least = value_of(lo);
    return 0u;
  }
  __device__ double largest_value() const { return (double)topf; }
  __device__ unsigned long long weight(float x) const { return __double2ull_rn(exp_falling(((double)x - (double)topf) * inv_T, s.powers) * WEIGHT_UNIT); }
  // Falls with x; what is too far below the largest shares the last bin.
  __device__ uint32_t bin_of(float x) const { return min((uint32_t)BINS - 1, __float2uint_rz((topf - x) * step)); }

  __device__ void clear() {
    for (int i = threadIdx.x; i < BINS * (1 + LIMBS) / 4; i += SM_THREADS) reinterpret_cast<uint4*>(bins)[i] = make_uint4(0u, 0u, 0u, 0u);
    __syncthreads();
  }
  __device__ void add(uint32_t bin, unsigned long long w) {
    const uint32_t a = smem_u32(bins + bin);
    add_shared(a, 1u);
#pragma unroll
    for (int i = 0; i < LIMBS; ++i) {
      const uint32_t limb = i + 1 < LIMBS ? (uint32_t)w & ((1u << LIMB_BITS) - 1) : (uint32_t)w;
      if (limb) add_shared(a + 4 * BINS * (i + 1), limb);
      w >>= LIMB_BITS;
    }
  }
  // this thread's bins summed over the row, and the runs they make
  __device__ void collect(Runs& r, uint32_t* c, double* w, uint32_t& first, uint32_t nm, double m, double raw) {
    const uint32_t per = CLUSTER ? BINS / ctas : BINS, each = (per + SM_THREADS - 1) / SM_THREADS;
    first = cta * per + threadIdx.x * each;
    r.n = 0u;
    r.w = 0.0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      c[i] = 0u;
      w[i] = 0.0;
      if (i >= (int)each || threadIdx.x * each + i >= per) continue;
      const uint32_t a = smem_u32(bins + first + i);
      unsigned long long limb[LIMBS] = {};
      for (int p = 0; p < (CLUSTER ? ctas : 1); ++p) {
        const uint32_t b = CLUSTER ? mapa_u32(a, p) : 0u;
        c[i] += CLUSTER ? ld_cluster_u32(b) : bins[first + i];
#pragma unroll
        for (int l = 0; l < LIMBS; ++l) limb[l] += CLUSTER ? ld_cluster_u32(b + 4 * BINS * (l + 1)) : bins[first + i + BINS * (l + 1)];
      }
      double v = 0.0;
#pragma unroll
      for (int l = LIMBS - 1; l >= 0; --l) v = v * (double)(1 << LIMB_BITS) + (double)limb[l];
      w[i] = v / WEIGHT_UNIT;
      r.n += c[i];
      r.w += w[i];
    }
    sum_runs<CLUSTER>(s, r, nm, m, raw, ctas, cta);
  }
  // the bin that holds what is asked for
  __device__ Found open(const Ask& ask, const Runs& r, const uint32_t* c, const double* w, uint32_t first) {
    return F::search(ask, r, [&](Walk& k) {
#pragma unroll
      for (int i = 0; i < EACH; ++i)
        if (c[i] && k.step(ask, c[i], w[i] / c[i], first + i)) break;
    });
  }
  uint32_t first0;
  __device__ void sum(const Share<T>& row, const Settings& set, float least) {
    inv_T = set.greedy ? 1.0 : 1.0 / set.T;
    // beyond 50 T the weights are below 2^-72 of the largest
    const float span = (float)fmin((double)topf - (double)least, 50.0 / inv_T);
    step = span > 0.f ? fminf((float)BINS / span, 3.4e38f) : 0.f;
    clear();
    uint32_t nm = 0u;
    double m = 0.0, raw = 0.0;
    row.each([&](float x) {
      if (x == -INFINITY) return;
      const unsigned long long w = weight(x);
      add(bin_of(x), w);
      const double v = (double)w / WEIGHT_UNIT;
      raw += inv_T == 1.0 ? v : (double)expf(x - topf);
      if (v >= set.min_p) {
        ++nm;
        m += v;
      }
    });
    row_sync<CLUSTER>();
    collect(q, c0, w0, first0, nm, m, raw);
  }
  // Members of a bin: of the first binning, and where that was not enough keys from ka to kb.
  struct Members {
    uint32_t bin, ka, kb;
  };
  __device__ bool in(const Members& b, float x, uint32_t k) const { return x != -INFINITY && bin_of(x) == b.bin && k >= b.ka && k <= b.kb; }

  __device__ Found find(const Share<T>& row, const Ask& asked) {
    Ask ask = asked;
    Found f = open(ask, q, c0, w0, first0);
    if (!f.valid) return F::behind_all(q.total_w);
    Members b = {f.key, 0u, 0xffffffffu};
    while (f.tokens > LIST) {
      // the keys that occur, and bins for them
      if (threadIdx.x == 0) {
        s.hi = 0u;
        s.lo = 0xffffffffu;
      }
      clear();
      uint32_t lo = 0xffffffffu, hi = 0u;
      row.each([&](float x) {
        const uint32_t k = key_of(x);
        if (in(b, x, k)) {
          lo = min(lo, k);
          hi = max(hi, k);
        }
      });
      lo = __reduce_min_sync(0xffffffffu, lo);
      hi = __reduce_max_sync(0xffffffffu, hi);
      if ((threadIdx.x & 31) == 0) {
        atomicMin(&s.lo, lo);
        atomicMax(&s.hi, hi);
      }
      row_sync<CLUSTER>();
      lo = s.lo;
      hi = s.hi;
      for (int c = 0; CLUSTER && c < ctas; ++c) {
        lo = min(lo, ld_cluster_u32(mapa_u32(smem_u32(&s.lo), c)));
        hi = max(hi, ld_cluster_u32(mapa_u32(smem_u32(&s.hi), c)));
      }
      if (lo == hi) {                               // one value: no need to look at its tokens
        Walk k;
        k.cum = f.before_w;
        k.n = f.before_n;
        k.step(ask, f.tokens, (double)weight(value_of(lo)) / WEIGHT_UNIT, lo);
        row_sync<CLUSTER>();
        return k.f;
      }
      const int shift = max(0, 21 - __clz(hi - lo));  // 32 - clz bits, of which the bins tell 11
      row.each([&](float x) {
        const uint32_t k = key_of(x);
        if (in(b, x, k)) add((hi - k) >> shift, weight(x));
      });
      row_sync<CLUSTER>();
      uint32_t c[EACH], first;
      double w[EACH];
      Runs r;
      collect(r, c, w, first, 0u, 0.0, 0.0);
      r.excl_n += f.before_n; r.incl_n += f.before_n;
      r.excl_w += f.before_w; r.incl_w += f.before_w;
      const uint32_t last = f.before_n + f.tokens - 1;
      Found g = open(ask, r, c, w, first);
      if (!g.valid) {                               // by roundings: the last token of the bin
        ask = ask_rank(last);
        g = open(ask, r, c, w, first);
      }
      f = g;
      b.kb = hi - (g.key << shift);
      b.ka = shift ? max(lo, b.kb - ((1u << shift) - 1)) : b.kb;
    }
    // few tokens: each is ranked against all
    if (threadIdx.x == 0) s.list_n = 0u;
    __syncthreads();
    row.each([&](float x) {
      const uint32_t k = key_of(x);
      if (in(b, x, k)) {
        const uint32_t at = atomicAdd(&s.list_n, 1u);
        if (at < LIST) list[at] = k;
      }
    });
    row_sync<CLUSTER>();
    const uint32_t n = f.tokens, i = threadIdx.x;
    if (i < n) {
      uint32_t at = i, k = 0u;
      for (int c = 0; c < (CLUSTER ? ctas : 1); ++c) {
        const uint32_t has = CLUSTER ? ld_cluster_u32(mapa_u32(smem_u32(&s.list_n), c)) : s.list_n;
        if (at < has) {
          k = CLUSTER ? ld_cluster_u32(mapa_u32(smem_u32(list + at), c)) : list[at];
          break;
        }
        at -= has;
      }
      keys[i] = k;
      weights[i] = weight(value_of(k));
    }
    if (i == 0) s.owner = 0xffffffffu;
    __syncthreads();
    uint32_t before = 0u, same = 0u;
    unsigned long long sum = 0ull;
    if (i < n) {
      const uint32_t k = keys[i];
      for (uint32_t j = 0; j < n; ++j) {
        const uint32_t o = keys[j];
        same += o == k;
        if (o > k) {
          ++before;
          sum += weights[j];
        }
      }
      const double w = (double)weights[i] / WEIGHT_UNIT, cum = f.before_w + (double)sum / WEIGHT_UNIT;
      if (ask.by_rank ? ask.rank < f.before_n + before + same : reaches(cum + same * w, ask.target, ask.strict)) atomicMin(&s.owner, before);
    }
    __syncthreads();
    const bool none = s.owner == 0xffffffffu;        // by roundings: the last token
    if (i < n && (none ? before + same == n : before == s.owner)) {
      if (none) ask = ask_rank(f.before_n + n - 1);
      Walk k;
      k.cum = f.before_w + (double)sum / WEIGHT_UNIT;
      k.n = f.before_n + before;
      k.step(ask, same, (double)weights[i] / WEIGHT_UNIT, keys[i]);
      s.here = k.f;                                  // equal tokens write the same
    }
    __syncthreads();
    return s.here;
  }
};

// The settings' prefix and the token drawn from it.
template <typename S, typename T> __device__ Found draw(S& sums, const Share<T>& row, const Settings& set, uint32_t& kept) {
  const Runs& q = sums.q;
  uint32_t n = q.total_n;
  double mass = q.total_w;
  if (set.greedy) {
    kept = 1u;
    return sums.find(row, ask_rank(0u));
  }
  if (set.top_k > 0 && (uint32_t)set.top_k < n) {
    n = (uint32_t)set.top_k;
    mass = sums.find(row, ask_rank(n - 1)).mass;
  }
  if (set.top_p < 1.0) {
    const Found f = sums.find(row, ask_mass(set.top_p * mass, false));
    if (f.rank < n - 1) {
      n = f.rank + 1;
      mass = f.mass;
    }
  }
  if (q.total_nm < n) {                              // min-p keeps the largest at least: its weight is 1
    n = q.total_nm;
    mass = q.total_m;
  }
  kept = n;
  const Found f = sums.find(row, ask_mass((double)set.u * mass, true));
  return f.rank < n ? f : sums.find(row, ask_rank(n - 1));
}

// The tokens of a 16-byte word that equal x, a bit for each, and their number.
template <typename T> struct Matcher;
template <> struct Matcher<float> {
  float x;
  __device__ Matcher(float v) : x(v) {}
  __device__ uint32_t bits(const uint4& u) const {
    return (__uint_as_float(u.x) == x) | (__uint_as_float(u.y) == x) << 1 | (__uint_as_float(u.z) == x) << 2 | (__uint_as_float(u.w) == x) << 3;
  }
  __device__ uint32_t number(const uint4& u) const {
    return (__uint_as_float(u.x) == x) + (__uint_as_float(u.y) == x) + (__uint_as_float(u.z) == x) + (__uint_as_float(u.w) == x);
  }
};
template <> struct Matcher<bf16> {
  __nv_bfloat162 x;
  __device__ Matcher(float v) : x(__float2bfloat162_rn(v)) {}
  __device__ uint32_t mask(uint32_t w) const { return __heq2_mask(*reinterpret_cast<const __nv_bfloat162*>(&w), x); }   // 0xffff for each
  __device__ uint32_t bits(const uint4& u) const {
    const uint32_t a = (mask(u.x) & 0x20001u) | (mask(u.y) & 0x80004u) | (mask(u.z) & 0x200010u) | (mask(u.w) & 0x800040u);
    return (a | a >> 16) & 0xffu;
  }
  __device__ uint32_t number(const uint4& u) const {
    return __popc((mask(u.x) & 0x10001u) | (mask(u.y) & 0x20002u) | (mask(u.z) & 0x40004u) | (mask(u.w) & 0x80008u));
  }
};

// The nth token of the value that has this key: a count over the row, then the one warp's words that hold it once more.
template <typename T, bool CLUSTER>
__device__ void write_token(Shared& s, const Share<T>& row, const Found& f, int cta, int ctas, int32_t* token) {
  constexpr int V = Share<T>::V;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const float x = value_of(f.key);
  const uint4* words = row.words();
  const int a = row.v0 + (int)((long long)(row.v1 - row.v0) * warp / SM_WARPS), b = row.v0 + (int)((long long)(row.v1 - row.v0) * (warp + 1) / SM_WARPS);
  const int heads = row.first && warp == 0 ? row.head : 0, tails = row.last && warp == SM_WARPS - 1 ? row.vocab - row.tail0 : 0;
  uint32_t n = 0u;
  const Matcher<T> equal(x);
  int v = a + lane;
  for (; v + 96 < b; v += 128) {
    const uint4 u[4] = {words[v], words[v + 32], words[v + 64], words[v + 96]};
#pragma unroll
    for (int i = 0; i < 4; ++i) n += equal.number(u[i]);
  }
  for (; v < b; v += 32) n += equal.number(words[v]);
  const bool in_head = lane < heads && to_f(row.row[lane]) == x, in_tail = lane < tails && to_f(row.row[row.tail0 + lane]) == x;
  n = warp_sum(n + in_head + in_tail);
  if (lane == 0) s.matches[warp] = n;
  __syncthreads();
  uint32_t before = 0u, all = 0u;
  for (int i = 0; i < SM_WARPS; ++i) {
    if (i == warp) before = all;
    all += s.matches[i];
  }
  if (CLUSTER) {
    if (threadIdx.x == 0) s.cta_matches = all;
    cluster_sync_all();
    for (int c = 0; c < cta; ++c) before += ld_cluster_u32(mapa_u32(smem_u32(&s.cta_matches), c));
  }
  if (f.nth < before || f.nth >= before + n) return;
  uint32_t left = f.nth - before;                    // of this warp's tokens of that value
  const uint32_t head_at = __ballot_sync(0xffffffffu, in_head);
  if (left < (uint32_t)__popc(head_at)) {
    if (in_head && (uint32_t)__popc(head_at & ((1u << lane) - 1)) == left) *token = lane;
    return;
  }
  left -= __popc(head_at);
  for (int v0 = a; v0 < b; v0 += 32) {
    v = v0 + lane;
    uint32_t m = v < b ? equal.bits(words[v]) : 0u, sum = __popc(m);
    const uint32_t mine = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t y = __shfl_up_sync(0xffffffffu, sum, o);
      if (lane >= o) sum += y;
    }
    const uint32_t here = __shfl_sync(0xffffffffu, sum, 31);
    if (left < here) {
      if (sum > left && sum - mine <= left) {
        for (uint32_t skip = left - (sum - mine); skip > 0; --skip) m &= m - 1;
        *token = row.head + v * V + __ffs(m) - 1;
      }
      return;
    }
    left -= here;
  }
  const uint32_t tail_at = __ballot_sync(0xffffffffu, in_tail);
  if (in_tail && (uint32_t)__popc(tail_at & ((1u << lane) - 1)) == left) *token = row.tail0 + lane;
}

template <typename T, bool CLUSTER> struct SampleSmem {
  static constexpr int BYTES = BinnedSums<T, CLUSTER>::SMEM;
};
template <bool CLUSTER> struct SampleSmem<bf16, CLUSTER> {
  static constexpr int W = WindowSums<CLUSTER>::SMEM, R = BinnedSums<bf16, CLUSTER>::SMEM, BYTES = W > R ? W : R;
};

template <typename S, typename T, bool CLUSTER>
__device__ void finish(Shared& s, S& sums, const Share<T>& row, const Settings& set, const SampleArgs& a, int r, int cta, int ctas) {
  uint32_t kept;
  const Found f = draw(sums, row, set, kept);
  write_token<T, CLUSTER>(s, row, f, cta, ctas, a.token + r);
  if (cta == 0 && threadIdx.x == 0) {
    if (a.conf) a.conf[r] = (float)(exp((double)value_of(f.key) - sums.largest_value()) / sums.q.total_raw);
    if (a.n_kept) a.n_kept[r] = (int32_t)kept;
  }
}

// apart, so that the bf16 rows' method keeps its registers
template <typename T, bool CLUSTER>
__device__ __noinline__ uint32_t sample_binned(Shared& s, void* smem, const Share<T>& row, const Settings& set, const SampleArgs& a, int r,
                                               int cta, int ctas) {
  BinnedSums<T, CLUSTER> sums(s, smem, cta, ctas);
  float least;
  const uint32_t state = sums.range(row, least);
  if (state == 0u) {
    sums.sum(row, set, least);
    finish<BinnedSums<T, CLUSTER>, T, CLUSTER>(s, sums, row, set, a, r, cta, ctas);
  }
  return state;
}

template <typename T, bool CLUSTER>
__global__ void __launch_bounds__(SM_THREADS, 2) sample_kernel(const __grid_constant__ SampleArgs a) {
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ Shared s;
  griddep_wait();
  griddep_launch();
  if (threadIdx.x < 32) s.powers[threadIdx.x] = exp2(threadIdx.x / 32.0);   // seen after the first barrier
  int cta = 0, ctas = 1;
  if (CLUSTER) {
    uint32_t n;
    asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(n));
    ctas = (int)n;
    cta = (int)cluster_ctarank();
  }
  const int r = blockIdx.x / ctas;
  if (r >= min(*a.n_active, a.max_rows)) return;
  Settings set;
  {
    const int i = a.set_of_row ? a.set_of_row[r] : a.sets.n_sets == 1 ? 0 : r;
    set.ok = (unsigned)i < (unsigned)a.sets.n_sets;
    if (!set.ok && threadIdx.x == 0) set_status(a.status, SL_DEV_BAD_INDEX);
    const int j = set.ok ? i : 0;
    const float t = a.sets.temperature ? a.sets.temperature[j] : 1.f;
    set.ok = set.ok && t >= 0.f;                     // not where it is NaN
    set.greedy = t == 0.f;
    set.T = t;
    set.top_k = a.sets.top_k ? a.sets.top_k[j] : 0;
    const float p = a.sets.top_p ? a.sets.top_p[j] : 1.f, m = a.sets.min_p ? a.sets.min_p[j] : 0.f;
    set.top_p = p < 1.f ? (double)p : 1.0;
    set.min_p = m > 0.f ? (double)fminf(m, 1.f) : 0.0;
    set.u = fminf(fmaxf(a.u[r], 0.f), 0.99999994f);
  }
  const Share<T> row((const T*)a.logits + r * a.row_stride, a.vocab, cta, ctas);
  uint32_t state = ROW_UNDEFINED;
  if (set.ok) {
    bool binned = true;
    if constexpr (sizeof(T) == 2) {
      WindowSums<CLUSTER> sums(s, smem, cta, ctas);
      state = sums.count(row);
      binned = state == ROW_OUTSIDE;
      if (state == 0u) {
        sums.sum(set);
        finish<WindowSums<CLUSTER>, T, CLUSTER>(s, sums, row, set, a, r, cta, ctas);
      }
    }
    if (binned) {
      const Share<T> row1 = row;                     // copies: the function wants their addresses
      const Settings set1 = set;
      state = sample_binned<T, CLUSTER>(s, smem, row1, set1, a, r, cta, ctas);
    }
  }
  if (state == ROW_UNDEFINED && cta == 0 && threadIdx.x == 0) {
    a.token[r] = -1;
    if (a.conf) a.conf[r] = __int_as_float(0x7fffffff);
    if (a.n_kept) a.n_kept[r] = 0;
  }
  if (CLUSTER) cluster_sync_all();                   // nobody reads this CTA's shared memory any more
}

template <typename T, bool CLUSTER>
int launch_sample_ctas(const SampleArgs& a, int ctas, cudaStream_t st) {
  constexpr int bytes = SampleSmem<T, CLUSTER>::BYTES;
  static std::atomic<uint64_t> done{0};
  SL_CUDA_TRY(allow_smem(sample_kernel<T, CLUSTER>, bytes, done));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)a.max_rows * ctas);
  cfg.blockDim = dim3(SM_THREADS);
  cfg.dynamicSmemBytes = bytes;
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = ctas;
  at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
  cfg.attrs = pdl_enabled() ? at : at + 1;
  cfg.numAttrs = (pdl_enabled() ? 1 : 0) + (CLUSTER ? 1 : 0);
  SL_CUDA_TRY(cudaLaunchKernelEx(&cfg, sample_kernel<T, CLUSTER>, a));
  return SL_OK;
}

template <typename T> int launch_sample_typed(const SampleArgs& a, cudaStream_t st) {
  int ctas = 8;
  while (ctas > 1 && ((long long)a.max_rows * ctas > 2ll * sm_count() || a.vocab < ctas * 4096)) ctas >>= 1;
  while (a.vocab / ctas > (1 << 17) - 16) ctas <<= 1;   // limbs' sums are 32 bits wide
  if ((long long)a.max_rows * ctas > 0x7fffffffll) return SL_EUNSUPPORTED;
  return ctas > 1 ? launch_sample_ctas<T, true>(a, ctas, st) : launch_sample_ctas<T, false>(a, ctas, st);
}

}  // namespace

int launch_sample(const void* logits, long long row_stride, const surelock_sampling& sets, const int32_t* set_of_row, const float* u,
                  const int32_t* n_active, int max_rows, int vocab, int dtype, int32_t* token, float* conf, int32_t* n_kept,
                  int32_t* status, cudaStream_t st) {
  SampleArgs a = {logits, row_stride, sets, set_of_row, n_active, u, token, n_kept, status, conf, max_rows, vocab};
  if (vocab > (1 << 20) - 128) return SL_EUNSUPPORTED;
  return dtype == SL_BF16 ? launch_sample_typed<bf16>(a, st) : launch_sample_typed<float>(a, st);
}

}  // namespace sl
