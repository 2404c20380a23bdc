// A token per row of logits from one given uniform number, with temperature, top-k, top-p and min-p.
//
// With m the row's largest logit and w_v = exp((x_v - m) / T), put the tokens in order of falling x (ties: the lowest index first;
// tokens of -inf do not count).  Each filter keeps a prefix of that order:
//   top-k   the first k;   top-p  of those, the shortest prefix whose weights sum to at least top_p of theirs;
//   min-p   the tokens with w_v >= min_p;
// the token drawn is the first one of the shortest prefix whose running sum of weights exceeds u times the prefix's.  So nothing
// needs sorting: all that is asked of the row is "which token has rank n" and "at which token does the running sum reach s", and
// both are answered by sums over values.  Sums are held in 64 bits: with 100000 tokens in the prefix, 32 would draw a neighbour of
// the right token in one row of a hundred.  (In the bins of the second method below a weight is a whole number of units of 2^-54 of the largest, so each
// token is off by half a unit there; min-p looks at the weight itself.)
//
// bf16 rows (WindowSums): a bf16 number is its own histogram bin.  One pass counts the row's values in shared memory, 5120 bins
// to a sign for magnitudes in [2^-28, 2^12), which leaves the sums to the few thousand distinct values: one exponential each instead of
// one per token, and a sum is exact but for 2^-53 roundings.  The occupied range of bins is then walked in order, a few bins to
// a thread.  The token's index is found by a second pass that counts the tokens of the value that was drawn, out of the L2.  A row with a
// finite value outside the window (not zero) is done by the other method, after it has been counted in vain: tokens forbidden by a large finite number instead
// of -inf cost that (a third of 126464 at -1e4 or the type's lowest value, top-p: 1 row 53 instead of 21 us, 33 rows 111 instead of 27, 1536 rows 1304 instead
// of 207).
//
// fp32 rows (BinnedSums): 2048 bins of equal width over the values that weigh anything.  One pass adds every token's weight, as four limbs of
// a fixed-point number (exact sums in any order), to its bin; a bin that is asked for is opened by another pass over the row's tokens
// in it: a few are ranked against one another, more of them are binned once more by their keys.
//
// A row is one CTA's work, or with few rows that of a cluster of CTAs, whose shares meet through distributed shared memory.
//
// Bounds, and what it measured in a graph: one bf16 row of 126464 tokens with top-k and top-p 21 - 22 us (latency: counting 8.5 k cycles, sums over the
// cluster 5 k, three finds of 3 to 4 k, meeting the token 4.5 k), 33 fp32 rows of 32003 with all filters 41 - 42 us (each find has three cluster barriers and
// a pass over the row), 1536 bf16 rows with top-p 185 us for 388 MB: the counts' atomics meet in a bank 3.4 at a time, 80 us, and what follows
// the counting overlaps another CTA's only in part; a temperature other than 1 adds an exponential to each value that occurs, for conf, 15 us more.  (A search for the k largest and a sort of 126464 numbers per row take 20 ms.)
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
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr));
  return v;
}
__device__ __forceinline__ void add_shared(uint32_t addr, uint32_t v) {
  asm volatile("red.shared.add.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}

// of two 16-bit numbers at a time
__device__ __forceinline__ uint32_t add_u16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("add.u16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.u16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t min_u16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("min.u16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

// all threads of the row: one CTA's, or a cluster's
template <int CTAS> __device__ __forceinline__ void row_sync() {
  if (CTAS > 1) cluster_sync_all(); else __syncthreads();
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

// a token by its place in the order: its rank (0 = the largest), the sum of weights up to and with it, its value's key and which of the
// tokens of that value it is; `entry` is the value's or bin's number, `tokens` how many it has, before_* what lies before it
struct Found {
  double mass, before_w;
  uint32_t rank, key, nth, before_n, tokens, entry;
};

// sums over the whole row: tokens, their weights, those that min-p keeps, and weights at T = 1
struct Totals {
  double w, m, raw;
  uint32_t n, nm;
};

constexpr int MOST_CTAS = 8, MOST_GROUPS = 400;

struct Shared {                     // beside the bins
  double powers[32];                // 2^(i / 32)
  // in the first CTA, written by all of the row's: sums of groups of 32 entries, and every warp's share of the other sums
  double group_w[MOST_GROUPS], warp_m[MOST_CTAS * SM_WARPS], warp_raw[MOST_CTAS * SM_WARPS];
  uint32_t group_n[MOST_GROUPS], warp_nm[MOST_CTAS * SM_WARPS];
  Found found[2];                   // by turns, so that none is overwritten while somebody reads it
  Totals totals;
  uint32_t matches[2][SM_WARPS], cta_matches;
  uint32_t top, lo, hi, flags, zeros, list_n, owner, exps[2];
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

__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ uint32_t warp_sum(uint32_t v) { return __reduce_add_sync(0xffffffffu, v); }

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
  // whether a run with these running sums up to and with it holds it, if none before did
  __device__ bool in(uint32_t incl_n, double incl_w) const { return by_rank ? rank < incl_n : reaches(incl_w, target, strict); }
  // the token among c of weight w, before which there are before_n of sum before_w
  __device__ void among(uint32_t c, double w, Found& f) const {
    const uint32_t j = by_rank ? rank - f.before_n + 1 : tokens_until(f.before_w, w, c, target, strict);
    f.tokens = c;
    f.nth = j - 1;
    f.rank = f.before_n + f.nth;
    f.mass = f.before_w + j * w;
  }
};
__device__ __forceinline__ Ask ask_rank(uint32_t rank) { return {true, false, rank, 0.0}; }
__device__ __forceinline__ Ask ask_mass(double target, bool strict) { return {false, strict, 0u, target}; }

// The first lane of a warp whose n tokens, in and iw being the warp's running sums, hold what is asked for; f.before_*, the sums before the
// warp's, become those before the lane's.  Where roundings leave none: the last lane that has tokens, and its last token is asked for from
// there on.
__device__ __forceinline__ int pick_lane(Ask& ask, uint32_t n, uint32_t in, double iw, Found& f) {
  const unsigned some = __ballot_sync(0xffffffffu, n != 0u), hit = __ballot_sync(0xffffffffu, n && ask.in(f.before_n + in, f.before_w + iw));
  const int l = hit ? __ffs(hit) - 1 : 31 - __clz(some);
  const uint32_t upto = __shfl_sync(0xffffffffu, in, l), mine = __shfl_sync(0xffffffffu, n, l);
  if (!hit) ask = ask_rank(f.before_n + upto - 1);
  const double before = __shfl_sync(0xffffffffu, iw, max(l - 1, 0));
  f.before_n += upto - mine;
  f.before_w += l ? before : 0.0;
  return l;
}
__device__ __forceinline__ int pick_lane(Ask& ask, uint32_t n, double w, Found& f) {
  const int lane = threadIdx.x & 31;
  uint32_t in = n;
  double iw = w;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t a = __shfl_up_sync(0xffffffffu, in, o);
    const double b = __shfl_up_sync(0xffffffffu, iw, o);
    if (lane >= o) {
      in += a;
      iw += b;
    }
  }
  return pick_lane(ask, n, in, iw, f);
}

// The leading warp's view of the groups: every lane has a run of them, with the sums of the run and up to and with it.
struct Ladder {
  uint32_t n, in;
  double w, iw;
  __device__ void climb(const Shared& s, int groups) {
    const int lane = threadIdx.x & 31, per = (groups + 31) >> 5;
    n = 0u;
    w = 0.0;
    for (int g = lane * per; g < min(groups, (lane + 1) * per); ++g) {
      n += s.group_n[g];
      w += s.group_w[g];
    }
    in = n;
    iw = w;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t a = __shfl_up_sync(0xffffffffu, in, o);
      const double b = __shfl_up_sync(0xffffffffu, iw, o);
      if (lane >= o) {
        in += a;
        iw += b;
      }
    }
  }
};

// The entry that holds what is asked for, by one warp: first among 32 runs of groups, then among a run's groups, then among a
// group's 32 entries; entry(i, tokens, weight of a token).
template <typename F> __device__ Found search(const Shared& s, const Ladder& ladder, int groups, Ask& ask, F entry, uint32_t before_n = 0u, double before_w = 0.0) {
  const int lane = threadIdx.x & 31, per = (groups + 31) >> 5;
  Found f;
  f.before_n = before_n;
  f.before_w = before_w;
  int g = pick_lane(ask, ladder.n, ladder.in, ladder.iw, f) * per;
  const bool one = lane < per && g + lane < groups;
  g += pick_lane(ask, one ? s.group_n[g + lane] : 0u, one ? s.group_w[g + lane] : 0.0, f);
  uint32_t c;
  double each;
  entry(32 * g + lane, c, each);
  const int l = pick_lane(ask, c, c * each, f);
  f.entry = 32 * g + l;
  c = __shfl_sync(0xffffffffu, c, l);
  each = __shfl_sync(0xffffffffu, each, l);
  ask.among(c, each, f);
  return f;
}

template <int CTAS> __device__ __forceinline__ uint32_t in_first_cta(const void* p) { return CTAS > 1 ? mapa_u32(smem_u32(p), 0) : smem_u32(p); }
template <int CTAS> __device__ __forceinline__ void put(uint32_t addr, double v) {
  if (CTAS > 1) asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(addr), "d"(v) : "memory");
  else asm volatile("st.shared.f64 [%0], %1;" ::"r"(addr), "d"(v) : "memory");
}
template <int CTAS> __device__ __forceinline__ void put(uint32_t addr, uint32_t v) {
  if (CTAS > 1) asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
  else asm volatile("st.shared.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}
// a struct of whole words to its place in every CTA of the row, lane by lane
template <int CTAS, typename S> __device__ __forceinline__ void publish(S& to, const S& v) {
  static_assert(sizeof(S) % 4 == 0, "whole words");
  uint32_t words[sizeof(S) / 4];
  memcpy(words, &v, sizeof(S));
  const int lane = threadIdx.x & 31;
  if (lane < CTAS) {
    const uint32_t a = CTAS > 1 ? mapa_u32(smem_u32(&to), lane) : smem_u32(&to);
#pragma unroll
    for (int i = 0; i < (int)(sizeof(S) / 4); ++i) put<CTAS>(a + 4 * i, words[i]);
  }
}

// What both methods share.
template <int CTAS> struct Sums {
  Shared& s;
  int cta, groups = 0;
  double inv_T;                     // (x - max) / T as a product: off by 2^-52 of itself
  __device__ Sums(Shared& sh, int c) : s(sh), cta(c) {}
  __device__ bool leads() const { return cta == 0 && threadIdx.x < 32; }   // the warp that searches
  // a group of 32 entries, c tokens of weight cw in all to a lane
  __device__ void put_group(int g, uint32_t c, double cw) {
    c = warp_sum(c);
    cw = warp_sum(cw);
    if ((threadIdx.x & 31) == 0) {
      put<CTAS>(in_first_cta<CTAS>(&s.group_n[g]), c);
      put<CTAS>(in_first_cta<CTAS>(&s.group_w[g]), cw);
    }
  }
  // four groups at once, of which lanes exchange what the others sum: lane's bits 4 and 3 say whose sums it ends with
  __device__ void put_groups4(int g, const uint32_t* c, const double* cw) {
    const int lane = threadIdx.x & 31;
    const bool a = lane & 16, b = lane & 8;
    uint32_t n0 = (a ? c[2] : c[0]) + __shfl_xor_sync(0xffffffffu, a ? c[0] : c[2], 16), n1 = (a ? c[3] : c[1]) + __shfl_xor_sync(0xffffffffu, a ? c[1] : c[3], 16);
    double w0 = (a ? cw[2] : cw[0]) + __shfl_xor_sync(0xffffffffu, a ? cw[0] : cw[2], 16), w1 = (a ? cw[3] : cw[1]) + __shfl_xor_sync(0xffffffffu, a ? cw[1] : cw[3], 16);
    uint32_t n = (b ? n1 : n0) + __shfl_xor_sync(0xffffffffu, b ? n0 : n1, 8);
    double w = (b ? w1 : w0) + __shfl_xor_sync(0xffffffffu, b ? w0 : w1, 8);
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) {
      n += __shfl_xor_sync(0xffffffffu, n, o);
      w += __shfl_xor_sync(0xffffffffu, w, o);
    }
    if ((lane & 7) == 0) {
      const int at = g + (a ? 2 : 0) + (b ? 1 : 0);
      put<CTAS>(in_first_cta<CTAS>(&s.group_n[at]), n);
      put<CTAS>(in_first_cta<CTAS>(&s.group_w[at]), w);
    }
  }
  __device__ void put_rest(const Settings& set, uint32_t nm, double m, double raw) {
    const int at = cta * SM_WARPS + (threadIdx.x >> 5);
    if (set.min_p > 0.0) {
      nm = warp_sum(nm);
      m = warp_sum(m);
    }
    if (inv_T != 1.0) raw = warp_sum(raw);
    if ((threadIdx.x & 31) == 0) {
      put<CTAS>(in_first_cta<CTAS>(&s.warp_nm[at]), nm);
      put<CTAS>(in_first_cta<CTAS>(&s.warp_m[at]), m);
      put<CTAS>(in_first_cta<CTAS>(&s.warp_raw[at]), raw);
    }
  }
  // by the leading warp, after a barrier
  Ladder ladder;
  __device__ Totals total(const Settings& set) {
    const int lane = threadIdx.x & 31;
    Totals t = {};
    ladder.climb(s, groups);
    t.n = __shfl_sync(0xffffffffu, ladder.in, 31);
    t.w = __shfl_sync(0xffffffffu, ladder.iw, 31);
    if (set.min_p > 0.0 || inv_T != 1.0) {
      for (int i = lane; i < CTAS * SM_WARPS; i += 32) {
        t.nm += s.warp_nm[i];
        t.m += s.warp_m[i];
        t.raw += s.warp_raw[i];
      }
      t.nm = warp_sum(t.nm);
      t.m = warp_sum(t.m);
      t.raw = warp_sum(t.raw);
    }
    if (!(set.min_p > 0.0)) t.nm = t.n;
    if (inv_T == 1.0) t.raw = t.w;
    return t;
  }
};

// ---- bf16: counts of values -----------------------------------------------------------------------------------------------
constexpr uint32_t WIN_LO = (127 - 28) << 7, WIN_HI = (127 + 12) << 7, WIN_BINS = WIN_HI - WIN_LO;   // magnitudes' bits
constexpr int EXPS = WIN_BINS / 128;
static_assert(8 * EXPS + 1 <= MOST_GROUPS && EXPS <= 64, "groups and exponents of the window");

// Entries, in falling order: the positive values from the window's top binary exponent down, 128 to an exponent; zero, with 31 empty
// ones behind it; the negative values.  So 32 neighbours have one exponent, and their weights are a geometric sequence.
template <int CTAS> struct WindowSums : Sums<CTAS> {
  typedef Sums<CTAS> F;
  using F::s; using F::cta; using F::groups; using F::inv_T;
  static constexpr int SMEM = 2 * (WIN_BINS + 32) * 4;
  static constexpr uint32_t ZERO = WIN_BINS;          // entry of zero
  uint32_t* bins;                   // [magnitude][sign], and 32 magnitudes for what is outside
  uint32_t zeros;
  unsigned long long exps;          // the binary exponents that occur, the window's lowest first
  double top;
  Totals totals;                    // of the leading warp

  __device__ WindowSums(Shared& sh, void* smem, int c) : F(sh, c), bins(reinterpret_cast<uint32_t*>(smem)) { groups = 8 * EXPS + 1; }

  // Counts the row.  0, ROW_UNDEFINED (a NaN, +inf, or nothing finite) or ROW_OUTSIDE (values outside the window).
  __device__ uint32_t count(const Share<bf16>& row) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint4* b4 = reinterpret_cast<uint4*>(bins);
    for (int i = threadIdx.x; i < SMEM / 16; i += SM_THREADS) b4[i] = make_uint4(0u, 0u, 0u, 0u);
    for (int i = threadIdx.x; i < groups; i += SM_THREADS) {
      s.group_n[i] = 0u;
      s.group_w[i] = 0.0;
    }
    if (threadIdx.x == 0) {
      s.hi = s.flags = s.zeros = s.exps[0] = s.exps[1] = 0u;
      s.lo = WIN_BINS;
    }
    __syncthreads();
    // Two numbers at a time: the place of a magnitude in the window, that of this lane's bin aside where it is outside, and from it and
    // the sign the bin's address.
    constexpr uint32_t START = (0x10000u - WIN_LO) * 0x10001u;
    const uint32_t aside = (WIN_BINS + lane) * 0x10001u;
    auto two = [&](uint32_t w) { return (min_u16x2(add_u16x2(w & 0x7fff7fffu, START), aside) << 3) + ((w >> 13) & 0x00040004u); };
    auto count_one = [&](uint32_t at) { atomicAdd(reinterpret_cast<uint32_t*>(reinterpret_cast<char*>(bins) + at), 1u); };
    const uint4* words = row.words();
    int v = row.v0 + (int)threadIdx.x;
    auto eight = [&](const uint4& u) {
      const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t at = two(w[i]);
        count_one(at & 0xffffu);
        count_one(at >> 16);
      }
    };
    uint4 u[4];                                      // the next words, always on their way
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (v + i * SM_THREADS < row.v1) u[i] = words[v + i * SM_THREADS];
    for (; v < row.v1; v += 4 * SM_THREADS) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint4 now = u[i];
        if (v + (i + 4) * SM_THREADS < row.v1) u[i] = words[v + (i + 4) * SM_THREADS];
        if (v + i * SM_THREADS < row.v1) eight(now);
      }
    }
    const uint16_t* raw = reinterpret_cast<const uint16_t*>(row.row);
    const int at_head = row.first && (int)threadIdx.x < row.head ? (int)threadIdx.x : -1;
    const int at_tail = row.last && row.tail0 + (int)threadIdx.x < row.vocab ? row.tail0 + (int)threadIdx.x : -1;
    if (at_head >= 0) count_one(two(raw[at_head]) & 0xffffu);
    if (at_tail >= 0) count_one(two(raw[at_tail]) & 0xffffu);
    __syncthreads();
    // which binary exponents occur, and the largest positive and the smallest negative magnitude
    for (int x = warp; x < EXPS; x += SM_WARPS) {
      uint32_t hi = 0u, lo = WIN_BINS;
#pragma unroll
      for (int k = 3; k >= 0; --k) {
        const uint32_t m = 128 * x + 32 * k + lane;
        const uint2 c = reinterpret_cast<const uint2*>(bins)[m];
        if (c.x && !hi) hi = m + 1;
        if (c.y) lo = m;
      }
      if (!__any_sync(0xffffffffu, hi || lo < WIN_BINS)) continue;
      hi = __reduce_max_sync(0xffffffffu, hi);
      lo = __reduce_min_sync(0xffffffffu, lo);
      if (lane == 0) {
        atomicOr(&s.exps[x >> 5], 1u << (x & 31));
        atomicMax(&s.hi, hi);
        atomicMin(&s.lo, lo);
      }
    }
    // were there any outside?  zeros are counted apart, -inf is left out, and the rest is for the row to know
    const uint2 out = reinterpret_cast<const uint2*>(bins)[WIN_BINS + lane];
    if (__any_sync(0xffffffffu, out.x | out.y)) {    // the same for all warps
      uint32_t zero = 0u, worst = 0u;                // two at a time
      auto explain = [&](uint32_t w) {
        const __nv_bfloat162 x = *reinterpret_cast<const __nv_bfloat162*>(&w);
        const uint32_t z = __heq2_mask(x, __float2bfloat162_rn(0.f)), none = __heq2_mask(x, __float2bfloat162_rn(-INFINITY));
        zero += z & 0x10001u;
        worst = max_u16x2(worst, add_u16x2(w & 0x7fff7fffu, START) & ~(z | none));
      };
      for (v = row.v0 + (int)threadIdx.x; v < row.v1; v += SM_THREADS) {
        const uint4 w = words[v];
        explain(w.x);
        explain(w.y);
        explain(w.z);
        explain(w.w);
      }
      if (at_head >= 0) explain(raw[at_head] | 0xff800000u);
      if (at_tail >= 0) explain(raw[at_tail] | 0xff800000u);
      zero = warp_sum((zero & 0xffffu) + (zero >> 16));
      uint32_t flags = max(worst & 0xffffu, worst >> 16) < WIN_BINS ? 0u : ROW_OUTSIDE;
      if (__any_sync(0xffffffffu, flags)) {
        row.each([&](float x) {
          if (!(x < INFINITY)) flags |= ROW_UNDEFINED;
        });
        flags = __reduce_or_sync(0xffffffffu, flags);
      }
      if (lane == 0) {
        atomicAdd(&s.zeros, zero);
        atomicOr(&s.flags, flags);
      }
    }
    row_sync<CTAS>();
    uint32_t f = s.flags, hi = s.hi, lo = s.lo, e0 = s.exps[0], e1 = s.exps[1];
    zeros = s.zeros;
    if (CTAS > 1) {
      uint32_t got[CTAS][6];
      const uint32_t from[6] = {smem_u32(&s.flags), smem_u32(&s.hi), smem_u32(&s.lo), smem_u32(&s.exps[0]), smem_u32(&s.exps[1]), smem_u32(&s.zeros)};
#pragma unroll
      for (int c = 0; c < CTAS; ++c)
#pragma unroll
        for (int i = 0; i < 6; ++i) got[c][i] = ld_cluster_u32(mapa_u32(from[i], c));
      zeros = 0u;
#pragma unroll
      for (int c = 0; c < CTAS; ++c) {
        f |= got[c][0];
        hi = max(hi, got[c][1]);
        lo = min(lo, got[c][2]);
        e0 |= got[c][3];
        e1 |= got[c][4];
        zeros += got[c][5];
      }
    }
    exps = (unsigned long long)e1 << 32 | e0;
    if (f) return f & ROW_UNDEFINED ? ROW_UNDEFINED : ROW_OUTSIDE;
    if (!hi && !zeros && lo == WIN_BINS) return ROW_UNDEFINED;
    top = hi ? (double)value(WIN_BINS - hi) : zeros ? 0.0 : (double)value(ZERO + 32 + lo);
    return 0u;
  }
  // value of an entry
  __device__ static float value(uint32_t e) {
    if (e < ZERO) return __uint_as_float((WIN_HI - 1 - e) << 16);
    return e < ZERO + 32 ? 0.f : __uint_as_float(0x80000000u | (WIN_LO + e - ZERO - 32) << 16);
  }
  __device__ double largest_value() const { return top; }
  // tokens of a magnitude, positive and negative
  __device__ uint2 both(uint32_t m) const {
    if (CTAS == 1) return reinterpret_cast<const uint2*>(bins)[m];
    uint2 c[CTAS], sum = make_uint2(0u, 0u);
#pragma unroll
    for (int i = 0; i < CTAS; ++i)
      asm volatile("ld.shared::cluster.v2.u32 {%0, %1}, [%2];" : "=r"(c[i].x), "=r"(c[i].y) : "r"(mapa_u32(smem_u32(bins + 2 * m), i)));
#pragma unroll
    for (int i = 0; i < CTAS; ++i) {
      sum.x += c[i].x;
      sum.y += c[i].y;
    }
    return sum;
  }
  __device__ uint32_t tokens(uint32_t e) const {
    if (e - ZERO < 32u) return e == ZERO ? zeros : 0u;
    const uint2 c = both(e < ZERO ? WIN_BINS - 1 - e : e - ZERO - 32);
    return e < ZERO ? c.x : c.y;
  }
  // of an entry that has tokens
  __device__ double weight(uint32_t e) const { return exp_falling(fmin((double)value(e) - top, 0.0) * inv_T, s.powers); }

  // An exponent at a time, its 4 groups of either sign: 128 neighbours, lane + 32 k from the largest magnitude down.  Weights 32 apart have a fixed
  // ratio, so there is an exponential for it and one for either sign; but in the exponent of the largest logit, where there are values above it.
  __device__ void sum(const Settings& set) {
    inv_T = set.greedy ? 1.0 : 1.0 / set.T;
    const int lane = threadIdx.x & 31, mine = cta * SM_WARPS + (threadIdx.x >> 5);
    uint32_t nm = 0u;
    double m = 0.0, raw = 0.0;
    auto account = [&](uint32_t c, double w, double cw, uint32_t e) {
      if (inv_T != 1.0 && c) raw += c * exp_falling(fmin((double)value(e) - top, 0.0), s.powers);
      if (set.min_p > 0.0 && w >= set.min_p) {
        nm += c;
        m += cw;
      }
    };
    auto four = [&](const uint32_t* c, uint32_t e, double ratio) {
      if (!__any_sync(0xffffffffu, c[0] | c[1] | c[2] | c[3])) return;
      const bool with_top = (double)value(e & ~127u | (e < ZERO ? 0u : 32u)) > top;
      double w = 0.0, cw[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        w = k == 0 || with_top ? weight(e + 32 * k) : w * ratio;
        cw[k] = c[k] ? c[k] * w : 0.0;
        account(c[k], w, cw[k], e + 32 * k);
      }
      this->put_groups4((int)(e >> 5), c, cw);
    };
    int turn = 0;
    for (unsigned long long left = exps; left; left &= left - 1, ++turn) {
      if (turn % (CTAS * SM_WARPS) != mine) continue;
      const uint32_t x = __ffsll((long long)left) - 1, big = 128 * x + 127 - lane;   // the lane's largest magnitude
      uint32_t pos[4], neg[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint2 c = both(big - 32 * k);
        pos[k] = c.x;
        neg[3 - k] = c.y;
      }
      const double ratio = exp_falling(((double)value(WIN_BINS - 1 - big + 32) - (double)value(WIN_BINS - 1 - big)) * inv_T, s.powers);
      four(pos, WIN_BINS - 1 - big, ratio);
      four(neg, ZERO + 32 + big - 96, ratio);
    }
    if (turn % (CTAS * SM_WARPS) == mine && zeros) {
      const uint32_t c = lane ? 0u : zeros;
      const double w = weight(ZERO), cw = c * w;
      account(c, w, cw, ZERO);
      this->put_group(ZERO / 32, c, cw);
    }
    this->put_rest(set, nm, m, raw);
    row_sync<CTAS>();
    if (this->leads()) totals = this->total(set);
  }
  // by the leading warp alone
  __device__ Found find(const Share<bf16>&, Ask ask) const {
    Found f = search(s, this->ladder, groups, ask, [&](int e, uint32_t& c, double& w) {
      c = tokens(e);
      w = c ? weight(e) : 0.0;
    });
    f.key = key_of(value(f.entry));
    return f;
  }
};

// ---- any type: bins with exact sums of weights ---------------------------------------------------------------------------------
constexpr int BINS = 2048, LIMBS = 4, LIMB_BITS = 14;   // of a weight in units of 2^-54; 2^17 tokens to a CTA fit a 32-bit sum of limbs
constexpr double WEIGHT_UNIT = 18014398509481984.0;     // 2^54
constexpr int LIST = 256;                               // tokens that are ranked against one another

template <typename T, int CTAS> struct BinnedSums : Sums<CTAS> {
  typedef Sums<CTAS> F;
  using F::s; using F::cta; using F::groups; using F::inv_T;
  static constexpr int SMEM = BINS * (1 + LIMBS) * 4 + LIST * 16;
  uint32_t* bins;                   // [1 + LIMBS][BINS]: tokens, limbs
  unsigned long long* weights;      // [LIST]
  uint32_t *list, *keys;            // [LIST]: this CTA's tokens of a bin, and those of the whole row
  float topf, step;                 // the largest, and bins to a unit of the logits
  int turn = 0;
  bool whole = false;               // the bins are those of the whole row
  Totals totals;

  __device__ BinnedSums(Shared& sh, void* smem, int c) : F(sh, c) {
    bins = reinterpret_cast<uint32_t*>(smem);
    weights = reinterpret_cast<unsigned long long*>(bins + BINS * (1 + LIMBS));
    list = reinterpret_cast<uint32_t*>(weights + LIST);
    keys = list + LIST;
    groups = BINS / 32;
  }
  // the row's largest and smallest finite logits; 0 or ROW_UNDEFINED
  __device__ uint32_t range(const Share<T>& row, float& least) {
    row_sync<CTAS>();                            // nobody reads what these words held before
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
    row_sync<CTAS>();
    t = s.top;
    lo = s.lo;
    flags = s.flags;
    for (int c = 0; CTAS > 1 && c < CTAS; ++c) {
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
  __device__ double weight_of(float x) const { return exp_falling(((double)x - (double)topf) * inv_T, s.powers); }
  __device__ static unsigned long long units(double w) { return __double2ull_rn(w * WEIGHT_UNIT); }
  __device__ unsigned long long weight(float x) const { return units(weight_of(x)); }
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
  // a bin summed over the row: tokens and their mean weight
  __device__ void entry(uint32_t e, uint32_t& c, double& w) const {
    const uint32_t a = smem_u32(bins + e);
    unsigned long long limb[LIMBS] = {};
    c = 0u;
    uint32_t part[CTAS][1 + LIMBS];
#pragma unroll
    for (int p = 0; p < CTAS; ++p)
#pragma unroll
      for (int l = 0; l <= LIMBS; ++l) part[p][l] = CTAS > 1 ? ld_cluster_u32(mapa_u32(a, p) + 4 * BINS * l) : bins[e + BINS * l];
#pragma unroll
    for (int p = 0; p < CTAS; ++p) {
      c += part[p][0];
#pragma unroll
      for (int l = 0; l < LIMBS; ++l) limb[l] += part[p][l + 1];
    }
    double v = 0.0;
#pragma unroll
    for (int l = LIMBS - 1; l >= 0; --l) v = v * (double)(1 << LIMB_BITS) + (double)limb[l];
    w = v / (WEIGHT_UNIT * max(c, 1u));
  }
  __device__ void collect() {
    for (int g = cta * SM_WARPS + (threadIdx.x >> 5); g < groups; g += CTAS * SM_WARPS) {
      uint32_t c;
      double w;
      entry(32 * g + (threadIdx.x & 31), c, w);
      this->put_group(g, c, c * w);
    }
  }
  template <typename G> __device__ void bin_all(const Share<T>& row, G also) {
    clear();
    row.each([&](float x) {
      if (x == -INFINITY) return;
      const double w = weight_of(x);
      add(bin_of(x), units(w));
      also(x, w);
    });
    row_sync<CTAS>();
    collect();
    whole = true;
  }
  __device__ void sum(const Share<T>& row, const Settings& set, float least) {
    inv_T = set.greedy ? 1.0 : 1.0 / set.T;
    // beyond 50 T the weights are below 2^-72 of the largest
    const float span = (float)fmin((double)topf - (double)least, 50.0 / inv_T);
    step = span > 0.f ? fminf((float)BINS / span, 3.4e38f) : 0.f;
    uint32_t nm = 0u;
    double m = 0.0, raw = 0.0;
    bin_all(row, [&](float x, double w) {
      if (inv_T != 1.0) raw += exp_falling((double)x - (double)topf, s.powers);
      if (set.min_p > 0.0 && w >= set.min_p) {           // the weight itself: in units of the sums a small one is no number to compare
        ++nm;
        m += (double)units(w) / WEIGHT_UNIT;
      }
    });
    this->put_rest(set, nm, m, raw);
    row_sync<CTAS>();
    if (this->leads()) publish<CTAS>(s.totals, this->total(set));
    row_sync<CTAS>();
    totals = s.totals;
  }
  // the bin that holds what is asked for, for all threads; also whether roundings had it changed
  __device__ Found open(Ask& ask, uint32_t before_n, double before_w) {
    Found& slot = s.found[turn];
    turn ^= 1;
    if (this->leads()) {
      Ask mine = ask;
      this->ladder.climb(s, groups);
      const Found f = search(s, this->ladder, groups, mine, [&](int e, uint32_t& c, double& w) { entry(e, c, w); }, before_n, before_w);
      publish<CTAS>(slot, f);
    }
    row_sync<CTAS>();
    const Found f = slot;
    // the target lies behind the whole of what was searched: its last token
    if (!ask.by_rank && !reaches(f.mass, ask.target, ask.strict) && f.nth == f.tokens - 1) ask = ask_rank(f.rank);
    return f;
  }
  // Members of a bin: of the first binning, and where that was not enough keys from ka to kb.
  struct Members {
    uint32_t bin, ka, kb;
  };
  __device__ bool in(const Members& b, float x, uint32_t k) const { return x != -INFINITY && bin_of(x) == b.bin && k >= b.ka && k <= b.kb; }

  __device__ Found find(const Share<T>& row, Ask ask) {
    if (!whole) {                                   // an earlier find has opened a bin
      bin_all(row, [](float, double) {});
      row_sync<CTAS>();
    }
    Found f = open(ask, 0u, 0.0);
    Members b = {f.entry, 0u, 0xffffffffu};
    while (f.tokens > LIST) {
      // the keys that occur, and bins for them
      whole = false;
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
      row_sync<CTAS>();
      lo = s.lo;
      hi = s.hi;
      for (int c = 0; CTAS > 1 && c < CTAS; ++c) {
        lo = min(lo, ld_cluster_u32(mapa_u32(smem_u32(&s.lo), c)));
        hi = max(hi, ld_cluster_u32(mapa_u32(smem_u32(&s.hi), c)));
      }
      if (lo == hi) {                               // one value: no need to look at its tokens
        ask.among(f.tokens, (double)weight(value_of(lo)) / WEIGHT_UNIT, f);
        f.key = lo;
        row_sync<CTAS>();
        return f;
      }
      const int shift = max(0, 21 - __clz(hi - lo));  // 32 - clz bits, of which the bins tell 11
      row.each([&](float x) {
        const uint32_t k = key_of(x);
        if (in(b, x, k)) add((hi - k) >> shift, weight(x));
      });
      row_sync<CTAS>();
      collect();
      row_sync<CTAS>();
      f = open(ask, f.before_n, f.before_w);
      b.kb = hi - (f.entry << shift);
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
    row_sync<CTAS>();
    const uint32_t n = f.tokens, i = threadIdx.x;
    if (i < n) {
      uint32_t at = i, k = 0u;
      for (int c = 0; c < CTAS; ++c) {
        const uint32_t has = CTAS > 1 ? ld_cluster_u32(mapa_u32(smem_u32(&s.list_n), c)) : s.list_n;
        if (at < has) {
          k = CTAS > 1 ? ld_cluster_u32(mapa_u32(smem_u32(list + at), c)) : list[at];
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
      if (ask.in(f.before_n + before + same, cum + same * w)) atomicMin(&s.owner, before);
    }
    __syncthreads();
    const bool none = s.owner == 0xffffffffu;        // by roundings: the last token
    Found& here = s.found[turn];
    turn ^= 1;
    if (i < n && (none ? before + same == n : before == s.owner)) {
      if (none) ask = ask_rank(f.before_n + n - 1);
      Found g = f;
      g.before_w = f.before_w + (double)sum / WEIGHT_UNIT;
      g.before_n = f.before_n + before;
      g.key = keys[i];
      ask.among(same, (double)weights[i] / WEIGHT_UNIT, g);
      here = g;                                      // equal tokens write the same
    }
    row_sync<CTAS>();
    return here;
  }
};

// The settings' prefix and the token drawn from it: up to four finds, one after another.
template <typename S, typename T> __device__ Found draw(S& sums, const Share<T>& row, const Settings& set, uint32_t& kept) {
  const Totals& q = sums.totals;
  uint32_t n = q.n;
  double mass = q.w;
  enum { TOP_K, TOP_P, MIN_P, DRAW, LAST };
  Found f;
#pragma unroll 1
  for (int step = TOP_K;; ++step) {
    Ask ask;
    if (step == TOP_K) {
      if (set.top_k <= 0 || (uint32_t)set.top_k >= n || set.greedy) continue;
      ask = ask_rank((uint32_t)set.top_k - 1);
    } else if (step == TOP_P) {
      if (!(set.top_p < 1.0) || set.greedy) continue;
      ask = ask_mass(set.top_p * mass, false);
    } else if (step == MIN_P) {                      // keeps the largest at least: its weight is 1
      if (set.greedy) n = 1u;
      else if (q.nm < n) {
        n = q.nm;
        mass = q.m;
      }
      continue;
    } else if (step == DRAW && !set.greedy) ask = ask_mass((double)set.u * mass, true);
    else ask = ask_rank(n - 1);                      // the largest, or by roundings the prefix's last
    f = sums.find(row, ask);
    if (step <= TOP_P) {
      if (f.rank < n - 1) {
        n = f.rank + 1;
        mass = f.mass;
      }
    } else if (f.rank < n) break;
  }
  kept = n;
  return f;
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
template <typename T, int CTAS>
__device__ void write_token(Shared& s, const Share<T>& row, const Found& f, int cta, int32_t* token) {
  constexpr int V = Share<T>::V;
  // one CTA looks at a quarter of the row after the other until it has met the token: 5 / 8 of it on average (all of it at once: 51 us
  // more for 1536 rows of 126464); a cluster's shares are short and looked at as a whole
  constexpr int ROUNDS = CTAS == 1 ? 4 : 1;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const float x = value_of(f.key);
  const Matcher<T> equal(x);
  const uint4* words = row.words();
  const long long all_words = row.v1 - row.v0;
  uint32_t met = 0u;                                 // in the rounds so far
  for (int round = 0; round < ROUNDS; ++round) {
    const int part = round * SM_WARPS + warp;
    const int a = row.v0 + (int)(all_words * part / (ROUNDS * SM_WARPS)), b = row.v0 + (int)(all_words * (part + 1) / (ROUNDS * SM_WARPS));
    const int heads = row.first && part == 0 ? row.head : 0, tails = row.last && part == ROUNDS * SM_WARPS - 1 ? row.vocab - row.tail0 : 0;
    uint32_t n = 0u;
    int v = a + lane;
    uint4 u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (v + 32 * i < b) u[i] = words[v + 32 * i];
    for (; v < b; v += 128) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint4 now = u[i];
        if (v + 32 * (i + 4) < b) u[i] = words[v + 32 * (i + 4)];
        if (v + 32 * i < b) n += equal.number(now);
      }
    }
    const bool in_head = lane < heads && to_f(row.row[lane]) == x, in_tail = lane < tails && to_f(row.row[row.tail0 + lane]) == x;
    n = warp_sum(n + in_head + in_tail);
    uint32_t* matches = s.matches[round & 1];
    if (lane == 0) matches[warp] = n;
    __syncthreads();
    uint32_t before = 0u;
#pragma unroll
    for (int i = 0; i < SM_WARPS; ++i) {
      if (i == warp) before = met;
      met += matches[i];
    }
    if (CTAS > 1) {
      if (threadIdx.x == 0) s.cta_matches = met;
      cluster_sync_all();
      for (int c = 0; c < cta; ++c) before += ld_cluster_u32(mapa_u32(smem_u32(&s.cta_matches), c));
    } else if (f.nth >= met) continue;               // all warps go on to the next round
    if (f.nth < before || f.nth >= before + n) return;
    uint32_t left = f.nth - before;                  // of this warp's tokens of that value
    const uint32_t head_at = __ballot_sync(0xffffffffu, in_head);
    if (left < (uint32_t)__popc(head_at)) {
      if (in_head && (uint32_t)__popc(head_at & ((1u << lane) - 1)) == left) *token = lane;
      return;
    }
    left -= __popc(head_at);
    for (int v0 = a; v0 < b; v0 += 32) {
      v = v0 + lane;
      uint32_t m = v < b ? equal.bits(words[v]) : 0u, sum = __popc(m);
      const uint32_t here = warp_sum(sum);
      if (left >= here) {
        left -= here;
        continue;
      }
      const uint32_t mine = sum;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t y = __shfl_up_sync(0xffffffffu, sum, o);
        if (lane >= o) sum += y;
      }
      if (sum > left && sum - mine <= left) {
        for (uint32_t skip = left - (sum - mine); skip > 0; --skip) m &= m - 1;
        *token = row.head + v * V + __ffs(m) - 1;
      }
      return;
    }
    const uint32_t tail_at = __ballot_sync(0xffffffffu, in_tail);
    if (in_tail && (uint32_t)__popc(tail_at & ((1u << lane) - 1)) == left) *token = row.tail0 + lane;
    return;
  }
}

template <typename T, int CTAS> struct SampleSmem {
  static constexpr int BYTES = BinnedSums<T, CTAS>::SMEM;
};
template <int CTAS> struct SampleSmem<bf16, CTAS> {
  static constexpr int W = WindowSums<CTAS>::SMEM, R = BinnedSums<bf16, CTAS>::SMEM, BYTES = W > R ? W : R;
};

// by one thread of the row, which has the sums
template <typename S> __device__ void write_rest(const S& sums, const Found& f, uint32_t kept, const SampleArgs& a, int r) {
  if (a.conf) a.conf[r] = (float)(exp_falling((double)value_of(f.key) - sums.largest_value(), sums.s.powers) / sums.totals.raw);
  if (a.n_kept) a.n_kept[r] = (int32_t)kept;
}

// apart, so that the bf16 rows' method keeps its registers
template <typename T, int CTAS>
__device__ __noinline__ uint32_t sample_binned(Shared& s, void* smem, const Share<T>& row, const Settings& set, const SampleArgs& a, int r,
                                               int cta) {
  BinnedSums<T, CTAS> sums(s, smem, cta);
  float least;
  const uint32_t state = sums.range(row, least);
  if (state == 0u) {
    sums.sum(row, set, least);
    uint32_t kept;
    const Found f = draw(sums, row, set, kept);
    if (cta == 0 && threadIdx.x == 0) write_rest(sums, f, kept, a, r);
    write_token<T, CTAS>(s, row, f, cta, a.token + r);
  }
  return state;
}

template <typename T, int CTAS>
__device__ __forceinline__ void sample_row(const SampleArgs& a, Shared& s, unsigned char* smem, int r, int cta) {
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
  const Share<T> row((const T*)a.logits + r * a.row_stride, a.vocab, cta, CTAS);
  uint32_t state = ROW_UNDEFINED;
  if (set.ok) {
    bool binned = true;
    if constexpr (sizeof(T) == 2) {
      WindowSums<CTAS> sums(s, smem, cta);
      state = sums.count(row);
      binned = state == ROW_OUTSIDE;
      if (state == 0u) {
        sums.sum(set);
        if (sums.leads()) {
          uint32_t kept;
          const Found f = draw(sums, row, set, kept);
          publish<CTAS>(s.found[0], f);
          if (threadIdx.x == 0) write_rest(sums, f, kept, a, r);
        }
        row_sync<CTAS>();
        write_token<T, CTAS>(s, row, s.found[0], cta, a.token + r);
      }
    }
    if (binned) {
      const Share<T> row1 = row;                     // copies: the function wants their addresses
      const Settings set1 = set;
      state = sample_binned<T, CTAS>(s, smem, row1, set1, a, r, cta);
    }
  }
  if (state == ROW_UNDEFINED && cta == 0 && threadIdx.x == 0) {
    a.token[r] = -1;
    if (a.conf) a.conf[r] = __int_as_float(0x7fffffff);
    if (a.n_kept) a.n_kept[r] = 0;
  }
}

template <typename T, int CTAS>
__global__ void __launch_bounds__(SM_THREADS, 2) sample_kernel(const __grid_constant__ SampleArgs a) {
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ Shared s;
  griddep_wait();
  griddep_launch();
  if (threadIdx.x < 32) s.powers[threadIdx.x] = exp2(threadIdx.x / 32.0);   // seen after the first barrier
  const int r = blockIdx.x / CTAS, cta = CTAS > 1 ? (int)cluster_ctarank() : 0;
  if (r >= min(*a.n_active, a.max_rows)) return;
  sample_row<T, CTAS>(a, s, smem, r, cta);
  if (CTAS > 1) cluster_sync_all();                   // nobody reads this CTA's shared memory any more
}

template <typename T, int CTAS>
int launch_sample_ctas(const SampleArgs& a, cudaStream_t st) {
  constexpr int bytes = SampleSmem<T, CTAS>::BYTES;
  static std::atomic<uint64_t> done{0};
  SL_CUDA_TRY(allow_smem(sample_kernel<T, CTAS>, bytes, done));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)a.max_rows * CTAS);
  cfg.blockDim = dim3(SM_THREADS);
  cfg.dynamicSmemBytes = bytes;
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = CTAS;
  at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
  cfg.attrs = pdl_enabled() ? at : at + 1;
  cfg.numAttrs = (pdl_enabled() ? 1 : 0) + (CTAS > 1 ? 1 : 0);
  SL_CUDA_TRY(cudaLaunchKernelEx(&cfg, sample_kernel<T, CTAS>, a));
  return SL_OK;
}

template <typename T> int launch_sample_typed(const SampleArgs& a, cudaStream_t st) {
  // A cluster shortens a row's passes and pays for its barriers and for the histograms' way through distributed shared memory.  Rows of 126464, T 0.8, top-k
  // 50 and top-p 0.95, us with 1 / 2 / 4 / 8 CTAs, bf16: 1 row 27 / 27 / 23 / 23, 18 rows 33 / 27 / 23 / 29, 37: 33 / 29 / 29 / 45, 74: 33 / 29 / 45 / 72,
  // 148: 33 / 39 / 68 / 123; fp32: 1 row 206 / 127 / 78 / 58, 18 rows 224 / 129 / 81 / 73, 37: 225 / 133 / 103 / 125, 148: 226 / 178 / 263 / 342, 296: 372 / 355 /
  // 457 / 639.  Rows of 32000, bf16: 1 row 21 / 19 / 20 / 23, 37: 21 / 21 / 25 / 43, 148: 21 / 27 / 57 / 112; fp32: 1 row 70 / 49 / 39 / 40, 18: 73 / 51 / 41 /
  // 47, 37: 72 / 52 / 48 / 82, 148: 74 / 68 / 127 / 219, 296: 98 / 128 / 216 / 403.  So many CTAs while each has an SM and more to itself, two up to about one
  // CTA (fp32: two) per SM, and 4096 tokens to a CTA at least (8 of them for one row of 32000: 2 us more in bf16 than with 4, 1 in fp32).
  const long long room = (long long)sm_count() * (sizeof(T) == 2 ? 1 : 2);
  int ctas = 8;
  while (ctas > 1 && ((long long)a.max_rows * ctas > (ctas == 2 ? room : room / 2) || a.vocab < ctas * 4096)) ctas >>= 1;
  while (a.vocab / ctas > (1 << 17) - 16) ctas <<= 1;   // limbs' sums are 32 bits wide
  if ((long long)a.max_rows * ctas > 0x7fffffffll) return SL_EUNSUPPORTED;
  return ctas == 8   ? launch_sample_ctas<T, 8>(a, st)
         : ctas == 4 ? launch_sample_ctas<T, 4>(a, st)
         : ctas == 2 ? launch_sample_ctas<T, 2>(a, st)
                     : launch_sample_ctas<T, 1>(a, st);
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
