// Attention of few query rows per sequence against a paged K/V cache in bf16, e4m3 or int8 (Algorithm 1 line 12 over a
// cache in pages; with one row per sequence, the attention of a new token):
//
//   o[r][h] = sum_j p_j V_j / sum_j p_j,   p_j = exp(q[r][h] . K_j / sqrt(d_h)),   j < seq_len of the row's sequence,
//
// K_j = sk_j * ck_j and V_j = sv_j * cv_j with codes c and one fp32 scale per (token, head).  H query heads share Hkv heads
// of keys (head h reads head h / (H / Hkv)); the H / Hkv heads of a row are "rows" of one query tile, so a cache byte is read
// once for all of them.
//
// What bounds it: the cache is read once, 2 len (d_h + 4) bytes per key head, and each code takes part in 2 x 16 (padded)
// multiply-adds, so the kernel streams.  Work is cut into UNITS of 64 keys of one (sequence, key head, tile of 16 MT rows);
// all units of the call, in order, are dealt to the CTAs in equal contiguous runs whatever the sequences' lengths are
// (derived on the device from seq_lens and row_offsets).  A run that covers an item whole writes o; the pieces of an item cut
// by run borders leave (unnormalised O, maximum, sum) in the workspace and attention_paged_join_kernel, launched behind
// with programmatic dependent launch, adds them in unit order: no atomics, no counters, nothing kept between calls.
//   warp 4     producer: TMA boxes of a page (and of its scales) into a ring of stages, 128-byte (64-byte for rows of 64
//              bytes) swizzle; a page number outside the pool is replaced by one past its end, which TMA fills with zeros
//   warps 0-3  with up to 8 rows to a tile: each warp alone with 16 keys of the unit, keys and columns of V as the 16-row
//              operand of mma.sync m16n8k16, rows as the 8 columns: S^T = K Q^T, exp2, the weights transposed in registers, and
//              O^T += V^T P; the four warps' O, maxima and sums meet once per item.  With tiles of 16 or 32 rows: S = Q K^T for
//              16 keys each (a tile of 16 rows is an eighth of a tcgen05 tile), exp2, the weights into shared memory as the A
//              fragments they already are; then O += P V for a quarter of the columns each, over all 64 keys.  Codes become
//              fp16, exactly, in registers on the way to the products.
// Measured in replayed graphs (a plain copy: 6.57 TB/s): one new token each, 4 x 16384 tokens of 32 key heads in e4m3 85 us (6.5 TB/s), 32
// ragged sequences of up to 4099 tokens of 8 key heads 38 us (5.4 TB/s); 8 x 4096 tokens in bf16 87 us (6.2 TB/s); 16 rows each,
// 4 x 8192 tokens in e4m3 64 us, 32 rows each 92 us: there the products and the conversions bound it; 23 rows of one sequence
// of 512 tokens 11 us, launches and waits.
// The contraction index is permuted (the same way for Q and K) so that a lane reads its share of a key as 16-byte loads, and
// the columns of O so that it reads neighbouring bytes of a value row; two keys' bytes are interleaved by byte permutes.
// Numerics: q becomes fp16 times a power of two per row (its largest magnitude in [1, 2)), the weight w_j = p_j sv_j becomes
// fp16 under a power of two per row that follows the row's largest weight so far; both keep 11 bits, and weights below
// 2^-33 of the largest vanish.  For w that is a choice: the results' error against the definition is 1 % above that of their
// own rounding to bf16 (0.00168 against 0.00166, relative to the values), and a second fp16 term for what the first leaves cost
// 1 to 11 % for single tokens, 12 % for 16 rows, 19 % for 32.  S, the statistics and O are fp32.  O is rescaled when a maximum
// grows by more than 2^6 or a weight outgrows its power of two.  With a bf16 cache V cannot become fp16, so q is bf16 as it is and
// p two bf16 terms, p rounded and what that left, of 16 bits together: with the first term alone (8 bits) the error was a third
// above that of the results' rounding (0.0022 against 0.0017; 5 sequences of 33 rows and 64 columns 17.8 us with one term, 19.0
// with two).
#include "paged_kv.cuh"
#include "tc_common.cuh"

namespace sl {

namespace {

constexpr int AP_THREADS = 160;
constexpr int AP_KEYS = 64;                // keys per unit
constexpr int AP_MAX_B = 1024;
constexpr float AP_TAU = 6.f;              // log2 growth of a row maximum that is tolerated before O is rescaled
constexpr int AP_W_EXP = 8;                // a weight of exponent E becomes an fp16 of exponent AP_W_EXP ...
constexpr float AP_W_MOST = 32768.f;       // ... and one that would pass this makes E follow it
constexpr int AP_E_LEAST = -110;           // smallest E: 2^(AP_W_EXP - E) stays a normal fp32 number

struct PagedAttnArgs {
  const int32_t *row_offsets, *seq_lens, *table;
  const bf16* q;
  bf16* o;
  long long q_stride, o_stride;
  int B, Hkv, G, max_rows, n_pages, page_size, max_pages, max_tokens;
  float scale_log2;
  int4* desc;      // [grid]: {first packed row of the sequence, first row of the tile, valid rows << 16 | key head, last CTA} of the
                   // item that starts in this CTA and goes on in later ones; valid rows = 0: none
  float2* ml;      // [grid][2][rows]
  float* part;     // [grid][2][rows][DH]
  int32_t* status;
  int lost;        // bytes that the second CTA's first stage waits for in vain: 0, but for the diagnostic
};

__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, int w, uint32_t bar, uint64_t policy) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%2, %3, %4, %5}], [%6], %7;"
      ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(bar), "l"(policy)
      : "memory");
}
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
      ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
      : "memory");
}
__device__ __forceinline__ uint4 lds128(uint32_t a) {
  uint4 r;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "r"(a) : "memory");
  return r;
}
__device__ __forceinline__ uint32_t lds32(uint32_t a) {
  uint32_t r;
  asm volatile("ld.shared.b32 %0, [%1];" : "=r"(r) : "r"(a) : "memory");
  return r;
}
__device__ __forceinline__ uint2 lds64(uint32_t a) {
  uint2 r;
  asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(r.x), "=r"(r.y) : "r"(a) : "memory");
  return r;
}
// 8 x 8 matrix of 16-bit elements, two of a row per lane
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}
__device__ __forceinline__ void ldsm_x4_t(uint32_t a, uint32_t* r) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
// bounded wait of a whole warp, with the same answer in every lane
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
  return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag));
}
// whether the flag is set in any of the 128 consumer threads; also a barrier of them
__device__ __forceinline__ bool consumers_any(bool x) {
  int r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.b32 q, %1, 0;\n\t"
      "bar.red.or.pred p, 3, 128, q;\n\t"
      "selp.b32 %0, 1, 0, p;\n\t}"
      : "=r"(r) : "r"((int)x) : "memory");
  return r != 0;
}
__device__ __forceinline__ void bar_consumers() { asm volatile("bar.sync 2, 128;" ::: "memory"); }

// c += a b, m16n8k16, fp32 accumulators, both operands bf16 or both fp16
template <bool BF> __device__ __forceinline__ void mma16(float* c, const uint4& a, uint32_t b0, uint32_t b1) {
  if (BF)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b0), "r"(b1));
}

// bytes 0,1 (LO) or 2,3 of a word of codes as two fp16 values, exactly.  int8: the byte (offset by 128) becomes the low bits
// of 1024 + u, an fp16 whose unit is 1.
template <int KIND> __device__ __forceinline__ void codes_to_f16(uint32_t w, uint32_t& lo, uint32_t& hi) {
  if (KIND == SL_E4M3) {
    lo = e4m3x2_to_f16x2((uint16_t)(w & 0xffffu));
    hi = e4m3x2_to_f16x2((uint16_t)(w >> 16));
  } else {
    const uint32_t u = w ^ 0x80808080u;
    const uint32_t a = __byte_perm(u, 0x64646464u, 0x4140), b = __byte_perm(u, 0x64646464u, 0x4342);
    const __half2 off = __halves2half2(__ushort_as_half(0x6480), __ushort_as_half(0x6480));   // 1152
    const __half2 x = __hsub2(*reinterpret_cast<const __half2*>(&a), off), y = __hsub2(*reinterpret_cast<const __half2*>(&b), off);
    lo = *reinterpret_cast<const uint32_t*>(&x);
    hi = *reinterpret_cast<const uint32_t*>(&y);
  }
}
__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
  const __half2 v = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}
// two values as bf16; what the rounding left of them takes their place
__device__ __forceinline__ uint32_t take_bf16(float& a, float& b) {
  const uint32_t w = pack_bf16(a, b);
  a -= __uint_as_float(w << 16);
  b -= __uint_as_float(w & 0xffff0000u);
  return w;
}
__device__ __forceinline__ float pow2i(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }   // -126 <= e <= 127

// rows of a query tile: MT tiles of 16 as the 16-row operand of the products, or (MT = 0) 8 as their columns
template <int MT> __host__ __device__ constexpr int ap_rows() { return MT == 0 ? 8 : 16 * MT; }

// one sequence's share of the units
struct Seq {
  int r0, rows, len, tiles, nb;   // first packed row, rows, keys, query tiles, units per (key head, tile)
};
template <int MT> __device__ __forceinline__ Seq seq_of(const PagedAttnArgs& a, int b) {
  Seq s;
  s.r0 = min(max(a.row_offsets[b], 0), a.max_rows);   // both clamped before the difference, which then cannot overflow
  s.rows = min(max(a.row_offsets[b + 1], 0), a.max_rows) - s.r0;
  const int len = a.seq_lens[b];
  s.len = min(max(len, 0), a.max_tokens);
  s.tiles = s.rows > 0 ? (int)(((long long)s.rows * a.G + ap_rows<MT>() - 1) / ap_rows<MT>()) : 0;
  s.nb = max(1, (s.len + AP_KEYS - 1) / AP_KEYS);   // a sequence without keys has one unit, which writes its zeros
  return s;
}

template <int DH, int KIND> struct Tile {
  static constexpr int ROW = DH * KvKind<KIND>::BYTES;          // bytes of a key: 64, 128 or 256
  static constexpr int SLABS = ROW > 128 ? ROW / 128 : 1;       // column blocks of at most 128 bytes
  static constexpr int SLAB_ROW = ROW > 128 ? 128 : ROW;
  static constexpr int SLAB = AP_KEYS * SLAB_ROW;
  static constexpr int KV = SLABS * SLAB;
  static constexpr bool SCALED = KIND != SL_BF16;
  static constexpr int STAGE = 2 * KV + (SCALED ? 1024 : 0);    // K, V, K scales, V scales (512 bytes each)
  static constexpr int STEPS = DH / 16;
};
// CTAs per SM, and stages of the ring: what then fits the shared memory.  (Single tokens, 4 x 16384 in e4m3: 85 us with three
// CTAs of three stages, 93 with registers for four, which fit with two stages at most, 89 with two CTAs of five.)
constexpr int AP_OCC = 3;
template <int DH, int KIND, int MT> struct Plan {
  using T = Tile<DH, KIND>;
  static constexpr int TILES = MT ? MT : 1;
  static constexpr int TERMS = KIND == SL_BF16 ? 2 : 1;         // of a weight
  static constexpr int EXCHANGE = MT ? TERMS * MT * 4 * 512 : 4 * 8 * (DH + 4) * 4;   // weights, or the warps' results
  static constexpr int FIXED = 1024 + TILES * T::STEPS * 512 + EXCHANGE + 16 * TILES * 4 * 9 + 256;   // Q, exchange, row factors, statistics
  static constexpr int ROOM = 228 * 1024 / AP_OCC - 1024 - 256 - FIXED;                             // 256: prefix sums of up to 31 sequences
  static constexpr int FIT = ROOM / T::STAGE;
  static constexpr int STAGES = FIT < 2 ? 2 : FIT > 6 ? 6 : FIT;
  static constexpr int SMEM = FIXED + STAGES * T::STAGE;                                           // and 8 bytes per sequence
};

// a row's bf16 words (this lane's W of them, LANES lanes to the row) become fp16 times a power of two that brings the row's
// largest magnitude into [1, 2); returns the inverse power.  In two factors each, as 2^-126 ... 2^127 need not be normal
// numbers both ways; a row with an infinity or NaN stays as it is.
template <int W, int LANES> __device__ __forceinline__ float rows_to_f16(uint32_t* w) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < W; ++i) top = max(top, max(w[i] & 0x7fffu, (w[i] >> 16) & 0x7fffu));
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
  int ex = (int)(top >> 7) - 127;
  ex = top == 0 || ex > 127 ? 0 : max(ex, -126);
  const float d0 = pow2i(-ex / 2), d1 = pow2i(-ex - (-ex / 2));
#pragma unroll
  for (int i = 0; i < W; ++i) w[i] = pack_f16(__uint_as_float(w[i] << 16) * d0 * d1, __uint_as_float(w[i] & 0xffff0000u) * d0 * d1);
  return pow2i(ex / 2) * pow2i(ex - ex / 2);
}
// Values behind the last key may be anything, NaN included: they become zeros (their weight is zero too).  Rows are cleared
// whole, so the swizzle does not matter; the fence orders this before the next copy into the stage.
template <typename T> __device__ __forceinline__ void clear_rows(uint32_t vb, int key0, int left, int lane) {
  const int row = lane >> 1, half = lane & 1;
  if (row >= left) {
#pragma unroll
    for (int i = 0; i < T::ROW / 32; ++i) {
      const int byte = half * (T::ROW / 2) + 16 * i;
      st_shared_f4(vb + (byte / T::SLAB_ROW) * T::SLAB + (key0 + row) * T::SLAB_ROW + byte % T::SLAB_ROW, 0, 0, 0, 0);
    }
  }
  fence_async_smem();
}
// A row's maximum becomes max(m, top): returns the factor of O.  The weights shrink with it, and E, their exponent, follows,
// so that O keeps its size instead.
template <bool SCALED> __device__ __forceinline__ float follow_max(float& m, float& l, int& E, float top) {
  const float x = fmaxf(top, m), d = m - x;
  const bool fresh = m == -INFINITY;             // nothing summed yet
  m = x;
  float f = fresh ? 0.f : fast_exp2(d);
  l *= f;
  if (SCALED) {
    const int En = fresh ? AP_E_LEAST : max(E + (int)fmaxf(floorf(d), -400.f), AP_E_LEAST);
    f = fresh ? 0.f : fast_exp2(d + (float)(E - En));
    E = En;
  }
  return f;
}
// E becomes the exponent of the largest weight if that is more: returns the factor of O
__device__ __forceinline__ float follow_weight(int& E, float top) {
  const int En = max(E, (int)(__float_as_uint(top) >> 23) - 127);
  const float f = E - En < -126 ? 0.f : pow2i(E - En);
  E = En;
  return f;
}
// four keys of step k (2 t, 2 t + 1, and 8 on) of this warp's quarter of the columns: four consecutive ones (DH = 128), or
// a word with this lane's two in it
template <int DH> __device__ __forceinline__ void load_values(uint32_t vb, int k, int warp, int g, int t, uint32_t* v) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t key = 16 * k + (i >> 1) * 8 + 2 * t + (i & 1);
    if (DH == 128) v[i] = lds32(vb + key * 128 + (((2 * warp + (g >> 2)) ^ (key & 7)) << 4) + (g & 3) * 4);
    else v[i] = lds32(vb + key * 64 + ((warp ^ ((key >> 1) & 3)) << 4) + (g >> 1) * 4);
  }
}

}  // namespace

template <int DH, int KIND, int MT>
__global__ void __launch_bounds__(AP_THREADS, AP_OCC)
attention_paged_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                       const __grid_constant__ CUtensorMap tmKs, const __grid_constant__ CUtensorMap tmVs, const PagedAttnArgs a) {
  using T = Tile<DH, KIND>;
  constexpr bool BF = KIND == SL_BF16;
  constexpr int QK = BF ? SL_E4M3 : KIND;   // a type for the conversions that a bf16 cache does not reach
  constexpr int ROWS = ap_rows<MT>();
  constexpr int TILES = Plan<DH, KIND, MT>::TILES;
  constexpr int STAGES = Plan<DH, KIND, MT>::STAGES;
  constexpr int NT = DH / 32;               // column tiles of O per warp

  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint8_t* sStage = smem;
  uint4* sQ = reinterpret_cast<uint4*>(sStage + STAGES * T::STAGE);                         // [TILES][STEPS][32]
  uint4* sP = sQ + TILES * T::STEPS * 32;                                                   // [terms][TILES][4][32]
  float* sJoin = reinterpret_cast<float*>(sP);                                              // [4][8][DH + 4]: MT = 0
  float* sRow = reinterpret_cast<float*>(reinterpret_cast<uint8_t*>(sP) + Plan<DH, KIND, MT>::EXCHANGE);   // [ROWS] factor of S
  float* sM = sRow + ROWS;                                                                  // [4][ROWS]
  float* sL = sM + 4 * ROWS;                                                                // [4][ROWS]
  uint64_t* bars = reinterpret_cast<uint64_t*>(sL + 4 * ROWS);
  volatile int* s_abort = reinterpret_cast<volatile int*>(bars + 2 * STAGES);
  long long* sCum = reinterpret_cast<long long*>(bars + 2 * STAGES + 1);                    // [B + 1]

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t bar0 = smem_u32(bars);
  auto full = [&](int s) { return bar0 + 8u * s; };
  auto empty = [&](int s) { return bar0 + 8u * (STAGES + s); };
  if (threadIdx.x == 0) {
    for (int i = 0; i < STAGES; ++i) {
      mbar_init(full(i), 1);
      mbar_init(empty(i), 4);
    }
    *s_abort = 0;
    fence_mbar_init();
  }
  griddep_wait();
  griddep_launch();

  // units before each sequence
  for (int b = threadIdx.x; b < a.B; b += AP_THREADS) {
    const Seq s = seq_of<MT>(a, b);
    sCum[b + 1] = (long long)a.Hkv * s.tiles * s.nb;
    if (blockIdx.x == 0 && (a.seq_lens[b] != s.len || a.row_offsets[b] != s.r0 || a.row_offsets[b + 1] != s.r0 + s.rows || s.rows < 0))
      set_status(a.status, SL_DEV_BAD_INDEX);
  }
  if (threadIdx.x == 0) sCum[0] = 0;
  __syncthreads();
  if (warp == 0) {
    long long carry = 0;
    for (int b0 = 0; b0 < a.B; b0 += 32) {
      long long x = b0 + lane < a.B ? sCum[b0 + lane + 1] : 0;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const long long y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
      }
      x += carry;
      if (b0 + lane < a.B) sCum[b0 + lane + 1] = x;
      carry = __shfl_sync(0xffffffffu, x, 31);
    }
  }
  __syncthreads();
  const long long total = sCum[a.B];
  const long long per = (total + gridDim.x - 1) / gridDim.x;
  const long long u0 = per * blockIdx.x, u1 = u0 + per < total ? u0 + per : total;
  if (threadIdx.x == 0) a.desc[blockIdx.x] = make_int4(0, 0, 0, 0);
  if (u0 >= u1) return;
  int b = 0;
  {
    int lo = 0, hi = a.B;   // last b with sCum[b] <= u0
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (sCum[mid] <= u0) lo = mid; else hi = mid;
    }
    b = lo;
  }

  if (warp == 4) {
    // ---- producer ----
    const int box = a.page_size < AP_KEYS ? a.page_size : AP_KEYS, pieces = AP_KEYS / box;
    const uint64_t once = l2_policy_evict_first(), keep = l2_policy_evict_normal();
    unsigned cnt = 0;
    bool ok = true;
    for (long long u = u0; u < u1 && ok;) {
      while (sCum[b + 1] <= u) ++b;
      const Seq s = seq_of<MT>(a, b);
      const long long off = u - sCum[b], item = off / s.nb;
      const int blk0 = (int)(off - item * s.nb), kvh = (int)(item / s.tiles);
      const int nblk = (int)min((long long)(s.nb - blk0), u1 - u);
      const uint64_t policy = s.tiles > 1 ? keep : once;   // several query tiles read the same keys
      const int32_t* pages = a.table + (long long)b * a.max_pages;
      auto page_of = [&](int j) {                          // page of this lane's piece of unit j, or -1 behind the last key
        const int t = j * AP_KEYS + lane * box;
        return lane < pieces && t < s.len ? __ldg(pages + t / a.page_size) : -1;
      };
      int next = page_of(blk0);
      for (int j = blk0; j < blk0 + nblk; ++j, ++cnt) {
        const int st = (int)(cnt % STAGES);
        const uint32_t ph = (cnt / STAGES) & 1;
        const int t = j * AP_KEYS + lane * box;
        const bool have = lane < pieces && t < s.len;
        int page = next;
        if (j + 1 < blk0 + nblk) next = page_of(j + 1);
        if (have && (unsigned)page >= (unsigned)a.n_pages) {
          set_status(a.status, SL_DEV_BAD_INDEX);
          page = a.n_pages;                                // reads as zeros
        }
        if (!(ok = warp_wait(empty(st), ph ^ 1, s_abort))) break;
        const int n = __popc(__ballot_sync(0xffffffffu, have));
        if (lane == 0) mbar_expect_tx(full(st), (uint32_t)(n * box * 2 * (T::ROW + (T::SCALED ? 4 : 0)) + (cnt == 0 && blockIdx.x == (gridDim.x > 1) ? a.lost : 0)));
        __syncwarp();
        if (have) {
          const int x = t % a.page_size;
          const uint32_t base = smem_u32(sStage + st * T::STAGE), at = (uint32_t)(lane * box * T::SLAB_ROW);
#pragma unroll
          for (int sl = 0; sl < T::SLABS; ++sl) {
            tma_load_4d(base + sl * T::SLAB + at, &tmK, sl * (BF ? 64 : 128), x, kvh, page, full(st), policy);
            tma_load_4d(base + T::KV + sl * T::SLAB + at, &tmV, sl * (BF ? 64 : 128), x, kvh, page, full(st), policy);
          }
          if (T::SCALED) {
            const uint32_t sc = base + 2 * T::KV + lane * max(box * 4, 128);   // a copy starts on a 128-byte boundary
            tma_load_3d(sc, &tmKs, x, kvh, page, full(st));
            tma_load_3d(sc + 512, &tmVs, x, kvh, page, full(st));
          }
        }
        __syncwarp();
      }
      u += nblk;
    }
    // The copies in flight still write to this CTA's shared memory: they have landed (a bounded wait) before this warp leaves,
    // whichever warp's wait may have run out.
    const unsigned long long t0 = clock64();
    for (unsigned i = cnt > (unsigned)STAGES ? cnt - STAGES : 0; i < cnt; ++i)
      while (!mbar_try(full((int)(i % STAGES)), (i / STAGES) & 1) && clock64() - t0 < TC_WAIT_CYCLES) {}
    if (!ok && lane == 0) set_status(a.status, SL_DEV_ATTN_TIMEOUT);
    return;
  }

  // ---- consumers ----
  // A wait ran out.  Of an item that started in an earlier CTA, this one's piece becomes NaN, so that the rows do; the rows of the
  // items that start here are not written.
  auto give_up = [&](bool piece) {
    if (threadIdx.x == 0) set_status(a.status, SL_DEV_ATTN_TIMEOUT);
    const float nan = __uint_as_float(0x7fffffffu);
    if (piece && threadIdx.x < ROWS) a.ml[(long long)blockIdx.x * 2 * ROWS + threadIdx.x] = make_float2(nan, nan);
  };
  const int g = lane >> 2, t = lane & 3;
  const uint32_t jkey = warp * 16;                 // this warp's keys in a unit
  unsigned cnt = 0;
  bool ok = true;
  for (long long u = u0; u < u1;) {
    while (sCum[b + 1] <= u) ++b;
    const Seq s = seq_of<MT>(a, b);
    const long long off = u - sCum[b], item = off / s.nb;
    const int blk0 = (int)(off - item * s.nb), kvh = (int)(item / s.tiles), tile = (int)(item % s.tiles);
    const int nblk = (int)min((long long)(s.nb - blk0), u1 - u);
    const int valid = (int)min((long long)ROWS, (long long)s.rows * a.G - (long long)tile * ROWS);

    if constexpr (MT == 0) {
      // ---- at most 8 rows: S^T = K Q^T and O^T = V^T P^T, the rows are the 8 columns of the products ----
      // Q -> B fragments; 16 threads per row, DH / 16 elements each
      {
        constexpr int PER = DH / 16, RUN = (DH == 128 && !BF) ? 32 : 16;
        const int row = threadIdx.x >> 4, part = threadIdx.x & 15, e = tile * ROWS + row;
        uint32_t w[PER / 2];
#pragma unroll
        for (int i = 0; i < PER / 2; ++i) w[i] = 0;
        if (row < valid) {
          const uint2* src = reinterpret_cast<const uint2*>(a.q + (long long)(s.r0 + e / a.G) * a.q_stride +
                                                            (long long)(kvh * a.G + e % a.G) * DH + part * PER);
#pragma unroll
          for (int i = 0; i < PER / 4; ++i) {
            const uint2 x = src[i];
            w[2 * i] = x.x;
            w[2 * i + 1] = x.y;
          }
        }
        const float factor = BF ? a.scale_log2 : a.scale_log2 * rows_to_f16<PER / 2, 16>(w);
        if (part == 0) sRow[row] = factor;
        uint32_t* dst = reinterpret_cast<uint32_t*>(sQ);       // [step][lane][2]
#pragma unroll
        for (int i = 0; i < PER / 2; ++i) {
          const int d = part * PER + 2 * i, block = d / (4 * RUN), in = d % (4 * RUN), tt = in / RUN, rem = in % RUN;
          dst[((block * (RUN / 4) + rem / 4) * 32 + row * 4 + tt) * 2 + ((rem & 3) >> 1)] = w[i];
        }
      }
      bar_consumers();
      constexpr int VT = DH / 16;                              // tiles of 16 columns
      uint2 qb[T::STEPS];
#pragma unroll
      for (int i = 0; i < T::STEPS; ++i) qb[i] = reinterpret_cast<const uint2*>(sQ)[i * 32 + lane];
      const float fr[2] = {sRow[2 * t], sRow[2 * t + 1]};      // of this lane's two rows, and so are m, l, E
      float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f}, acc[VT][4];
      int E[2] = {AP_E_LEAST, AP_E_LEAST};
#pragma unroll
      for (int j = 0; j < VT; ++j) acc[j][0] = acc[j][1] = acc[j][2] = acc[j][3] = 0.f;
      for (int j = blk0; j < blk0 + nblk; ++j, ++cnt) {
        const int st = (int)(cnt % STAGES);
        if (!(ok = warp_wait(full(st), (cnt / STAGES) & 1, s_abort))) break;
        const int left = s.len - j * AP_KEYS - (int)jkey;      // keys from this warp's first one on
        const uint32_t kb = smem_u32(sStage + st * T::STAGE), vb = kb + T::KV;
        if (left > 0 && left < 16) {
          clear_rows<T>(vb, (int)jkey, left, lane);
          __syncwarp();
        }
        float sc[2][4] = {};                                   // two chains; key g + 8 (i >> 1), row 2 t + (i & 1)
        float ks[2] = {0.f, 0.f}, vs[2] = {0.f, 0.f};
        if (left > 0) {
          if (T::SCALED) {
            const float* scp = reinterpret_cast<const float*>(sStage + st * T::STAGE + 2 * T::KV) + (a.page_size == 16 ? 32 : 16) * warp + g;
#pragma unroll
            for (int n = 0; n < 2; ++n) {
              const bool in = 8 * n + g < left;
              ks[n] = in ? scp[8 * n] : 0.f;
              vs[n] = in ? scp[128 + 8 * n] : 0.f;
            }
          }
#pragma unroll
          for (int sl = 0; sl < T::SLABS; ++sl) {
            constexpr int CH = T::SLAB_ROW / 64;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
              uint32_t w[2][4];
#pragma unroll
              for (int n = 0; n < 2; ++n) {
                const uint32_t key = jkey + n * 8 + g, chunk = t * CH + c;
                const uint32_t sw = T::SLAB_ROW == 128 ? (chunk ^ (key & 7)) : (chunk ^ ((key >> 1) & 3));
                const uint4 w4 = lds128(kb + sl * T::SLAB + key * T::SLAB_ROW + (sw << 4));
                w[n][0] = w4.x; w[n][1] = w4.y; w[n][2] = w4.z; w[n][3] = w4.w;
              }
#pragma unroll
              for (int i = 0; i < (BF ? 2 : 4); ++i) {
                const int step = BF ? sl * 4 + c * 2 + i : c * 4 + i;
                uint4 k4;
                if (BF) k4 = make_uint4(w[0][BF ? 2 * i : 0], w[1][BF ? 2 * i : 0], w[0][BF ? 2 * i + 1 : 0], w[1][BF ? 2 * i + 1 : 0]);
                else {
                  codes_to_f16<QK>(w[0][i], k4.x, k4.z);
                  codes_to_f16<QK>(w[1][i], k4.y, k4.w);
                }
                mma16<BF>(sc[i & 1], k4, qb[step].x, qb[step].y);
              }
            }
          }
        }
        if (left > 0) {
          float x[4];
          bool grow = false;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            x[i] = (sc[0][i] + sc[1][i]) * fr[i & 1];
            if (T::SCALED) x[i] *= ks[i >> 1];
            x[i] = 8 * (i >> 1) + g < left ? x[i] : -INFINITY;
            grow |= x[i] > m[i & 1] + AP_TAU;
          }
          auto over_keys = [&](float a0, float a1) {           // the larger of the two, over this warp's 16 keys
            float y = fmaxf(a0, a1);
#pragma unroll
            for (int o = 4; o < 32; o <<= 1) y = fmaxf(y, __shfl_xor_sync(0xffffffffu, y, o));
            return y;
          };
          auto rescale = [&](int i, float f) {
#pragma unroll
            for (int c = 0; c < VT; ++c) {
              acc[c][i] *= f;
              acc[c][i + 2] *= f;
            }
          };
          if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const float top = over_keys(x[i], x[i + 2]);
              rescale(i, follow_max<T::SCALED>(m[i], l[i], E[i], top));
            }
          }
          bool over = false;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float mm = m[i & 1] == -INFINITY ? 0.f : m[i & 1];
            x[i] = fast_exp2(x[i] - mm);
            l[i & 1] += x[i];
            if (T::SCALED) {
              x[i] *= vs[i >> 1];
              over |= fabsf(x[i] * pow2i(AP_W_EXP - E[i & 1])) >= AP_W_MOST;
            }
          }
          if (T::SCALED && __any_sync(0xffffffffu, over)) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const float top = over_keys(fabsf(x[i]), fabsf(x[i + 2]));
              rescale(i, follow_weight(E[i], top));
            }
          }
          // the weights to 16 bits, [key][row] -> [row][key]: the B operand of O^T += V^T P^T
          const float u0 = T::SCALED ? pow2i(AP_W_EXP - E[0]) : 1.f, u1 = T::SCALED ? pow2i(AP_W_EXP - E[1]) : 1.f;
          const uint32_t p0 = transposed(BF ? take_bf16(x[0], x[1]) : pack_f16(x[0] * u0, x[1] * u1));
          const uint32_t p1 = transposed(BF ? take_bf16(x[2], x[3]) : pack_f16(x[2] * u0, x[3] * u1));
          if (BF) {
            const uint32_t r0 = transposed(pack_bf16(x[0], x[1])), r1 = transposed(pack_bf16(x[2], x[3]));
#pragma unroll
            for (int c = 0; c < VT; ++c) {
              uint4 v;
              const uint32_t key = jkey + (lane >> 4) * 8 + (lane & 7), chunk = 2 * c + ((lane >> 3) & 1);
              ldsm_x4_t(vb + (chunk >> 3) * T::SLAB + key * 128 + (((chunk & 7) ^ (key & 7)) << 4), reinterpret_cast<uint32_t*>(&v));
              mma16<BF>(acc[c], v, p0, p1);
              mma16<BF>(acc[c], v, r0, r1);
            }
          } else {
            uint32_t v[4][VT / 2];                             // four keys, DH / 8 consecutive columns
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint32_t key = jkey + (i >> 1) * 8 + 2 * t + (i & 1);
              if (DH == 128) {
                const uint4 y = lds128(vb + key * 128 + ((g ^ (key & 7)) << 4));
                v[i][0] = y.x; v[i][1] = y.y; v[i][VT / 2 - 2] = y.z; v[i][VT / 2 - 1] = y.w;
              } else {
                const uint2 y = lds64(vb + key * 64 + (((g >> 1) ^ ((key >> 1) & 3)) << 4) + (g & 1) * 8);
                v[i][0] = y.x; v[i][1] = y.y;
              }
            }
#pragma unroll
            for (int c = 0; c < VT; ++c) {
              const uint32_t sel = c & 1 ? 0x7362 : 0x5140;    // columns 2, 3 or 0, 1 of a word
              uint4 v4;
              codes_to_f16<QK>(__byte_perm(v[0][c / 2], v[1][c / 2], sel), v4.x, v4.y);
              codes_to_f16<QK>(__byte_perm(v[2][c / 2], v[3][c / 2], sel), v4.z, v4.w);
              mma16<BF>(acc[c], v4, p0, p1);
            }
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(empty(st));
      }

      // the four warps' results become one
#pragma unroll
      for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], o);
        if (g == 0) {
          sM[warp * ROWS + 2 * t + i] = m[i];
          sL[warp * ROWS + 2 * t + i] = l[i];
        }
      }
      if (!epilogue_warps_agree(ok)) {
        give_up(blk0 > 0);
        return;
      }
      const bool starts = blk0 == 0, whole = starts && nblk == s.nb;
      const long long slot = ((long long)blockIdx.x * 2 + (starts ? 1 : 0)) * ROWS;
      if (starts && !whole && threadIdx.x == 0) {
        const long long last = (u + s.nb - 1) / per;           // CTA of the item's last unit
        a.desc[blockIdx.x] = make_int4(s.r0, tile * ROWS, (valid << 16) | kvh, (int)last);
      }
      constexpr int PITCH = DH + 4;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float* p = sM + 2 * t + i;
        const float top = fmaxf(fmaxf(p[0], p[ROWS]), fmaxf(p[2 * ROWS], p[3 * ROWS]));
        const float f = m[i] == -INFINITY ? 0.f : fast_exp2(m[i] - top) * (T::SCALED ? pow2i(E[i] - AP_W_EXP) : 1.f);
        float* dst = sJoin + (warp * 8 + 2 * t + i) * PITCH;
        if (BF) {
#pragma unroll
          for (int c = 0; c < VT; ++c) {
            dst[16 * c + g] = acc[c][i] * f;
            dst[16 * c + 8 + g] = acc[c][2 + i] * f;
          }
        } else {
#pragma unroll
          for (int c = 0; c < VT; c += 2)                      // columns DH / 8 g + 2 c ...
            *reinterpret_cast<float4*>(dst + 2 * VT * g + 2 * c) = make_float4(acc[c][i] * f, acc[c][2 + i] * f, acc[c + 1][i] * f, acc[c + 1][2 + i] * f);
        }
      }
      bar_consumers();
      {
        const int row = threadIdx.x >> 4, part = threadIdx.x & 15;
        if (row < valid) {
          float top = -INFINITY, sum = 0.f;
#pragma unroll
          for (int w = 0; w < 4; ++w) top = fmaxf(top, sM[w * ROWS + row]);
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const float mw = sM[w * ROWS + row];
            sum += sL[w * ROWS + row] * (mw == -INFINITY ? 1.f : fast_exp2(mw - top));   // without keys 0, or NaN from a score that is none
          }
          const int e = tile * ROWS + row;
          const float inv = !whole ? 1.f : s.len == 0 ? 0.f : 1.f / sum;   // a sum of 0 over keys (all scores -inf): 0 / 0
          if (!whole && part == 0) a.ml[slot + row] = make_float2(top, sum);
          bf16* o = a.o + (long long)(s.r0 + e / a.G) * a.o_stride + (long long)(kvh * a.G + e % a.G) * DH;
          float* pt = a.part + (slot + row) * DH;
#pragma unroll
          for (int i = 0; i < DH / 64; ++i) {
            const int col = i * 64 + part * 4;
            float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < 4; ++w) {
              const float4 y = *reinterpret_cast<const float4*>(sJoin + (w * 8 + row) * PITCH + col);
              x.x += y.x; x.y += y.y; x.z += y.z; x.w += y.w;
            }
            if (whole) *reinterpret_cast<uint2*>(o + col) = make_uint2(pack_bf16(x.x * inv, x.y * inv), pack_bf16(x.z * inv, x.w * inv));
            else *reinterpret_cast<float4*>(pt + col) = x;
          }
        }
      }
    } else {
      // query tile -> shared memory in the order of the A fragments; 8 threads per row, DH / 8 elements each
      {
        constexpr int PER = DH / 8, RUN = (DH == 128 && !BF) ? 32 : 16;
        const int row = threadIdx.x >> 3, part = threadIdx.x & 7;
        uint4 wq[MT][PER / 8];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          const int e = tile * ROWS + mt * 16 + row;
#pragma unroll
          for (int i = 0; i < PER / 8; ++i) wq[mt][i] = make_uint4(0, 0, 0, 0);
          if (mt * 16 + row < valid) {
            const uint4* src = reinterpret_cast<const uint4*>(a.q + (long long)(s.r0 + e / a.G) * a.q_stride +
                                                              (long long)(kvh * a.G + e % a.G) * DH + part * PER);
#pragma unroll
            for (int i = 0; i < PER / 8; ++i) wq[mt][i] = src[i];
          }
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          uint32_t* pw = reinterpret_cast<uint32_t*>(wq[mt]);
          const float factor = BF ? a.scale_log2 : a.scale_log2 * rows_to_f16<PER / 2, 8>(pw);
          if (part == 0) sRow[mt * 16 + row] = factor;
          uint32_t* dst = reinterpret_cast<uint32_t*>(sQ + mt * T::STEPS * 32);
#pragma unroll
          for (int i = 0; i < PER / 2; ++i) {
            const int d = part * PER + 2 * i, block = d / (4 * RUN), in = d % (4 * RUN), tt = in / RUN, rem = in % RUN;
            const int step = block * (RUN / 4) + rem / 4, pair = (rem & 3) >> 1;
            dst[((step * 32 + (row & 7) * 4 + tt) << 2) + (row >> 3) + 2 * pair] = pw[i];
          }
        }
      }
      bar_consumers();
      float fr[MT][2], m[MT][2], l[MT][2], acc[MT][NT][4];
      int E[MT][2];                                // exponent of the largest weight so far, in units of the present maximum
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          fr[mt][h] = sRow[mt * 16 + g + 8 * h];
          m[mt][h] = -INFINITY;                    // the same in all four warps, and so is E; l is of this warp's keys
          l[mt][h] = 0.f;
          E[mt][h] = AP_E_LEAST;
        }
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[mt][j][0] = acc[mt][j][1] = acc[mt][j][2] = acc[mt][j][3] = 0.f;
      }

      for (int j = blk0; j < blk0 + nblk; ++j, ++cnt) {
        const int st = (int)(cnt % STAGES);
        if (ok) ok = warp_wait(full(st), (cnt / STAGES) & 1, s_abort);
        const int here = min(s.len - j * AP_KEYS, AP_KEYS);    // keys of the unit
        const int left = here - (int)jkey;                     // of this warp: 16 or more, fewer, none
        const uint32_t kb = smem_u32(sStage + st * T::STAGE), vb = kb + T::KV;
        const float* scp = reinterpret_cast<const float*>(sStage + st * T::STAGE + 2 * T::KV) + (a.page_size == 16 ? 32 : 16) * warp + 2 * t;
        if (left > 0 && left < 16) clear_rows<T>(vb, (int)jkey, left, lane);
        float ks[2][2], vs[2][2];
        float sc[MT][2][4];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int i = 0; i < 8; ++i) sc[mt][i >> 2][i & 3] = 0.f;
        if (left > 0) {
          if (T::SCALED) {
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
              for (int c = 0; c < 2; ++c) {
                const bool in = 8 * n + 2 * t + c < left;
                ks[n][c] = in ? scp[8 * n + c] : 0.f;
                vs[n][c] = in ? scp[128 + 8 * n + c] : 0.f;
              }
          }
          // S = Q K^T: two tiles of 8 keys
#pragma unroll
          for (int sl = 0; sl < T::SLABS; ++sl) {
            constexpr int CH = T::SLAB_ROW / 64;              // 16-byte chunks of the row that belong to a lane: 1 or 2
#pragma unroll
            for (int c = 0; c < CH; ++c) {
              uint32_t w[2][4];
#pragma unroll
              for (int n = 0; n < 2; ++n) {
                const uint32_t key = jkey + n * 8 + g, chunk = t * CH + c;
                const uint32_t sw = T::SLAB_ROW == 128 ? (chunk ^ (key & 7)) : (chunk ^ ((key >> 1) & 3));
                const uint4 w4 = lds128(kb + sl * T::SLAB + key * T::SLAB_ROW + (sw << 4));
                w[n][0] = w4.x; w[n][1] = w4.y; w[n][2] = w4.z; w[n][3] = w4.w;
              }
#pragma unroll
              for (int i = 0; i < (BF ? 2 : 4); ++i) {
                const int step = BF ? sl * 4 + c * 2 + i : c * 4 + i;
                uint4 q4[MT];
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) q4[mt] = sQ[(mt * T::STEPS + step) * 32 + lane];
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                  uint32_t b0, b1;
                  if (BF) {
                    b0 = w[n][BF ? 2 * i : 0];
                    b1 = w[n][BF ? 2 * i + 1 : 0];
                  } else {
                    codes_to_f16<QK>(w[n][i], b0, b1);
                  }
#pragma unroll
                  for (int mt = 0; mt < MT; ++mt) mma16<BF>(sc[mt][n], q4[mt], b0, b1);
                }
              }
            }
          }
        }
        // scores in log2 units; keys behind the last one take no part
        bool grow = !ok;
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const bool in = 8 * n + 2 * t + c < left;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                float x = sc[mt][n][2 * h + c] * fr[mt][h];
                if (T::SCALED && left > 0) x *= ks[n][c];
                x = in ? x : -INFINITY;
                sc[mt][n][2 * h + c] = x;
                grow |= x > m[mt][h] + AP_TAU;
              }
          }
        auto rescale = [&](int mt, int h, float f) {
#pragma unroll
          for (int i = 0; i < NT; ++i) {
            acc[mt][i][2 * h] *= f;
            acc[mt][i][2 * h + 1] *= f;
          }
        };
        // largest score (or weight's magnitude) of every row over the four warps' keys
        auto row_tops = [&](bool mag, float (*top)[2]) {
#pragma unroll
          for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              float x = mag ? 0.f : -INFINITY;
#pragma unroll
              for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int c = 0; c < 2; ++c) x = fmaxf(x, mag ? fabsf(sc[mt][n][2 * h + c]) : sc[mt][n][2 * h + c]);
              x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
              x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));
              if (t == 0) sM[warp * ROWS + mt * 16 + g + 8 * h] = x;
            }
          bar_consumers();
#pragma unroll
          for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const float* p = sM + mt * 16 + g + 8 * h;
              top[mt][h] = fmaxf(fmaxf(p[0], p[ROWS]), fmaxf(p[2 * ROWS], p[3 * ROWS]));
            }
        };
        if (consumers_any(grow)) {
          if (!epilogue_warps_agree(ok)) {                     // a wait ran out: all four warps leave together
            ok = false;
            break;
          }
          float top[MT][2];
          row_tops(false, top);
#pragma unroll
          for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int h = 0; h < 2; ++h)
              rescale(mt, h, follow_max<T::SCALED>(m[mt][h], l[mt][h], E[mt][h], top[mt][h]));
        }
        // P: exp2, times the value scales
        bool over = false;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const float mm = m[mt][h] == -INFINITY ? 0.f : m[mt][h];
            const float up = T::SCALED ? pow2i(AP_W_EXP - E[mt][h]) : 1.f;
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
              for (int c = 0; c < 2; ++c) {
                float& x = sc[mt][n][2 * h + c];
                x = fast_exp2(x - mm);
                l[mt][h] += x;
                if (T::SCALED && left > 0) {
                  x *= vs[n][c];
                  over |= fabsf(x * up) >= AP_W_MOST;
                }
              }
          }
        // to 16 bits; a warp's weights are the A operand of its 16 keys' step as they stand
        auto put_weights = [&]() {
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) {
            uint32_t pr[4], rest[4];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const float up = T::SCALED ? pow2i(AP_W_EXP - E[mt][h]) : 1.f;
#pragma unroll
              for (int n = 0; n < 2; ++n) {
                float &x = sc[mt][n][2 * h], &y = sc[mt][n][2 * h + 1];
                pr[2 * n + h] = BF ? take_bf16(x, y) : pack_f16(x * up, y * up);
                if (BF) rest[2 * n + h] = pack_bf16(x, y);
              }
            }
            sP[(mt * 4 + warp) * 32 + lane] = make_uint4(pr[0], pr[1], pr[2], pr[3]);
            if (BF) sP[((MT + mt) * 4 + warp) * 32 + lane] = make_uint4(rest[0], rest[1], rest[2], rest[3]);
          }
        };
        put_weights();
        if (consumers_any(T::SCALED && over)) {
          float top[MT][2];
          row_tops(true, top);
#pragma unroll
          for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int h = 0; h < 2; ++h)
              rescale(mt, h, follow_weight(E[mt][h], top[mt][h]));
          put_weights();
          bar_consumers();
        }
        // O += P V: this warp's columns, 16 keys at a time
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          if (16 * k >= here) break;
          uint4 pa[MT];
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) pa[mt] = sP[(mt * 4 + k) * 32 + lane];
          if (BF) {
            uint4 pb[MT];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) pb[mt] = sP[((MT + mt) * 4 + k) * 32 + lane];
#pragma unroll
            for (int c = 0; c < NT; c += 2) {
              uint32_t v[4];
              const uint32_t key = 16 * k + (lane & 15), chunk = warp * NT + c + (lane >> 4);
              ldsm_x4_t(vb + (chunk >> 3) * T::SLAB + key * 128 + (((chunk & 7) ^ (key & 7)) << 4), v);
#pragma unroll
              for (int mt = 0; mt < MT; ++mt) {
                mma16<BF>(acc[mt][c], pa[mt], v[0], v[1]);
                mma16<BF>(acc[mt][c + 1], pa[mt], v[2], v[3]);
                mma16<BF>(acc[mt][c], pb[mt], v[0], v[1]);
                mma16<BF>(acc[mt][c + 1], pb[mt], v[2], v[3]);
              }
            }
          } else {
            uint32_t v[4];
            load_values<DH>(vb, k, warp, g, t, v);
#pragma unroll
            for (int hh = 0; hh < NT / 2; ++hh) {
              // columns 0,1 or 2,3 of the four; with 64 columns in all a lane has two of them
              const uint32_t sel = (DH == 128 ? hh == 1 : (g & 1) == 1) ? 0x7362 : 0x5140;
              uint32_t lo0, hi0, lo1, hi1;
              codes_to_f16<QK>(__byte_perm(v[0], v[1], sel), lo0, hi0);
              codes_to_f16<QK>(__byte_perm(v[2], v[3], sel), lo1, hi1);
#pragma unroll
              for (int mt = 0; mt < MT; ++mt) {
                mma16<BF>(acc[mt][2 * hh], pa[mt], lo0, lo1);
                mma16<BF>(acc[mt][2 * hh + 1], pa[mt], hi0, hi1);
              }
            }
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(empty(st));
      }

      // sums of the four warps' keys
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float x = l[mt][h];
          x += __shfl_xor_sync(0xffffffffu, x, 1);
          x += __shfl_xor_sync(0xffffffffu, x, 2);
          if (t == 0) sL[warp * ROWS + mt * 16 + g + 8 * h] = x;
        }
      if (!epilogue_warps_agree(ok)) {
        give_up(blk0 > 0);
        return;
      }
      const bool starts = blk0 == 0, whole = starts && nblk == s.nb;
      const long long slot = ((long long)blockIdx.x * 2 + (starts ? 1 : 0)) * ROWS;
      if (starts && !whole && threadIdx.x == 0) {
        const long long last = (u + s.nb - 1) / per;           // CTA of the item's last unit
        a.desc[blockIdx.x] = make_int4(s.r0, tile * ROWS, (valid << 16) | kvh, (int)last);
      }
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int row = mt * 16 + g + 8 * h;
          if (row >= valid) continue;
          const float* p = sL + row;
          const float sum = (p[0] + p[ROWS]) + (p[2 * ROWS] + p[3 * ROWS]);
          const int e = tile * ROWS + row;
          const float f = (T::SCALED ? pow2i(E[mt][h] - AP_W_EXP) : 1.f) * (whole ? (s.len == 0 ? 0.f : 1.f / sum) : 1.f);
          bf16* o = a.o + (long long)(s.r0 + e / a.G) * a.o_stride + (long long)(kvh * a.G + e % a.G) * DH + warp * (DH / 4);
          float* part = a.part + (slot + row) * DH + warp * (DH / 4);
          if (!whole && warp == 0 && t == 0) a.ml[slot + row] = make_float2(m[mt][h], sum);
          if (BF) {
#pragma unroll
            for (int i = 0; i < NT; ++i) {
              const float x = acc[mt][i][2 * h] * f, y = acc[mt][i][2 * h + 1] * f;
              if (whole) *reinterpret_cast<uint32_t*>(o + 8 * i + 2 * t) = pack_bf16(x, y);
              else *reinterpret_cast<float2*>(part + 8 * i + 2 * t) = make_float2(x, y);
            }
          } else {
            float x[2 * NT];                                   // consecutive columns 2 NT t ...
#pragma unroll
            for (int i = 0; i < NT; ++i) {
              x[i] = acc[mt][i][2 * h] * f;
              x[NT + i] = acc[mt][i][2 * h + 1] * f;
            }
#pragma unroll
            for (int i = 0; i < 2 * NT; i += 4) {
              if (whole) *reinterpret_cast<uint2*>(o + 2 * NT * t + i) = make_uint2(pack_bf16(x[i], x[i + 1]), pack_bf16(x[i + 2], x[i + 3]));
              else *reinterpret_cast<float4*>(part + 2 * NT * t + i) = make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
            }
          }
        }
    }
    u += nblk;
  }
}

// The pieces of an item that run borders cut: o = sum_i w_i O_i / sum_i w_i l_i, w_i = 2^(m_i - max m), in unit order.  CTA
// (c, y) has the item that starts in run c.
//
// Few pieces (at most 16; at most 32 would fit the lanes): a warp per row, 32 rows at once over the grid's 4 y; lane i has the statistics of piece i, and the
// pieces' values are requested together with them.  (An item that was cut has keys: a sum of 0 means that all scores are -inf, and
// gives NaN.)
// (int8, 16 rows, 8 heads, a warp per row against the way below: 8 pieces 8.2 and 12.5 us in all, 16 pieces 9.2 and 13.1; 32 pieces
// 11.5 and 15.0 with 16 rows, but 9.6 and 9.2 with one.)
template <int DH, int ROWS> __device__ __forceinline__ void join_few(const PagedAttnArgs& a, const int4& d, int n) {
  constexpr int PER = DH / 32, LOADS = 8;
  const int valid = d.z >> 16, kvh = d.z & 0xffff, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int row = blockIdx.y * 8 + warp; row < valid; row += 32) {
    auto slot = [&](int i) { return (long long)((blockIdx.x + i) * 2 + (i == 0 ? 1 : 0)) * ROWS + row; };
    const float2 ml = lane < n ? a.ml[slot(lane)] : make_float2(-INFINITY, 0.f);
    float w = 0.f, sum = 0.f, x[PER] = {};
    for (int i0 = 0; i0 < n; i0 += LOADS) {
      float2 p[LOADS][PER / 2];
#pragma unroll
      for (int u = 0; u < LOADS; ++u)
#pragma unroll
        for (int c = 0; c < PER / 2; ++c)
          p[u][c] = i0 + u < n ? reinterpret_cast<const float2*>(a.part + slot(i0 + u) * DH + lane * PER)[c] : make_float2(0.f, 0.f);
      if (i0 == 0) {
        float top = ml.x;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        w = ml.x == -INFINITY ? 0.f : fast_exp2(ml.x - top);
        sum = ml.x == -INFINITY ? ml.y : w * ml.y;           // a piece without a maximum has the sum 0, or NaN
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      }
#pragma unroll
      for (int u = 0; u < LOADS; ++u) {
        const float wi = __shfl_sync(0xffffffffu, w, i0 + u);
#pragma unroll
        for (int c = 0; c < PER / 2; ++c) {
          x[2 * c] += wi * p[u][c].x;
          x[2 * c + 1] += wi * p[u][c].y;
        }
      }
    }
    const int e = d.y + row;
    const float inv = 1.f / sum;
    bf16* o = a.o + (long long)(d.x + e / a.G) * a.o_stride + (long long)(kvh * a.G + e % a.G) * DH + lane * PER;
#pragma unroll
    for (int c = 0; c < PER; c += 2) *reinterpret_cast<uint32_t*>(o + c) = pack_bf16(x[c] * inv, x[c + 1] * inv);
  }
}
// Many: the CTA's 8 warps take every eighth piece of a row each.
template <int DH, int ROWS> __device__ __forceinline__ void join_many(const PagedAttnArgs& a, const int4& d, int n, float (*sO)[DH], float* sSum) {
  constexpr int PER = DH / 32, LOADS = 4;
  const int valid = d.z >> 16, kvh = d.z & 0xffff, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int row = blockIdx.y; row < valid; row += 4) {
    auto slot = [&](int i) { return (long long)((blockIdx.x + i) * 2 + (i == 0 ? 1 : 0)) * ROWS + row; };
    float sum = 0.f, x[PER] = {}, top = -INFINITY;
    for (int i = lane; i < n; i += 32) top = fmaxf(top, a.ml[slot(i)].x);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    for (int i0 = warp; i0 < n; i0 += 8 * LOADS) {
      float2 ml[LOADS], p[LOADS][PER / 2];
#pragma unroll
      for (int u = 0; u < LOADS; ++u) {
        const int i = i0 + 8 * u;
        ml[u] = i < n ? a.ml[slot(i)] : make_float2(-INFINITY, 0.f);
#pragma unroll
        for (int c = 0; c < PER / 2; ++c)
          p[u][c] = i < n ? reinterpret_cast<const float2*>(a.part + slot(i) * DH + lane * PER)[c] : make_float2(0.f, 0.f);
      }
#pragma unroll
      for (int u = 0; u < LOADS; ++u) {
        const float w = ml[u].x == -INFINITY ? 0.f : fast_exp2(ml[u].x - top);
        sum += ml[u].x == -INFINITY ? ml[u].y : w * ml[u].y;
#pragma unroll
        for (int c = 0; c < PER / 2; ++c) {
          x[2 * c] += w * p[u][c].x;
          x[2 * c + 1] += w * p[u][c].y;
        }
      }
    }
#pragma unroll
    for (int c = 0; c < PER; ++c) sO[warp][lane * PER + c] = x[c];
    if (lane == 0) sSum[warp] = sum;
    __syncthreads();
    if (threadIdx.x < DH) {
      float y = 0.f, l = 0.f;
#pragma unroll
      for (int w = 0; w < 8; ++w) {
        y += sO[w][threadIdx.x];
        l += sSum[w];
      }
      const int e = d.y + row;
      a.o[(long long)(d.x + e / a.G) * a.o_stride + (long long)(kvh * a.G + e % a.G) * DH + threadIdx.x] =
          __float2bfloat16_rn(y / l);
    }
    __syncthreads();
  }
}
template <int DH, int ROWS>
__global__ void __launch_bounds__(256) attention_paged_join_kernel(const PagedAttnArgs a) {
  __shared__ float sO[8][DH];
  __shared__ float sSum[8];
  griddep_wait();
  griddep_launch();
  const int4 d = a.desc[blockIdx.x];
  const int n = d.w - (int)blockIdx.x + 1;
  if (d.z >> 16 == 0) return;
  if (n <= 16) join_few<DH, ROWS>(a, d, n);
  else join_many<DH, ROWS>(a, d, n, sO, sSum);
}

namespace {

constexpr int AP_SLOT_ROWS = AP_OCC * 32;   // most of (CTAs per SM) x (rows of a tile)

// pool [n_pages][Hkv][page_size][head_dim] (or its scales, without the last dimension) in boxes of at most 64 places
int page_map(CUtensorMap* out, const surelock_paged_kv& c, void* base, bool scales) {
  TensorMapEncodeFn fn = tensor_map_encode_fn();
  if (!fn) return SL_ECUDA;
  const int bytes = scales ? 4 : c.dtype == SL_BF16 ? 2 : 1, row = c.head_dim * (c.dtype == SL_BF16 ? 2 : 1);
  const cuuint32_t box_keys = c.page_size < AP_KEYS ? c.page_size : AP_KEYS;
  cuuint64_t dims[4], strides[3];
  cuuint32_t box[4], one[4] = {1, 1, 1, 1};
  int n = 0;
  cuuint64_t pitch = bytes;
  auto add = [&](cuuint64_t dim, cuuint32_t b) {
    if (n) strides[n - 1] = pitch;
    dims[n] = dim;
    box[n++] = b;
    pitch *= dim;
  };
  if (!scales) add(c.head_dim, row < 128 ? c.head_dim : 128 / bytes);
  add(c.page_size, box_keys);
  add(c.n_kv_heads, 1);
  add(c.n_pages, 1);
  const CUtensorMapDataType type = scales ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                   : c.dtype == SL_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_UINT8;
  const CUtensorMapSwizzle swizzle = scales ? CU_TENSOR_MAP_SWIZZLE_NONE : row < 128 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B;
  const CUresult r = fn(out, type, n, base, dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
                        CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? SL_OK : SL_ECUDA;
}

template <int DH, int KIND, int MT>
int launch_ap(const CUtensorMap* maps, PagedAttnArgs a, long long max_units, void* workspace, cudaStream_t st) {
  using PL = Plan<DH, KIND, MT>;
  const int smem = PL::SMEM + (a.B + 1) * 8;
  static std::atomic<uint64_t> allowed{0};
  SL_CUDA_TRY(allow_smem(attention_paged_kernel<DH, KIND, MT>, PL::SMEM + (AP_MAX_B + 1) * 8, allowed));
  const int fit = 228 * 1024 / (smem + 1024);   // all CTAs of the grid are resident at once, so equal runs end together
  const int occ = fit < AP_OCC ? fit : AP_OCC;
  const int cap = sm_count() * occ, grid = (int)(max_units < cap ? max_units : cap);
  const size_t rows = (size_t)sm_count() * AP_SLOT_ROWS * 2;
  a.part = reinterpret_cast<float*>(workspace);
  a.ml = reinterpret_cast<float2*>(a.part + rows * DH);
  a.desc = reinterpret_cast<int4*>(a.ml + rows);
  SL_CUDA_TRY(launch_pdl(attention_paged_kernel<DH, KIND, MT>, dim3(grid), dim3(AP_THREADS), (size_t)smem, st, maps[0], maps[1], maps[2],
                         maps[3], a));
  if (grid > 1 && a.max_tokens > AP_KEYS)   // otherwise no item has two units
    SL_CUDA_TRY(launch_pdl(attention_paged_join_kernel<DH, ap_rows<MT>()>, dim3(grid - 1, 4), dim3(256), 0, st, a));
  return SL_OK;
}

}  // namespace

size_t attention_paged_workspace_bytes(int head_dim) {
  if (head_dim != 64 && head_dim != 128) return 0;
  return (size_t)sm_count() * (AP_SLOT_ROWS * 2 * (head_dim * sizeof(float) + sizeof(float2)) + 4 * sizeof(int4));
}

int launch_attention_paged(const surelock_paged_kv& c, const void* q, long long q_stride, const int32_t* row_offsets,
                           const int32_t* seq_lens, int max_rows, int B, int H, void* o, long long o_stride, void* workspace,
                           int32_t* status, cudaStream_t st) {
  if (B > AP_MAX_B || c.n_kv_heads > 0xffff) return SL_EUNSUPPORTED;
  if ((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(o) | reinterpret_cast<uintptr_t>(workspace)) & 15) return SL_EUNSUPPORTED;
  if ((q_stride | o_stride) & 7) return SL_EUNSUPPORTED;
  CUtensorMap maps[4];
  int rc = page_map(&maps[0], c, c.k, false);
  if (rc == SL_OK) rc = page_map(&maps[1], c, c.v, false);
  if (rc == SL_OK && c.dtype != SL_BF16) rc = page_map(&maps[2], c, c.k_scale, true);
  if (rc == SL_OK && c.dtype != SL_BF16) rc = page_map(&maps[3], c, c.v_scale, true);
  if (rc != SL_OK) return rc;
  if (c.dtype == SL_BF16) maps[2] = maps[3] = maps[0];   // not read
  PagedAttnArgs a{};
  a.row_offsets = row_offsets;
  a.seq_lens = seq_lens;
  a.table = c.page_table;
  a.q = (const bf16*)q;
  a.o = (bf16*)o;
  a.q_stride = q_stride;
  a.o_stride = o_stride;
  a.B = B;
  a.Hkv = c.n_kv_heads;
  a.G = H / c.n_kv_heads;
  a.max_rows = max_rows;
  a.n_pages = c.n_pages;
  a.page_size = c.page_size;
  a.max_pages = c.max_pages;
  a.max_tokens = c.max_pages * c.page_size;
  a.scale_log2 = 1.4426950408889634f / sqrtf((float)c.head_dim);
  a.status = status;
  a.lost = take_lost_copy();
  // Rows of a tile: what a sequence has on average, padded as little as possible, up to 32.  Tiles of 64 share the conversions
  // of the codes among more rows, but leave fewer CTAs per SM: 4 x 8192 tokens, 64 rows each: 198 against 178 us; 1536 tokens,
  // 128 rows: 37 against 31 us; tiles of 16 there: 222 and 33 us.  But where tiles of 32 leave SMs without work, tiles of 16 give
  // more of it a start at once (512 tokens, 23 rows, 32 heads: 11.7 against 10.4 us).
  const long long rows = ((long long)max_rows * a.G + B - 1) / B, per_tile = (long long)a.Hkv * ((a.max_tokens + AP_KEYS - 1) / AP_KEYS);
  const bool little = B * ((rows + 31) / 32) * per_tile < (long long)sm_count() * AP_OCC;
  const int mt = rows <= 8 ? 0 : rows <= 16 || little ? 1 : 2, tile_rows = mt ? 16 * mt : 8;
  const long long max_units = (((long long)max_rows * a.G + tile_rows - 1) / tile_rows + B) * per_tile;
#define SL_AP(DH, KIND)                                                                                        \
  (mt == 0   ? launch_ap<DH, KIND, 0>(maps, a, max_units, workspace, st)                                       \
   : mt == 1 ? launch_ap<DH, KIND, 1>(maps, a, max_units, workspace, st)                                       \
             : launch_ap<DH, KIND, 2>(maps, a, max_units, workspace, st))
  if (c.head_dim == 128) return c.dtype == SL_BF16 ? SL_AP(128, SL_BF16) : c.dtype == SL_E4M3 ? SL_AP(128, SL_E4M3) : SL_AP(128, SL_INT8);
  return c.dtype == SL_BF16 ? SL_AP(64, SL_BF16) : c.dtype == SL_E4M3 ? SL_AP(64, SL_E4M3) : SL_AP(64, SL_INT8);
#undef SL_AP
}

}  // namespace sl
