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
//   warps 0-3  16 keys of the unit each, with their own running maximum and sum: S = Q K^T by mma.sync m16n8k16 (the tile
//              has 16 rows, an eighth of a tcgen05 tile; the codes become fp16, exactly, in registers on the way), exp2, O += P V.
// The contraction index is permuted (the same way for Q and K) so that a lane reads its share of a key as 16-byte loads, and
// the columns of O so that it reads 16 bytes of a value row; two keys' bytes are interleaved by byte permutes.
// Numerics: q becomes fp16 times a power of two per row (its largest magnitude in [1, 2)), the weight w_j = p_j sv_j becomes
// fp16 under a power of two per row that follows the row's largest weight so far; both keep 11 bits, and weights below
// 2^-33 of the largest vanish.  S, the statistics and O are fp32.  O is rescaled when a maximum grows by more than 2^6 or a
// weight outgrows its power of two.  With a bf16 cache q and p are bf16.
#include <mutex>

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
__device__ __forceinline__ uint2 lds64(uint32_t a) {
  uint2 r;
  asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(r.x), "=r"(r.y) : "r"(a) : "memory");
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
__device__ __forceinline__ float pow2i(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }   // -126 <= e <= 127

// one sequence's share of the units
struct Seq {
  int r0, rows, len, tiles, nb;   // first packed row, rows, keys, query tiles, units per (key head, tile)
};
template <int MT> __device__ __forceinline__ Seq seq_of(const PagedAttnArgs& a, int b) {
  Seq s;
  s.r0 = max(0, a.row_offsets[b]);
  s.rows = min(a.row_offsets[b + 1], a.max_rows) - s.r0;
  const int len = a.seq_lens[b];
  s.len = min(max(len, 0), a.max_tokens);
  s.tiles = s.rows > 0 ? (int)(((long long)s.rows * a.G + 16 * MT - 1) / (16 * MT)) : 0;
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
  static constexpr int STAGES = STAGE > 20000 ? 2 : STAGE > 17000 ? 3 : STAGE > 10000 ? 4 : 6;   // two CTAs per SM
  static constexpr int STEPS = DH / 16;
  static constexpr int PITCH = DH + 4 * (DH / 32);              // floats per row of the join buffer
  static constexpr int JOIN = 4 * 16 * PITCH * 4;
};
template <int DH, int KIND, int MT> constexpr int ap_smem() {
  using T = Tile<DH, KIND>;
  return 1024 + T::STAGES * T::STAGE + T::JOIN + MT * T::STEPS * 512 + 16 * MT * 4 + 2 * 4 * 16 * MT * 4 + 256;   // and 8 bytes per sequence
}

}  // namespace

template <int DH, int KIND, int MT>
__global__ void __launch_bounds__(AP_THREADS, 2)
attention_paged_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                       const __grid_constant__ CUtensorMap tmKs, const __grid_constant__ CUtensorMap tmVs, const PagedAttnArgs a) {
  using T = Tile<DH, KIND>;
  constexpr bool BF = KIND == SL_BF16;
  constexpr int QK = BF ? SL_E4M3 : KIND;   // a type for the conversions that a bf16 cache does not reach
  constexpr int ROWS = 16 * MT;
  constexpr int NT = DH / 8;                // column tiles of O

  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint8_t* sStage = smem;
  float* sJoin = reinterpret_cast<float*>(sStage + T::STAGES * T::STAGE);
  uint4* sQ = reinterpret_cast<uint4*>(reinterpret_cast<uint8_t*>(sJoin) + T::JOIN);       // [MT][STEPS][32]
  float* sRow = reinterpret_cast<float*>(sQ + MT * T::STEPS * 32);                          // [ROWS] factor of S
  float* sM = sRow + ROWS;                                                                  // [4][ROWS]
  float* sL = sM + 4 * ROWS;                                                                // [4][ROWS]
  uint64_t* bars = reinterpret_cast<uint64_t*>(sL + 4 * ROWS);
  volatile int* s_abort = reinterpret_cast<volatile int*>(bars + 2 * T::STAGES);
  long long* sCum = reinterpret_cast<long long*>(bars + 2 * T::STAGES + 1);                 // [B + 1]

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t bar0 = smem_u32(bars);
  auto full = [&](int s) { return bar0 + 8u * s; };
  auto empty = [&](int s) { return bar0 + 8u * (T::STAGES + s); };
  if (threadIdx.x == 0) {
    for (int i = 0; i < T::STAGES; ++i) {
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
    if (blockIdx.x == 0 && (a.seq_lens[b] != s.len || a.row_offsets[b] != s.r0 || s.rows < 0 || a.row_offsets[b + 1] > a.max_rows))
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
        const int st = (int)(cnt % T::STAGES);
        const uint32_t ph = (cnt / T::STAGES) & 1;
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
        if (lane == 0) mbar_expect_tx(full(st), (uint32_t)(n * box * 2 * (T::ROW + (T::SCALED ? 4 : 0))));
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
    if (!ok) {
      // gave up: the copies in flight still write to this CTA's shared memory, wait for them (bounded)
      const unsigned long long t0 = clock64();
      for (unsigned i = cnt > (unsigned)T::STAGES ? cnt - T::STAGES : 0; i < cnt; ++i)
        while (!mbar_try(full((int)(i % T::STAGES)), (i / T::STAGES) & 1) && clock64() - t0 < TC_WAIT_CYCLES) {}
      if (lane == 0) set_status(a.status, SL_DEV_ATTN_TIMEOUT);
    }
    return;
  }

  // ---- consumers ----
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

    // query tile -> shared memory in the order of the A fragments; 8 threads per row, DH / 8 elements each
    {
      constexpr int PER = DH / 8, RUN = (DH == 128 && !BF) ? 32 : 16;
      for (int mt = 0; mt < MT; ++mt) {
        const int row = threadIdx.x >> 3, part = threadIdx.x & 7, e = tile * ROWS + mt * 16 + row;
        uint4 w[PER / 8];
#pragma unroll
        for (int i = 0; i < PER / 8; ++i) w[i] = make_uint4(0, 0, 0, 0);
        if (mt * 16 + row < valid) {
          const uint4* src = reinterpret_cast<const uint4*>(a.q + (long long)(s.r0 + e / a.G) * a.q_stride +
                                                            (long long)(kvh * a.G + e % a.G) * DH + part * PER);
#pragma unroll
          for (int i = 0; i < PER / 8; ++i) w[i] = src[i];
        }
        uint32_t* pw = reinterpret_cast<uint32_t*>(w);
        float factor = a.scale_log2;
        if (!BF) {
          uint32_t top = 0;
#pragma unroll
          for (int i = 0; i < PER / 2; ++i) top = max(top, max(pw[i] & 0x7fffu, (pw[i] >> 16) & 0x7fffu));
#pragma unroll
          for (int o = 4; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
          int ex = (int)(top >> 7) - 127;                               // exponent of the row's largest magnitude
          ex = top == 0 || ex > 127 ? 0 : max(ex, -126);
          // times 2^-ex in two steps, since 2^-ex and 2^ex need not both be normal numbers
          const float d0 = pow2i(-ex / 2), d1 = pow2i(-ex - (-ex / 2));
#pragma unroll
          for (int i = 0; i < PER / 2; ++i)
            pw[i] = pack_f16(__uint_as_float(pw[i] << 16) * d0 * d1, __uint_as_float(pw[i] & 0xffff0000u) * d0 * d1);
          factor = factor * pow2i(ex / 2) * pow2i(ex - ex / 2);
        }
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
    float fr[MT][2];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      fr[mt][0] = sRow[mt * 16 + g];
      fr[mt][1] = sRow[mt * 16 + g + 8];
    }
    uint4 qa[MT == 1 ? T::STEPS : 1];
    if (MT == 1) {
#pragma unroll
      for (int i = 0; i < T::STEPS; ++i) qa[MT == 1 ? i : 0] = sQ[i * 32 + lane];
    }

    float acc[MT][NT][4];
    float m[MT][2], l[MT][2];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      m[mt][0] = m[mt][1] = -INFINITY;
      l[mt][0] = l[mt][1] = 0.f;
#pragma unroll
      for (int j = 0; j < NT; ++j) acc[mt][j][0] = acc[mt][j][1] = acc[mt][j][2] = acc[mt][j][3] = 0.f;
    }
    int E[MT][2];                                // exponent of the largest weight so far, in units of the present maximum
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) E[mt][0] = E[mt][1] = AP_E_LEAST;

    for (int j = blk0; j < blk0 + nblk && ok; ++j, ++cnt) {
      const int st = (int)(cnt % T::STAGES);
      if (!(ok = warp_wait(full(st), (cnt / T::STAGES) & 1, s_abort))) break;
      const int left = s.len - j * AP_KEYS - (int)jkey;      // keys from this warp's first one on
      if (left > 0) {
        uint8_t* stage = sStage + st * T::STAGE;
        const uint32_t sk_base = smem_u32(stage), sv_base = sk_base + T::KV;
        const bool tail = left < 16;
        if (tail) {
          // values behind the last key may be anything, NaN included: they become zeros (their weight is zero too)
          const int row = lane >> 1, half = lane & 1;
          if (row >= left) {
#pragma unroll
            for (int i = 0; i < T::ROW / 32; ++i) {
              const int byte = half * (T::ROW / 2) + 16 * i;   // a whole row is cleared, so the swizzle does not matter
              st_shared_f4(sv_base + (byte / T::SLAB_ROW) * T::SLAB + (jkey + row) * T::SLAB_ROW + byte % T::SLAB_ROW, 0, 0, 0, 0);
            }
          }
          fence_async_smem();   // before the stage is handed back to the copies
          __syncwarp();
        }
        float ks[4], vs[4];
        if (T::SCALED) {
          const float* sc = reinterpret_cast<const float*>(stage + 2 * T::KV) + (a.page_size == 16 ? 32 : 16) * warp + 2 * t;
          ks[0] = sc[0]; ks[1] = sc[1]; ks[2] = sc[8]; ks[3] = sc[9];
          vs[0] = sc[128]; vs[1] = sc[129]; vs[2] = sc[136]; vs[3] = sc[137];
        }
        // S = Q K^T: two tiles of 8 keys
        float sc[MT][2][4];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int i = 0; i < 8; ++i) sc[mt][i >> 2][i & 3] = 0.f;
#pragma unroll
        for (int nt = 0; nt < 2; ++nt) {
          const uint32_t key = jkey + nt * 8 + g;
#pragma unroll
          for (int sl = 0; sl < T::SLABS; ++sl) {
            constexpr int CH = T::SLAB_ROW / 64;            // 16-byte chunks of the row that belong to a lane: 1 or 2
#pragma unroll
            for (int c = 0; c < CH; ++c) {
              const uint32_t chunk = t * CH + c;
              const uint32_t sw = T::SLAB_ROW == 128 ? (chunk ^ (key & 7)) : (chunk ^ ((key >> 1) & 3));
              const uint4 w4 = lds128(sk_base + sl * T::SLAB + key * T::SLAB_ROW + (sw << 4));
              const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
#pragma unroll
              for (int i = 0; i < (BF ? 2 : 4); ++i) {
                const int step = BF ? sl * 4 + c * 2 + i : c * 4 + i;
                uint32_t b0, b1;
                if (BF) {
                  b0 = w[BF ? 2 * i : 0];
                  b1 = w[BF ? 2 * i + 1 : 0];
                } else {
                  codes_to_f16<QK>(w[i], b0, b1);
                }
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                  const uint4 q4 = MT == 1 ? qa[MT == 1 ? step : 0] : sQ[(mt * T::STEPS + step) * 32 + lane];
                  mma16<BF>(sc[mt][nt], q4, b0, b1);
                }
              }
            }
          }
        }
        // scores in log2 units; keys behind the last one take no part
        bool grow = false;
#pragma unroll
        for (int nt = 0; nt < 2; ++nt)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const bool out = tail && nt * 8 + 2 * t + c >= left;
            if (T::SCALED && out) vs[2 * nt + c] = 0.f;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                float x = sc[mt][nt][2 * h + c] * fr[mt][h];
                if (T::SCALED) x *= ks[2 * nt + c];
                if (out) x = -INFINITY;
                sc[mt][nt][2 * h + c] = x;
                if (x > m[mt][h] + AP_TAU) grow = true;
              }
          }
        if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
          for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              float x = fmaxf(fmaxf(sc[mt][0][2 * h], sc[mt][0][2 * h + 1]), fmaxf(sc[mt][1][2 * h], sc[mt][1][2 * h + 1]));
              x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
              x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));
              x = fmaxf(x, m[mt][h]);
              const float d = m[mt][h] - x;                  // <= 0; nothing summed yet: -inf (or, 0 x 0, NaN)
              const bool fresh = m[mt][h] == -INFINITY;
              m[mt][h] = x;
              l[mt][h] *= fresh ? 0.f : fast_exp2(d);
              float f = fresh ? 0.f : fast_exp2(d);
              if (T::SCALED) {                               // weights shrink by 2^d, and E with them
                const int En = fresh ? AP_E_LEAST : max(E[mt][h] + (int)fmaxf(floorf(d), -400.f), AP_E_LEAST);
                f = fresh ? 0.f : fast_exp2(d + (float)(E[mt][h] - En));
                E[mt][h] = En;
              }
#pragma unroll
              for (int i = 0; i < NT; ++i) {
                acc[mt][i][2 * h] *= f;
                acc[mt][i][2 * h + 1] *= f;
              }
            }
        }
        // P: exp2, times the value scales, to 16 bits; it is the A operand of O += P V as it stands
        uint4 pa[MT];
        bool over = false;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const float mm = m[mt][h] == -INFINITY ? 0.f : m[mt][h];
            const float up = T::SCALED ? pow2i(AP_W_EXP - E[mt][h]) : 1.f;
#pragma unroll
            for (int nt = 0; nt < 2; ++nt)
#pragma unroll
              for (int c = 0; c < 2; ++c) {
                float& x = sc[mt][nt][2 * h + c];
                x = fast_exp2(x - mm);
                l[mt][h] += x;
                if (T::SCALED) {
                  x *= vs[2 * nt + c];
                  over |= fabsf(x * up) >= AP_W_MOST;
                }
              }
          }
        }
        if (T::SCALED && __any_sync(0xffffffffu, over)) {
#pragma unroll
          for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              float x = fmaxf(fmaxf(fabsf(sc[mt][0][2 * h]), fabsf(sc[mt][0][2 * h + 1])), fmaxf(fabsf(sc[mt][1][2 * h]), fabsf(sc[mt][1][2 * h + 1])));
              x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
              x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));
              const int En = max(E[mt][h], (int)(__float_as_uint(x) >> 23) - 127);
              const float f = E[mt][h] - En < -126 ? 0.f : pow2i(E[mt][h] - En);
              E[mt][h] = En;
#pragma unroll
              for (int i = 0; i < NT; ++i) {
                acc[mt][i][2 * h] *= f;
                acc[mt][i][2 * h + 1] *= f;
              }
            }
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          uint32_t* pr = reinterpret_cast<uint32_t*>(&pa[mt]);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const float up = T::SCALED ? pow2i(AP_W_EXP - E[mt][h]) : 1.f;
#pragma unroll
            for (int nt = 0; nt < 2; ++nt)
              pr[2 * nt + h] = BF ? pack_bf16(sc[mt][nt][2 * h], sc[mt][nt][2 * h + 1])
                                  : pack_f16(sc[mt][nt][2 * h] * up, sc[mt][nt][2 * h + 1] * up);
          }
        }
        // O += P V
        if (BF) {
#pragma unroll
          for (int c = 0; c < DH / 8; c += 2) {
            uint32_t v[4];
            const uint32_t key = jkey + (lane & 15), chunk = c + (lane >> 4);
            ldsm_x4_t(sv_base + (chunk >> 3) * T::SLAB + key * 128 + (((chunk & 7) ^ (key & 7)) << 4), v);
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
              mma16<BF>(acc[mt][c], pa[mt], v[0], v[1]);
              mma16<BF>(acc[mt][c + 1], pa[mt], v[2], v[3]);
            }
          }
        } else {
          uint32_t v[4][NT / 4];                              // four keys, NT consecutive columns
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t key = jkey + (i >> 1) * 8 + 2 * t + (i & 1);
            if (DH == 128) {
              const uint4 x = lds128(sv_base + key * 128 + ((g ^ (key & 7)) << 4));
              v[i][0] = x.x; v[i][1] = x.y; v[i][NT / 4 - 2] = x.z; v[i][NT / 4 - 1] = x.w;
            } else {
              const uint2 x = lds64(sv_base + key * 64 + (((g >> 1) ^ ((key >> 1) & 3)) << 4) + (g & 1) * 8);
              v[i][0] = x.x; v[i][1] = x.y;
            }
          }
#pragma unroll
          for (int w = 0; w < NT / 4; ++w)
#pragma unroll
            for (int hh = 0; hh < 2; ++hh) {
              const uint32_t sel = hh ? 0x7362 : 0x5140;
              uint32_t lo0, hi0, lo1, hi1;
              codes_to_f16<QK>(__byte_perm(v[0][w], v[1][w], sel), lo0, hi0);
              codes_to_f16<QK>(__byte_perm(v[2][w], v[3][w], sel), lo1, hi1);
#pragma unroll
              for (int mt = 0; mt < MT; ++mt) {
                mma16<BF>(acc[mt][4 * w + 2 * hh], pa[mt], lo0, lo1);
                mma16<BF>(acc[mt][4 * w + 2 * hh + 1], pa[mt], hi0, hi1);
              }
            }
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(empty(st));
    }

    // the four warps' results become one
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float x = l[mt][h];
        x += __shfl_xor_sync(0xffffffffu, x, 1);
        x += __shfl_xor_sync(0xffffffffu, x, 2);
        if (t == 0) {
          sM[warp * ROWS + mt * 16 + g + 8 * h] = m[mt][h];
          sL[warp * ROWS + mt * 16 + g + 8 * h] = x;
        }
      }
    if (!epilogue_warps_agree(ok)) {
      if (threadIdx.x == 0) set_status(a.status, SL_DEV_ATTN_TIMEOUT);
      return;
    }
    const bool starts = blk0 == 0, ends = blk0 + nblk == s.nb;
    const long long slot = ((long long)blockIdx.x * 2 + (starts ? 1 : 0)) * ROWS;
    if (starts && !ends && threadIdx.x == 0) {
      const long long last = (u - blk0 + s.nb - 1) / per;    // CTA of the item's last unit
      a.desc[blockIdx.x] = make_int4(s.r0, tile * ROWS, (valid << 16) | kvh, (int)last);
    }
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      if (mt) bar_consumers();
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int row = g + 8 * h;
        float top = -INFINITY;
#pragma unroll
        for (int w = 0; w < 4; ++w) top = fmaxf(top, sM[w * ROWS + mt * 16 + row]);
        const float back = T::SCALED ? pow2i(E[mt][h] - AP_W_EXP) : 1.f;
        const float f = m[mt][h] == -INFINITY ? 0.f : fast_exp2(m[mt][h] - top) * back;
        float* dst = sJoin + (warp * 16 + row) * T::PITCH;
        if (BF) {
#pragma unroll
          for (int i = 0; i < NT; ++i) {
            const int col = 8 * i + 2 * t;
            *reinterpret_cast<float2*>(dst + col + 4 * (col >> 5)) = make_float2(acc[mt][i][2 * h] * f, acc[mt][i][2 * h + 1] * f);
          }
        } else {
#pragma unroll
          for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int i = 0; i < NT; i += 4) {
              const int col = (2 * t + c) * NT + i;
              *reinterpret_cast<float4*>(dst + col + 4 * (col >> 5)) =
                  make_float4(acc[mt][i][2 * h + c] * f, acc[mt][i + 1][2 * h + c] * f, acc[mt][i + 2][2 * h + c] * f, acc[mt][i + 3][2 * h + c] * f);
            }
        }
      }
      bar_consumers();
      const int row = threadIdx.x >> 3, part = threadIdx.x & 7, lr = mt * 16 + row;
      if (lr < valid) {
        float top = -INFINITY, sum = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) top = fmaxf(top, sM[w * ROWS + lr]);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const float mw = sM[w * ROWS + lr];
          if (mw != -INFINITY) sum += sL[w * ROWS + lr] * fast_exp2(mw - top);
          else sum += sL[w * ROWS + lr];                     // 0, or NaN from a score that is not a number
        }
        const int e = tile * ROWS + lr;
        const bool whole = starts && ends;
        const float inv = whole ? (sum == 0.f ? 0.f : 1.f / sum) : 1.f;
        if (!whole && part == 0) a.ml[slot + lr] = make_float2(top, sum);
        bf16* o = a.o + (long long)(s.r0 + e / a.G) * a.o_stride + (long long)(kvh * a.G + e % a.G) * DH;
        float* pt = a.part + (slot + lr) * DH;
#pragma unroll
        for (int i = 0; i < DH / 8; i += 4) {
          const int col = i * 8 + part * 4;                  // the 8 threads of a row take consecutive 16 bytes
          float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const float4 y = *reinterpret_cast<const float4*>(sJoin + (w * 16 + row) * T::PITCH + col + 4 * (col >> 5));
            x.x += y.x; x.y += y.y; x.z += y.z; x.w += y.w;
          }
          if (whole) {
            *reinterpret_cast<uint2*>(o + col) = make_uint2(pack_bf16(x.x * inv, x.y * inv), pack_bf16(x.z * inv, x.w * inv));
          } else {
            *reinterpret_cast<float4*>(pt + col) = x;
          }
        }
      }
    }
    u += nblk;
  }
}

// The pieces of an item that run borders cut: o = sum_i w_i O_i / sum_i w_i l_i, w_i = 2^(m_i - max m), in unit order.  CTA
// (c, y) takes rows y, y + 4, ... of the item that starts in run c; its 8 warps take every eighth piece each.
template <int DH, int ROWS>
__global__ void __launch_bounds__(256) attention_paged_join_kernel(const PagedAttnArgs a) {
  constexpr int PER = DH / 32;
  __shared__ float sO[8][DH];
  __shared__ float sSum[8];
  griddep_wait();
  griddep_launch();
  const int4 d = a.desc[blockIdx.x];
  const int valid = d.z >> 16, kvh = d.z & 0xffff, n = d.w - (int)blockIdx.x + 1;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int row = blockIdx.y; row < valid; row += gridDim.y) {
    auto slot = [&](int i) { return (long long)((blockIdx.x + i) * 2 + (i == 0 ? 1 : 0)) * ROWS + row; };
    float top = -INFINITY;
    for (int i = lane; i < n; i += 32) top = fmaxf(top, a.ml[slot(i)].x);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    float sum = 0.f, x[PER] = {};
#pragma unroll 4
    for (int i = warp; i < n; i += 8) {
      const float2 ml = a.ml[slot(i)];
      const float w = ml.x == -INFINITY ? 0.f : fast_exp2(ml.x - top);
      sum += w * ml.y;
      const float* p = a.part + slot(i) * DH + lane * PER;
#pragma unroll
      for (int c = 0; c < PER; ++c) x[c] += w * p[c];
    }
#pragma unroll
    for (int c = 0; c < PER; ++c) sO[warp][lane * PER + c] = x[c];
    if (lane == 0) sSum[warp] = sum;
    __syncthreads();
    if (threadIdx.x < DH) {
      float y = 0.f, l = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        y += sO[i][threadIdx.x];
        l += sSum[i];
      }
      const int e = d.y + row;
      a.o[(long long)(d.x + e / a.G) * a.o_stride + (long long)(kvh * a.G + e % a.G) * DH + threadIdx.x] =
          __float2bfloat16_rn(l == 0.f ? 0.f : y / l);
    }
    __syncthreads();
  }
}

namespace {

constexpr int AP_MAX_ROWS = 32, AP_MAX_OCC = 2;

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
  const int smem = ap_smem<DH, KIND, MT>() + (a.B + 1) * 8;
  static std::once_flag once;
  static cudaError_t attr;
  std::call_once(once, [] {
    attr = cudaFuncSetAttribute(attention_paged_kernel<DH, KIND, MT>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                ap_smem<DH, KIND, MT>() + (AP_MAX_B + 1) * 8);
  });
  SL_CUDA_TRY(attr);
  const int occ = 2 * (smem + 1024) <= 228 * 1024 ? 2 : 1;
  const int cap = sm_count() * occ, grid = (int)(max_units < cap ? max_units : cap);
  const size_t rows = (size_t)sm_count() * AP_MAX_OCC * 2 * AP_MAX_ROWS;
  a.part = reinterpret_cast<float*>(workspace);
  a.ml = reinterpret_cast<float2*>(a.part + rows * DH);
  a.desc = reinterpret_cast<int4*>(a.ml + rows);
  SL_CUDA_TRY(launch_pdl(attention_paged_kernel<DH, KIND, MT>, dim3(grid), dim3(AP_THREADS), (size_t)smem, st, maps[0], maps[1], maps[2],
                         maps[3], a));
  if (grid > 1 && a.max_tokens > AP_KEYS)   // otherwise no item has two units
    SL_CUDA_TRY(launch_pdl(attention_paged_join_kernel<DH, 16 * MT>, dim3(grid - 1, 4), dim3(256), 0, st, a));
  return SL_OK;
}

}  // namespace

size_t attention_paged_workspace_bytes(int head_dim) {
  if (head_dim != 64 && head_dim != 128) return 0;
  const size_t ctas = (size_t)sm_count() * AP_MAX_OCC;
  return ctas * 2 * AP_MAX_ROWS * (head_dim * sizeof(float) + sizeof(float2)) + ctas * sizeof(int4);
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
  // 16 or 32 rows to a tile: two row tiles share the conversions of the codes, but pad more rows
  const bool wide = (long long)max_rows * a.G > 16ll * B;
  const int tile_rows = wide ? 32 : 16;
  const long long tiles = ((long long)max_rows * a.G + tile_rows - 1) / tile_rows + B;
  const long long max_units = tiles * a.Hkv * ((a.max_tokens + AP_KEYS - 1) / AP_KEYS);
#define SL_AP(DH, KIND) (wide ? launch_ap<DH, KIND, 2>(maps, a, max_units, workspace, st) : launch_ap<DH, KIND, 1>(maps, a, max_units, workspace, st))
  if (c.head_dim == 128) return c.dtype == SL_BF16 ? SL_AP(128, SL_BF16) : c.dtype == SL_E4M3 ? SL_AP(128, SL_E4M3) : SL_AP(128, SL_INT8);
  return c.dtype == SL_BF16 ? SL_AP(64, SL_BF16) : c.dtype == SL_E4M3 ? SL_AP(64, SL_E4M3) : SL_AP(64, SL_INT8);
#undef SL_AP
}

}  // namespace sl
