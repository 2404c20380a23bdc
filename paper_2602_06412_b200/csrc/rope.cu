// Rotary positions on packed q and k rows at any position, for rows that a fused step does not rotate itself: pair i of the
// first `rotary_dim` elements of a head turns by the angle position * freq[i],
//   (a, b) -> scale (a cos - b sin, b cos + a sin),
// pairs (i, i + rotary_dim / 2) or (2i, 2i + 1); the rest of the head is copied.
//
// Far positions: position * freq is taken in 64 bits and reduced there to an eighth of a turn either side of a quarter turn (2 pi
// in two terms), sine and cosine of what is left in 32 bits, so that the angle's error is 2^-53 of it and not 2^-24.  Sines are shared by
// all heads of a row: a block computes those of its rows once, in shared memory, while its first loads are on their way, and a thread
// keeps those of its V pairs in registers while it goes through the heads.
//
// Memory-bound: 16-byte accesses of either half of V pairs, 4 heads in flight to a thread.  In a graph, 64 heads of 128 in bf16: 12288 rows
// 63.5 us (6.3 TB/s, 97 % of the copy rate; sines read from shared memory for every head instead: 120 us, two thirds of it bank conflicts and
// registers), 4 rows to a block (2: 69, 8: 66 us), 4 heads in flight (2: 66, 8: 65.5); 32 rows at positions up to 10^6 4.2 us.  Neighbours as pairs 75.5 us (a
// thread's two loads lie side by side, so a warp's are apart); fp32 125 us for 805 MB, neighbours 136.5 (that variant spills 60 bytes).
#include "common.cuh"

namespace sl {
namespace {

constexpr int ROPE_THREADS = 256, ROPE_ROWS = 4, ROPE_U = 4, ROPE_BLOCKS = 3;

struct RopeArgs {
  const void* in[2];
  void* out[2];
  long long in_stride[2], out_stride[2];
  int heads[2];
  const double* freq;
  const int32_t *positions, *n_active;
  int32_t* status;
  float scale, scale_sin;          // the sine's is negative for the transposed rotation
  int max_rows, N, half, dh;       // half = pairs to a head
  int chunks, rest;                // groups of V pairs to a head, and of V elements to be copied
  int rows, slots, parts;          // a block: rows, and heads of each at once; blocks that share these rows
};

// cosine and sine of pos * freq
__device__ __forceinline__ float2 turn(int pos, double freq) {
  const double angle = (double)pos * freq;
  const double n = rint(angle * 0.15915494309189535);               // 1 / (2 pi)
  const double r = fma(-n, 2.4492935982947064e-16, fma(-n, 6.283185307179586, angle));
  const double quarters = r * 0.6366197723675814;                   // 2 / pi
  const double q = rint(quarters);
  float s, c;
  sincospif(0.5f * (float)(quarters - q), &s, &c);
  const int k = (int)q & 3;
  return make_float2(k == 0 ? c : k == 1 ? -s : k == 2 ? -c : s, k == 0 ? s : k == 1 ? c : k == 2 ? -s : -c);
}

// V consecutive elements, as stored
template <typename T, int V> struct alignas(sizeof(T) * V) Vec { T e[V]; };
template <typename T, int V> __device__ __forceinline__ Vec<T, V> load(const T* p) {
  Vec<T, V> v;
  if (sizeof(T) * V == 16) *reinterpret_cast<uint4*>(&v) = *reinterpret_cast<const uint4*>(p);
  else
#pragma unroll
    for (int i = 0; i < V; ++i) v.e[i] = p[i];
  return v;
}
template <typename T, int V> __device__ __forceinline__ void store(T* p, const Vec<T, V>& v) {
  if (sizeof(T) * V == 16) *reinterpret_cast<uint4*>(p) = *reinterpret_cast<const uint4*>(&v);
  else
#pragma unroll
    for (int i = 0; i < V; ++i) p[i] = v.e[i];
}

// A thread keeps the sines of V pairs and goes through heads with them, U at a time.
template <typename T, int V, bool INTERLEAVED, int U>
__global__ void __launch_bounds__(ROPE_THREADS, ROPE_BLOCKS) rope_rows_kernel(RopeArgs a) {
  extern __shared__ float2 turns[];                  // [rows][half]
  griddep_wait();
  griddep_launch();
  const int M = min(*a.n_active, a.max_rows), group = blockIdx.x / a.parts, part = blockIdx.x % a.parts;
  const int r0 = group * a.rows, nr = min(a.rows, M - r0), all = a.heads[0] + a.heads[1];
  if (nr <= 0) return;
  const int second = INTERLEAVED ? V : a.half;       // how far behind a thread's first V elements its other V are
  const int wide = min(a.chunks, ROPE_THREADS), slot = threadIdx.x / wide, row = slot % a.rows, step = a.slots * a.parts;
  const int h0 = slot / a.rows + part * a.slots;
  const bool works = slot < a.rows * a.slots && row < nr && a.positions[r0 + min(row, nr - 1)] >= 0;
  const T *from_q = (const T*)a.in[0] + (r0 + row) * a.in_stride[0], *from_k = (const T*)a.in[1] + (r0 + row) * a.in_stride[1] - (long long)a.heads[0] * a.dh;
  T *to_q = (T*)a.out[0] + (r0 + row) * a.out_stride[0], *to_k = (T*)a.out[1] + (r0 + row) * a.out_stride[1] - (long long)a.heads[0] * a.dh;
  Vec<T, V> x[U], y[U];
  auto at = [&](int h, int c) { return h * a.dh + (INTERLEAVED ? 2 : 1) * V * c; };   // k's heads come after q's
  auto fetch = [&](int h, int c) {
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (h + u * step < all) {
        const T* p = (h + u * step < a.heads[0] ? from_q : from_k) + at(h + u * step, c);
        x[u] = load<T, V>(p);
        y[u] = load<T, V>(p + second);
      }
  };
  int c = threadIdx.x % wide;
  if (works) fetch(h0, c);
  for (int j = threadIdx.x; j < nr * a.half; j += ROPE_THREADS) {
    const int r = j / a.half;
    int pos = a.positions[r0 + r];
    if (pos < 0) {                                   // the row is left as it is
      set_status(a.status, SL_DEV_BAD_INDEX);
      continue;
    }
    if (a.N > 0) pos %= a.N;
    const float2 t = turn(pos, a.freq[j - r * a.half]);
    turns[j] = make_float2(t.x * a.scale, t.y * a.scale_sin);
  }
  __syncthreads();
  for (; works && c < a.chunks; c += wide) {
    float2 t[V];
#pragma unroll
    for (int k = 0; k < V; ++k) t[k] = turns[row * a.half + V * c + k];
    if (c >= wide) fetch(h0, c);
    for (int h = h0; h < all; h += U * step) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (h + u * step >= all) break;
        T* p = (h + u * step < a.heads[0] ? to_q : to_k) + at(h + u * step, c);
#pragma unroll
        for (int k = 0; k < V; ++k) {
          T& e = INTERLEAVED ? (2 * k < V ? x[u].e[(2 * k) % V] : y[u].e[(2 * k) % V]) : x[u].e[k];
          T& f = INTERLEAVED ? (2 * k + 1 < V ? x[u].e[(2 * k + 1) % V] : y[u].e[(2 * k + 1) % V]) : y[u].e[k];
          const float g = to_f(e), i = to_f(f);
          e = from_f<T>(g * t[k].x - i * t[k].y);
          f = from_f<T>(i * t[k].x + g * t[k].y);
        }
        store<T, V>(p, x[u]);
        store<T, V>(p + second, y[u]);
      }
      fetch(h + U * step, c);
    }
  }
  // what is not rotated, in a call that is not in place
  for (int i = part * ROPE_THREADS + threadIdx.x; i < nr * all * a.rest; i += a.parts * ROPE_THREADS) {
    const int w = i / a.rest, r = w / all, h = w - r * all, which = h >= a.heads[0];
    if (a.positions[r0 + r] < 0) continue;
    const long long e = (long long)(which ? h - a.heads[0] : h) * a.dh + 2 * a.half + V * (i - w * a.rest);
    store<T, V>((T*)a.out[which] + (r0 + r) * a.out_stride[which] + e, load<T, V>((const T*)a.in[which] + (r0 + r) * a.in_stride[which] + e));
  }
}

template <typename T, int V, bool INTERLEAVED>
int launch_rows(RopeArgs& a, bool copy, cudaStream_t st) {
  a.chunks = a.half / V;
  a.rest = copy ? (a.dh - 2 * a.half) / V : 0;
  const int wide = a.chunks < ROPE_THREADS ? a.chunks : ROPE_THREADS, all = a.heads[0] + a.heads[1], slots = ROPE_THREADS / wide;
  // Few rows: blocks of one row that share its heads, one head to a thread, so that every load of the call is on its way at once.
  // Many: as many rows to a block as leave each thread some heads.
  const bool few = (long long)a.max_rows * all * wide <= (long long)sm_count() * 8 * ROPE_THREADS;
  a.rows = few ? 1 : ROPE_ROWS < slots ? ROPE_ROWS : slots;
  a.slots = slots / a.rows;
  a.parts = few ? (all + a.slots - 1) / a.slots : 1;
  const long long groups = ((long long)a.max_rows + a.rows - 1) / a.rows;
  if (groups * a.parts > 0x7fffffffll) return SL_EUNSUPPORTED;
  const dim3 grid((unsigned)(groups * a.parts));
  const size_t smem = (size_t)a.rows * a.half * sizeof(float2);
  if (few) SL_CUDA_TRY(launch_pdl(rope_rows_kernel<T, V, INTERLEAVED, 1>, grid, dim3(ROPE_THREADS), smem, st, a));
  else SL_CUDA_TRY(launch_pdl(rope_rows_kernel<T, V, INTERLEAVED, ROPE_U>, grid, dim3(ROPE_THREADS), smem, st, a));
  return SL_OK;
}

template <typename T> int launch_typed(RopeArgs& a, bool interleaved, bool copy, cudaStream_t st) {
  constexpr int V = 16 / sizeof(T);
  bool wide = a.half % V == 0 && a.dh % V == 0;
  for (int i = 0; i < 2; ++i)
    if (a.heads[i])
      wide &= ((reinterpret_cast<uintptr_t>(a.in[i]) | reinterpret_cast<uintptr_t>(a.out[i])) & 15) == 0 &&
              (a.in_stride[i] | a.out_stride[i]) % V == 0;
  if (wide) return interleaved ? launch_rows<T, V, true>(a, copy, st) : launch_rows<T, V, false>(a, copy, st);
  return interleaved ? launch_rows<T, 1, true>(a, copy, st) : launch_rows<T, 1, false>(a, copy, st);
}

}  // namespace

int launch_rope_rows(const surelock_rope_cfg& c, const void* q, long long q_stride, int H, const void* k, long long k_stride, int Hkv,
                     int head_dim, const int32_t* positions, int N, const int32_t* n_active, int max_rows, void* q_out,
                     long long q_out_stride, void* k_out, long long k_out_stride, int dtype, int transposed, int32_t* status,
                     cudaStream_t st) {
  RopeArgs a = {};
  a.in[0] = q; a.in[1] = k; a.out[0] = q_out; a.out[1] = k_out;
  a.in_stride[0] = q_stride; a.in_stride[1] = k_stride; a.out_stride[0] = q_out_stride; a.out_stride[1] = k_out_stride;
  a.heads[0] = H; a.heads[1] = k ? Hkv : 0;
  a.freq = c.freq; a.positions = positions; a.n_active = n_active; a.status = status;
  a.scale = c.scale; a.scale_sin = transposed ? -c.scale : c.scale;
  a.max_rows = max_rows; a.N = N; a.half = c.rotary_dim / 2; a.dh = head_dim;
  const bool copy = q != q_out || (k && k != k_out);   // what is not rotated stays where it is in a call in place
  return dtype == SL_BF16 ? launch_typed<bf16>(a, c.interleaved, copy, st) : launch_typed<float>(a, c.interleaved, copy, st);
}

// Frequencies theta^(-2i / D) of the pairs, scaled for contexts longer than the model was trained on (include/surelock.h).
void rope_frequencies(double* freq, float* scale, int D, double theta, const surelock_rope_scaling* s) {
  const double two_pi = 6.283185307179586;
  const int kind = s ? s->kind : SL_ROPE_PLAIN;
  const double f = s ? s->factor : 1.0, L = s ? s->original_len : 0.0;
  double m = 1.0;
  if (kind == SL_ROPE_NTK) theta *= pow(f, (double)D / (D - 2));
  double low = 0.0, high = 1.0;
  if (kind == SL_ROPE_YARN) {
    // the pairs that make `fast` or more turns over the original length keep their frequency, those of `slow` or fewer are divided
    auto pair_of = [&](double turns) { return D * log(L / (turns * two_pi)) / (2.0 * log(theta)); };
    low = fmax(floor(pair_of(s->fast)), 0.0);
    high = fmin(ceil(pair_of(s->slow)), D - 1.0);
    if (high <= low) high = low + 0.001;
    m = s->attn_scale > 0.0 ? s->attn_scale : 0.1 * log(f) + 1.0;
    if (f <= 1.0 && !(s->attn_scale > 0.0)) m = 1.0;
  }
  for (int i = 0; i < D / 2; ++i) {
    double w = pow(theta, -2.0 * i / D);
    if (kind == SL_ROPE_LINEAR) w /= f;
    if (kind == SL_ROPE_YARN) {
      const double ramp = fmin(fmax((i - low) / (high - low), 0.0), 1.0);
      w = w / f * ramp + w * (1.0 - ramp);
    }
    if (kind == SL_ROPE_BANDS) {
      const double turns = L * w / two_pi;             // over the original length
      const double keep = fmin(fmax((turns - s->slow) / (s->fast - s->slow), 0.0), 1.0);
      w = w / f * (1.0 - keep) + w * keep;
    }
    freq[i] = w;
  }
  *scale = (float)m;
}

}  // namespace sl
