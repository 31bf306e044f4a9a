// Rows that join a token cache with their queries and keys turned by their
// position, into caches of bf16, fp32 and 4 bits.
//
// Row nth of sequence b stands at position p = seen - drop + nth.  With the
// angle t_j = p freq_j, a pair (x, y) of a query's or key's dims, (2j, 2j + 1)
// or (j, j + half), becomes (x cos t_j - y sin t_j, y cos t_j + x sin t_j).  The
// angle is a product of 64 bits, brought into -pi .. pi before it is rounded:
// in 32 bits position 2^20 would be off by 0.06.
//
// A block of 32 dims in 4 bits has the power of two as its scale that brings its
// largest magnitude to 4 .. 8 (the e2m1 numbers are 0, 1/2, 1, 3/2, 2, 3, 4, 6), and
// values go to the nearest number, ties to the even code.  Keys for it are turned in 64 bits
// and rounded to T first, as the turned keys that the call gives out are: so
// what is held does not go by how a product was rounded next to a border.
#include "paged.h"

namespace fusion {
namespace {

// An angle's cosine and sine in the type that the rotation computes in.
template <typename R> struct Turn {
  R c, s;
};

// The angle, up to 2^50, less the nearest multiple k of pi / 2 (pi / 2 as a sum of two numbers),
// then the series of sine and cosine, whose first terms left out are below 2^-54 of
// the result at pi / 4; k tells which of the two, and its sign.  (A general sincos
// carries the reduction of any angle, at the cost of half the registers.)
constexpr double kHalfPi = 1.570796326794896619;           // nearest to pi / 2
constexpr double kHalfPiRest = 6.123233995736766036e-17;   // pi / 2 - kHalfPi
template <typename R>
__device__ __forceinline__ Turn<R> turn_of(double angle) {
  double k = rint(angle * (1.0 / kHalfPi));
  double r = fma(-k, kHalfPiRest, fma(-k, kHalfPi, angle));
  // (the rounding of that quotient leaves up to 1.2 at 2^50: a second step, exact, brings it
  // within pi / 4)
  const double more = rint(r * (1.0 / kHalfPi));
  r = fma(-more, kHalfPiRest, fma(-more, kHalfPi, r));
  k += more;
  // (past 2^50 an angle of 64 bits holds no better than a quarter radian: whole quarters)
  r = fabs(angle) <= 0x1p50 ? r : r * 0.0;
  const double z = r * r;
  double s = 1.0 / 355687428096000.0, c = 1.0 / 20922789888000.0;  // 17!, 16!
  s = fma(s, z, -1.0 / 1307674368000.0);
  s = fma(s, z, 1.0 / 6227020800.0);
  s = fma(s, z, -1.0 / 39916800.0);
  s = fma(s, z, 1.0 / 362880.0);
  s = fma(s, z, -1.0 / 5040.0);
  s = fma(s, z, 1.0 / 120.0);
  s = fma(s, z, -1.0 / 6.0);
  s = fma(s * z, r, r);
  c = fma(c, z, -1.0 / 87178291200.0);
  c = fma(c, z, 1.0 / 479001600.0);
  c = fma(c, z, -1.0 / 3628800.0);
  c = fma(c, z, 1.0 / 40320.0);
  c = fma(c, z, -1.0 / 720.0);
  c = fma(c, z, 1.0 / 24.0);
  c = fma(c, z, -0.5);
  c = fma(c, z, 1.0);
  const int quarter = (int)(int64_t)k & 3;
  const double x = quarter & 1 ? s : c, y = quarter & 1 ? c : s;
  return {(R)(quarter == 1 || quarter == 2 ? -x : x), (R)(quarter >= 2 ? -y : y)};
}

// Dims d .. d + 7 of a row as they lie in memory, and of a key or query that
// turns in halves the dims that they turn with.
template <typename T> struct Piece {
  typedef typename std::conditional<sizeof(T) == 2, uint2, uint4>::type Quad;  // four values
  Quad x[2], y[2];
};
__device__ __forceinline__ void widen(uint2 u, float* x) {
  x[0] = __uint_as_float(u.x << 16); x[1] = __uint_as_float(u.x & 0xFFFF0000u);
  x[2] = __uint_as_float(u.y << 16); x[3] = __uint_as_float(u.y & 0xFFFF0000u);
}
__device__ __forceinline__ void widen(uint4 u, float* x) {
  x[0] = __uint_as_float(u.x); x[1] = __uint_as_float(u.y);
  x[2] = __uint_as_float(u.z); x[3] = __uint_as_float(u.w);
}

// The piece's eight values, turned in type C (turns: the row's angles).
template <typename C, typename T, typename R>
__device__ __forceinline__ void turn8(const RotaryArgs& a, const Piece<T>& p, int d, const Turn<R>* turns,
                                      float* x) {
  if (d >= 2 * a.half) return;
  if (a.pairs) {
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const Turn<C> t{(C)turns[d / 2 + i].c, (C)turns[d / 2 + i].s};
      const C u = x[2 * i], v = x[2 * i + 1];
      x[2 * i] = (float)fma(u, t.c, -(v * t.s));
      x[2 * i + 1] = (float)fma(v, t.c, u * t.s);
    }
    return;
  }
  // (half is a multiple of 4: four dims in a row belong to one half)
#pragma unroll
  for (int h = 0; h < 2; h++) {
    const int e = d + 4 * h;
    const bool second = e >= a.half;
    const int j = second ? e - a.half : e;
    float y[4];
    widen(p.y[h], y);
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const Turn<C> t{(C)turns[j + i].c, (C)turns[j + i].s};
      const C u = x[4 * h + i], v = y[i], s = second ? t.s : -t.s;
      x[4 * h + i] = (float)fma(u, t.c, v * s);
    }
  }
}

// Eight values in 4 bits, of a block whose other values are in the three lanes
// beside this one (lane / 4 is one block): codes, and the block's scale.
__device__ __forceinline__ uint32_t to_four(const float* x, uint32_t* scale) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; i++) top = max(top, __float_as_uint(x[i]) & 0x7FFFFFFFu);
  top = max(top, (uint32_t)lane_xor_i<1>((int)top));
  top = max(top, (uint32_t)lane_xor_i<2>((int)top));
  const uint32_t e = top >> 23;  // 127 + floor(log2(the largest))
  if (e == 255) {  // infinite or NaN: the block is NaN
    *scale = 255;
    return 0;
  }
  *scale = min(max(e, 4u) - 2, 252u);
  const float s = __uint_as_float(*scale << 23);
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[0], x[1], s, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[2], x[3], s, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[4], x[5], s, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[6], x[7], s, 3);
}

// Eight dims of a query, key or value row: where they come from.
template <typename T> struct Task {
  const T* row;
  int vec, d;  // queries, then keys, then values; first dim
  Piece<T> p;
};
// Task t of row r (all past the last: `real` false, nothing is read).
template <typename T>
__device__ __forceinline__ void load_task(const CacheArgs& c, const RotaryArgs& a, FastDiv pieces, int64_t r,
                                          int t, bool real, Task<T>* k) {
  typedef typename Piece<T>::Quad Quad;
  k->vec = (int)quot((uint32_t)t, pieces);
  k->d = (t - k->vec * (int)pieces.d) * 8;
  const int key = k->vec - a.H, value = key - c.Hkv;
  k->row = key < 0 ? (const T*)a.q + r * a.q_row + k->vec * a.q_head
           : value < 0 ? (const T*)a.k + r * a.k_row + key * a.k_head
                       : (const T*)a.v + r * a.v_row + value * a.v_head;
  if (!real) return;
  if constexpr (sizeof(T) == 2) {
    const uint4 u = *(const uint4*)(k->row + k->d);
    k->p.x[0] = make_uint2(u.x, u.y);
    k->p.x[1] = make_uint2(u.z, u.w);
  } else {
    k->p.x[0] = *(const uint4*)(k->row + k->d);
    k->p.x[1] = *(const uint4*)(k->row + k->d + 4);
  }
  if (value < 0 && !a.pairs && k->d < 2 * a.half) {
#pragma unroll
    for (int h = 0; h < 2; h++) {
      const int e = k->d + 4 * h;
      k->p.y[h] = *(const Quad*)(k->row + (e >= a.half ? e - a.half : e + a.half));
    }
  }
}

// The task's eight values, turned, to where they go: the call's outputs, and
// place `place` of page `page` (below 0: none).
template <typename T, bool FOUR, typename R>
__device__ __forceinline__ void store_task(const CacheArgs& c, const RotaryArgs& a, const Task<T>& k,
                                           const Turn<R>* turns, int64_t r, int page, int place) {
  const int d = k.d, key = k.vec - a.H, value = key - c.Hkv;
  float x[8];
  widen(k.p.x[0], x);
  widen(k.p.x[1], x + 4);
  if (key < 0) {
    turn8<float>(a, k.p, d, turns, x);
    store8((T*)a.q_out + (r * a.H + k.vec) * c.dh + d, x);
    return;
  }
  const int h = value < 0 ? key : value;
  if (value < 0) {
    turn8<R>(a, k.p, d, turns, x);
    if (sizeof(T) == 2 && FOUR)
#pragma unroll
      for (int i = 0; i < 8; i++) x[i] = bf16_to_f32(f32_to_bf16(x[i]));
    if (a.k_out) store8((T*)a.k_out + (r * c.Hkv + h) * c.dh + d, x);
  }
  if constexpr (FOUR) {
    uint32_t scale;
    const uint32_t codes = to_four(x, &scale);
    if (page < 0) return;
    uint8_t* to = value < 0 ? (uint8_t*)c.k + page * c.k_page + place * c.k_row + h * c.k_head
                            : (uint8_t*)c.v + page * c.v_page + place * c.v_row + h * c.v_head;
    uint8_t* sc = value < 0 ? c.ks + page * c.ks_page + place * c.ks_row + h * c.ks_head
                            : c.vs + page * c.vs_page + place * c.vs_row + h * c.vs_head;
    *(uint32_t*)(to + d / 2) = codes;
    if ((d & 31) == 0) sc[d / 32] = (uint8_t)scale;
  } else if (page >= 0) {
    T* to = value < 0 ? (T*)c.k + page * c.k_page + place * c.k_row + h * c.k_head
                      : (T*)c.v + page * c.v_page + place * c.v_row + h * c.v_head;
    store8(to + d, x);
  }
}

// Slots in use, positions so far, both without the tokens that are replaced.
struct Start {
  int have, seen, drop;
};
__device__ __forceinline__ Start start_of(const CacheArgs& c, const RotaryArgs& a, int b) {
  const int n = held(c, b), drop = a.drop ? max(0, min(a.drop[b], n)) : 0;
  return {n - drop, (int)((uint32_t)c.seen[b] - (uint32_t)drop), drop};
}
// Page and place in it of a slot; page -1: not held.
struct Place {
  int page, place;
};
__device__ __forceinline__ Place place_of(const CacheArgs& c, int b, int64_t slot) {
  if (slot >= c.cap) return {-1, 0};
  const uint32_t pg = quot((uint32_t)slot, c.page);
  return {page_of(c, b, pg), (int)(slot - (int64_t)pg * c.page.d)};
}
__device__ __forceinline__ void move_lengths(const CacheArgs& c, Start st, int b, int rows) {
  if (rows == 0 && st.drop == 0) return;
  const int fit = min(rows, c.cap - st.have);
  c.len[b] = st.have + fit;
  c.seen[b] = (int)((uint32_t)st.seen + (uint32_t)fit);
}

// One workgroup per sequence, for few rows each: the lengths move on in it.  A
// chain of loads bounds it, so the workgroup has a thread for every task (up to
// 1024), whose first load goes out before the angles are computed.
template <typename T, bool FOUR, typename Seqs>
__global__ __launch_bounds__(1024) void rotary_few(CacheArgs c, RotaryArgs a, FastDiv pieces, FastDiv tasks,
                                                   Seqs sq) {
  typedef typename std::conditional<FOUR, double, float>::type R;
  __shared__ Turn<R> turns[APPEND_FEW][64];
  const int tid = threadIdx.x, threads = blockDim.x;
  int b = blockIdx.x, n = 1;
  int64_t r0 = b;
  if constexpr (std::is_same<Seqs, AppendSeqs>::value) {
    b += sq.first;
    r0 = sq.cu[blockIdx.x];
    n = sq.cu[blockIdx.x + 1] - sq.cu[blockIdx.x];
  }
  const int total = n * (int)tasks.d;
  Task<T> k;
  auto load = [&](int t) {
    const int i = (int)quot((uint32_t)t, tasks);
    load_task(c, a, pieces, r0 + i, t - i * (int)tasks.d, true, &k);
  };
  if (tid < total) load(tid);
  const Start st = start_of(c, a, b);
  for (int i = tid; i < n * 64; i += threads)
    if ((i & 63) < a.half)
      turns[i >> 6][i & 63] = turn_of<R>((double)((int64_t)st.seen + (i >> 6)) * (double)a.freq[i & 63]);
  if (tid < n && (int64_t)st.have + tid < c.cap) {
    c.weight[(int64_t)b * c.cap + st.have + tid] = 0.f;
    c.pos[(int64_t)b * c.cap + st.have + tid] = (int)((int64_t)st.seen + tid);
  }
  __syncthreads();  // (all waves have the lengths, too)
  if (tid == 0) move_lengths(c, st, b, n);
  for (int t = tid; t < total; t += threads) {
    if (t != tid) load(t);
    const int i = (int)quot((uint32_t)t, tasks);
    const Place at = place_of(c, b, (int64_t)st.have + i);
    store_task<T, FOUR, R>(c, a, k, turns[i], r0 + i, at.page, at.place);
  }
}

// A wave per row, two tasks a lane at a time; the lengths move on in a launch of
// their own.  Bound by its bytes: 19,234 bf16 rows of 48 heads of 128 (512 MB in and
// out) take 102 us, 5.0 TB/s, where a copy reaches 5.2; 104 with one task at a
// time.  (A wave that goes on to further rows would hold the series' constants and the
// call's strides in registers that the tasks need.)
template <typename T, bool FOUR>
__global__ __launch_bounds__(256) void rotary_many(CacheArgs c, RotaryArgs a, FastDiv pieces, int tasks,
                                                   int block0, AppendSeqs sq) {
  typedef typename std::conditional<FOUR, double, float>::type R;
  constexpr int U = 2;
  __shared__ Turn<R> turns_all[4][64];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  Turn<R>* turns = turns_all[wave];
  const int r = sq.cu[0] + (block0 + (int)blockIdx.x) * 4 + wave;
  if (r >= sq.cu[sq.n]) return;
  int lo = 0, hi = sq.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (sq.cu[mid] <= r) lo = mid; else hi = mid - 1;
  }
  const int b = sq.first + lo, nth = r - sq.cu[lo];
  const Start st = start_of(c, a, b);
  const int64_t slot = (int64_t)st.have + nth, pos = (int64_t)st.seen + nth;
  const Place at = place_of(c, b, slot);
  if (lane < a.half) turns[lane] = turn_of<R>((double)pos * (double)a.freq[lane]);
  if (lane == 0 && slot < c.cap) {
    c.weight[(int64_t)b * c.cap + slot] = 0.f;
    c.pos[(int64_t)b * c.cap + slot] = (int)pos;
  }
  // (the angles are the wave's own, and its LDS operations stay in order)
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  for (int t0 = lane; t0 < tasks; t0 += 64 * U) {
    Task<T> k[U];
#pragma unroll
    for (int u = 0; u < U; u++) load_task(c, a, pieces, r, t0 + 64 * u, t0 + 64 * u < tasks, &k[u]);
#pragma unroll
    for (int u = 0; u < U; u++)
      if (t0 + 64 * u < tasks) store_task<T, FOUR, R>(c, a, k[u], turns, r, at.page, at.place);
  }
}

__global__ __launch_bounds__(256) void rotary_lengths(CacheArgs c, RotaryArgs a, AppendSeqs sq) {
  const int t = blockIdx.x * 256 + threadIdx.x;
  if (t >= sq.n) return;
  const int b = sq.first + t;
  move_lengths(c, start_of(c, a, b), b, sq.cu[t + 1] - sq.cu[t]);
}

template <typename T, bool FOUR>
hipError_t launch_rotary(const CacheArgs& c, const RotaryArgs& a, const int32_t* cu_host, hipStream_t s) {
  const FastDiv pieces = fast_div((uint32_t)c.dh / 8);
  const int tasks = (a.H + 2 * c.Hkv) * (c.dh / 8);
  const FastDiv by_row = fast_div((uint32_t)tasks);
  auto threads = [&](int rows) { return std::min((int64_t)1024, ((int64_t)rows * tasks + 63) / 64 * 64); };
  if (!cu_host) {
    rotary_few<T, FOUR><<<c.B, threads(1), 0, s>>>(c, a, pieces, by_row, OneRowEach{});
    return hipGetLastError();
  }
  AppendSeqs sq;
  for (int f = 0; f < c.B; f += APPEND_SEQS) {
    sq.first = f;
    sq.n = std::min(c.B - f, APPEND_SEQS);
    std::copy(cu_host + f, cu_host + f + sq.n + 1, sq.cu);
    const int rows = sq.cu[sq.n] - sq.cu[0];
    int most = 0;
    for (int i = 0; i < sq.n; i++) most = std::max(most, sq.cu[i + 1] - sq.cu[i]);
    if (most <= APPEND_FEW) {
      if (rows == 0 && !a.drop) continue;
      rotary_few<T, FOUR><<<sq.n, threads(std::max(most, 1)), 0, s>>>(c, a, pieces, by_row, sq);
    } else {
      if (hipError_t e = in_launches((rows + 3) / 4, 256, [&](int first, unsigned grid) {
            rotary_many<T, FOUR><<<grid, 256, 0, s>>>(c, a, pieces, tasks, first, sq);
          }))
        return e;
      rotary_lengths<<<(sq.n + 255) / 256, 256, 0, s>>>(c, a, sq);
    }
    if (hipError_t e = hipGetLastError()) return e;
  }
  return hipSuccess;
}
}  // namespace

template <typename T>
hipError_t launch_append_rotary(const CacheArgs& c, const RotaryArgs& a, const int32_t* cu_host,
                                hipStream_t s) {
  return c.ks ? launch_rotary<T, true>(c, a, cu_host, s) : launch_rotary<T, false>(c, a, cu_host, s);
}
template hipError_t launch_append_rotary<float>(const CacheArgs&, const RotaryArgs&, const int32_t*,
                                                hipStream_t);
template hipError_t launch_append_rotary<bf16_t>(const CacheArgs&, const RotaryArgs&, const int32_t*,
                                                 hipStream_t);

}  // namespace fusion
