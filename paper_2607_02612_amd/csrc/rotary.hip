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

constexpr double kTwoPi = 6.283185307179586477;        // nearest to 2 pi
constexpr double kTwoPiRest = 2.449293598294706414e-16;  // 2 pi - kTwoPi
template <typename R>
__device__ __forceinline__ Turn<R> turn_of(double angle) {
  const double k = rint(angle * (1.0 / kTwoPi));
  const double r = fma(-k, kTwoPiRest, fma(-k, kTwoPi, angle));
  double s, c;
  sincos(r, &s, &c);
  return {(R)c, (R)s};
}

// Dims d .. d + 7 of a row, turned (x: those dims; row: the row's memory).
template <typename T, typename R>
__device__ __forceinline__ void turn8(const RotaryArgs& a, const T* row, int d, const Turn<R>* turns,
                                      float* x) {
  if (d >= 2 * a.half) return;
  if (a.pairs) {
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const Turn<R> t = turns[d / 2 + i];
      const R u = x[2 * i], v = x[2 * i + 1];
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
    load4(row + (second ? j : j + a.half), y);
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const Turn<R> t = turns[j + i];
      const R u = x[4 * h + i], v = y[i], s = second ? t.s : -t.s;
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

// Row r of the call, to the slot `slot` of sequence b, position pos: `step` lanes
// take eight dims each.  turns: LDS of the lanes' wave, 64 angles.
template <typename T, bool FOUR, typename R>
__device__ __forceinline__ void rotary_row(const CacheArgs& c, const RotaryArgs& a, FastDiv pieces,
                                           Turn<R>* turns, int b, int64_t r, int64_t slot, int64_t pos,
                                           int lane, int step) {
  const int in_wave = lane & 63;
  if (in_wave < a.half) turns[in_wave] = turn_of<R>((double)pos * (double)a.freq[in_wave]);
  // (the angles are the wave's own, and its LDS operations stay in order)
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  const bool held = slot < c.cap;
  int page = -1, place = 0;
  if (held) {
    if (lane == 0) {
      c.weight[(int64_t)b * c.cap + slot] = 0.f;
      c.pos[(int64_t)b * c.cap + slot] = (int)pos;
    }
    const uint32_t pg = quot((uint32_t)slot, c.page);
    page = page_of(c, b, pg);
    place = (int)(slot - (int64_t)pg * c.page.d);
  }
  const int all = (a.H + 2 * c.Hkv) * (int)pieces.d;
  for (int t = lane; t < all; t += step) {
    const int vec = (int)quot((uint32_t)t, pieces), d = (t - vec * (int)pieces.d) * 8;
    float x[8];
    if (vec < a.H) {
      const T* row = (const T*)a.q + r * a.q_row + vec * a.q_head;
      load8(row + d, x);
      turn8(a, row, d, turns, x);
      store8((T*)a.q_out + (r * a.H + vec) * c.dh + d, x);
      continue;
    }
    const bool key = vec < a.H + c.Hkv;
    const int h = vec - a.H - (key ? 0 : c.Hkv);
    const T* row = key ? (const T*)a.k + r * a.k_row + h * a.k_head
                       : (const T*)a.v + r * a.v_row + h * a.v_head;
    load8(row + d, x);
    if (key) {
      turn8(a, row, d, turns, x);
      if (sizeof(T) == 2 && FOUR)
#pragma unroll
        for (int i = 0; i < 8; i++) x[i] = bf16_to_f32(f32_to_bf16(x[i]));
      if (a.k_out) store8((T*)a.k_out + (r * c.Hkv + h) * c.dh + d, x);
    }
    if constexpr (FOUR) {
      uint32_t scale;
      const uint32_t codes = to_four(x, &scale);
      if (page < 0) continue;
      uint8_t* to = key ? (uint8_t*)c.k + page * c.k_page + place * c.k_row + h * c.k_head
                        : (uint8_t*)c.v + page * c.v_page + place * c.v_row + h * c.v_head;
      uint8_t* sc = key ? c.ks + page * c.ks_page + place * c.ks_row + h * c.ks_head
                        : c.vs + page * c.vs_page + place * c.vs_row + h * c.vs_head;
      *(uint32_t*)(to + d / 2) = codes;
      if ((t & 3) == 0) sc[d / 32] = (uint8_t)scale;
    } else if (page >= 0) {
      T* to = key ? (T*)c.k + page * c.k_page + place * c.k_row + h * c.k_head
                  : (T*)c.v + page * c.v_page + place * c.v_row + h * c.v_head;
      store8(to + d, x);
    }
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // (the next row's angles come after its reads)
  __builtin_amdgcn_wave_barrier();
}

// Slots in use, positions so far, both without the tokens that are replaced.
struct Start {
  int have, seen, drop;
};
__device__ __forceinline__ Start start_of(const CacheArgs& c, const RotaryArgs& a, int b) {
  const int n = held(c, b), drop = a.drop ? max(0, min(a.drop[b], n)) : 0;
  return {n - drop, (int)((uint32_t)c.seen[b] - (uint32_t)drop), drop};
}
__device__ __forceinline__ void move_lengths(const CacheArgs& c, Start st, int b, int rows) {
  if (rows == 0 && st.drop == 0) return;
  const int fit = min(rows, c.cap - st.have);
  c.len[b] = st.have + fit;
  c.seen[b] = (int)((uint32_t)st.seen + (uint32_t)fit);
}

// One workgroup per sequence, for few rows each: the lengths move on in it.
template <typename T, bool FOUR, typename Seqs>
__global__ __launch_bounds__(256) void rotary_few(CacheArgs c, RotaryArgs a, FastDiv pieces, Seqs sq) {
  typedef typename std::conditional<FOUR, double, float>::type R;
  __shared__ Turn<R> turns[4][64];
  int b = blockIdx.x, n = 1;
  int64_t r0 = b;
  if constexpr (std::is_same<Seqs, AppendSeqs>::value) {
    b += sq.first;
    r0 = sq.cu[blockIdx.x];
    n = sq.cu[blockIdx.x + 1] - sq.cu[blockIdx.x];
  }
  const Start st = start_of(c, a, b);
  __syncthreads();  // all waves have the lengths
  if (threadIdx.x == 0) move_lengths(c, st, b, n);
  const int wave = threadIdx.x >> 6;
  if (n == 1) {
    rotary_row<T, FOUR, R>(c, a, pieces, turns[wave], b, r0, st.have, st.seen, threadIdx.x, 256);
  } else {
    for (int i = wave; i < n; i += 4)
      rotary_row<T, FOUR, R>(c, a, pieces, turns[wave], b, r0 + i, (int64_t)st.have + i,
                             (int64_t)st.seen + i, threadIdx.x & 63, 64);
  }
}

// A wave per row; the lengths move on in a launch of their own.
template <typename T, bool FOUR>
__global__ __launch_bounds__(256) void rotary_many(CacheArgs c, RotaryArgs a, FastDiv pieces,
                                                   AppendSeqs sq) {
  typedef typename std::conditional<FOUR, double, float>::type R;
  __shared__ Turn<R> turns[4][64];
  const int wave = threadIdx.x >> 6, end = sq.cu[sq.n];
  for (int r = sq.cu[0] + blockIdx.x * 4 + wave; r < end; r += gridDim.x * 4) {
    int lo = 0, hi = sq.n - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (sq.cu[mid] <= r) lo = mid; else hi = mid - 1;
    }
    const int b = sq.first + lo, nth = r - sq.cu[lo];
    const Start st = start_of(c, a, b);
    rotary_row<T, FOUR, R>(c, a, pieces, turns[wave], b, r, (int64_t)st.have + nth,
                           (int64_t)st.seen + nth, threadIdx.x & 63, 64);
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
  if (!cu_host) {
    rotary_few<T, FOUR><<<c.B, 256, 0, s>>>(c, a, pieces, OneRowEach{});
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
      rotary_few<T, FOUR><<<sq.n, 256, 0, s>>>(c, a, pieces, sq);
    } else {
      rotary_many<T, FOUR><<<std::min((rows + 3) / 4, APPEND_BLOCKS), 256, 0, s>>>(c, a, pieces, sq);
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
