// Attention over packed ragged rows under a sliding window with a few first
// rows that stay visible:
//   o_i = sum_{j in S_i} E_ij v_j / sum_{j in S_i} E_ij,
//   E_ij = exp(q_i k_j / sqrt(dh) + ln size_j - m_i),  m_i = max over S_i,
// S_i the rows of the sample that row i sees.
#include "kernels.h"

#include <algorithm>
#include <type_traits>

namespace fusion {
namespace {

// Samples of one launch: their offsets and the first row tile of each, as
// kernel arguments (a call with room for 448 took the host 1.0 to 1.5 us more).
constexpr int WIN_SEQS = 128;
struct WindowSeqs {
  int n;
  int cu[WIN_SEQS + 1];
  int tile[WIN_SEQS + 1];
};

// ------------------------------------------------------------ bf16 MFMA --
// A workgroup of 4 waves takes 32 query rows per wave: of the heads that
// share a key head as many as divide 4 at the same rows, else consecutive
// rows of one head (waves of one workgroup then read the same key tiles, and
// with shared key heads they also see the same ones).  Key tiles of 64 rows
// stream through two LDS stages by asynchronous copies, the next tile's in
// flight while the current one is computed, one barrier per tile; two
// workgroups share a CU (128-wide heads), so that one's softmax runs beside
// the other's matrix products.
//
// Scores are taken transposed, S^T = K Q^T, with v_mfma_f32_32x32x16_bf16:
// lane (hl, c) = (lane / 32, lane % 32) holds query c against keys
// 8 (i / 4) + 4 hl + i % 4, i < 16, of each 32-key half, so the row maximum
// and sum are reductions over registers and one lane swap, and the registers
// i = 8t .. 8t + 7, rounded to bf16, are the operand of the t-th step of
// O^T = V^T P^T as they stand.  (The matrix instruction takes no wider type
// beside bf16 values.  P as the sum of two bf16 numbers, half again the matrix
// work, brings the output's error against 64 bits from 0.0020 .. 0.0023 to the
// 0.0016 of its own rounding and costs 11 % of the images below, 23 % of the
// prompts and 32 % of the document, one sample of 197 rows nothing; the path's
// own attention rounds P too, so all calls do.  The sum of a row takes the
// unrounded numbers.)  V^T comes from the row-major tile by the
// transposing LDS read, with the same key order.  The running maximum moves
// only when a row's maximum grows by more than 8 in the base-2 exponent (P
// stays below 2^8, whose relative precision is that of 1), per row, so that
// no other row's values enter a row's result; rows whose maximum stays multiply by 1.
//
// LDS rows are 2 DP bytes.  K's 16-byte pieces are XOR-permuted by the row mod
// 16 (64-wide: row / 2 mod 8), V's pairs of 32-byte segments by the row mod 4
// (row / 2 mod 2): the 16-byte reads of 16 rows and the 8-byte transposing
// reads of 4 rows spread over all banks, and no read waits for another.  The
// copies write LDS in lane order, so the permutation is made in the source
// address.
//
// SPLIT: the waves share the keys of a row tile instead, 32 keys each, with a
// maximum, sum and output of their own that are joined through LDS at the end
// (4 waves a row tile of 64-wide heads, with tiles of 128 keys, 2 of wider
// ones).  share_keys says when, by the whole call: the order of a row's sums, and
// with it the last bits, is the kernel's.
//
// Measured: 16,384 rows, 16 heads of 128 over 2, window 4,096: 509 us, 950
// TFLOP/s of the pairs in the window, where a product of 8,192^3 reaches 1,070
// to 1,120; the matrix cores are busy half of the cycles and the clock falls
// under the load.  8 sequences of up to 4,096 rows, 32 heads over 8, window
// 1,024: 343 us, 747 TFLOP/s, matrix cores busy 38 %, with 18 tiles a workgroup
// between its first loads and its stores.  64 samples of up to 577 rows, 6 heads
// of 64, sizes, a two-sided window of 97: 37.3 us for 85 MB (90 read, 21
// written), bound by the vector instructions of softmax and masks and by the
// chain of 5 tiles.
//
// A probability of 0 does not take a value out of P V when that value is
// infinite or NaN.  A tile that some query of the workgroup sees and another
// does not is therefore searched for such values, and if there are any, they are
// cleared in LDS.  Rows of a workgroup that cleared values, and rows whose
// output is not finite, look through the values that they see after the last
// tile: an output with infinite or NaN ones is their sum (weights are positive,
// also one that underflowed, whose product with an infinity is NaN).
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr int WNW = 4;   // waves per workgroup

// global -> LDS copy of 16 bytes per lane (lane l's land at the wave-uniform
// LDS address + 16 l), awaited by wait_copies
__device__ __forceinline__ void copy16(const void* sbase, unsigned voff, unsigned lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1"
               :: "v"(voff), "s"(sbase), "s"(__builtin_amdgcn_readfirstlane(lds))
               : "memory", "m0");
}
__device__ __forceinline__ void copy16(const void* p, unsigned lds) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off"
               :: "v"(p), "s"(__builtin_amdgcn_readfirstlane(lds))
               : "memory", "m0");
}
__device__ __forceinline__ void wait_copies() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// What the dimensions past dh are read from when the head is not DP wide.
__device__ const uint4 kZeros = {0, 0, 0, 0};

// Whether row i of a sample sees its row j (both in the sample).
__device__ __forceinline__ bool sees(const WindowArgs& a, int i, int j) {
  if (a.causal) return j <= i && (i - j < a.window || j < a.sinks);
  return (i - j < a.window && j - i < a.window) || j < a.sinks;
}
// The rows that row i of a sample of n sees: those up to hi that are lo or
// later, or below first.
struct RowSpan {
  int lo, hi, first;
};
__device__ __forceinline__ RowSpan row_span(const WindowArgs& a, int i, int n) {
  RowSpan r;
  r.lo = max(0, i - a.window + 1);
  r.first = min(a.sinks, a.causal ? i + 1 : n);
  r.hi = max(min(n - 1, a.causal ? i : i + a.window - 1), r.first - 1);
  return r;
}

// How rows i0 .. i1 take a tile of keys j0 .. j0 + keys - 1: not at all, with
// no look at the pairs, with one at the later end or the earlier end of the
// rows' spans, or with all there is (without short cuts, so that it is one
// scalar value and the tile loop keeps its branches simple).  Tiles of which the
// rows see one half only have modes of their own (_1: the first half, _2: the
// second): with HALVES of 1 those at the ends, with 2 also those with sinks.
enum { TILE_SKIP, TILE_WHOLE, TILE_LATE, TILE_LATE_1, TILE_EARLY, TILE_EARLY_2, TILE_ALL, TILE_ALL_1 };
template <int HALVES>
__device__ __forceinline__ int tile_mode(const WindowArgs& a, int n, int i0, int i1, int j0, int keys,
                                         bool hidden) {
  const RowSpan r0 = row_span(a, i0, n), r1 = row_span(a, i1, n);
  const int j1 = j0 + keys - 1;
  const bool late = j1 > r0.hi, early = (j0 < r1.lo) & (j1 >= r0.first);
  const bool skip = (i0 >= n) | (j0 > r1.hi) | ((j1 < r0.lo) & (j0 >= r1.first));
  const bool all = hidden | (early & (late | (j0 < a.sinks)));
  const int mid = j0 + keys / 2;  // the second half's first key
  const int at_end = TILE_LATE + ((HALVES > 0) & (mid > r1.hi));
  const int at_start = TILE_EARLY + ((HALVES > 0) & (mid <= r0.lo));
  const int any = TILE_ALL + ((HALVES > 1) & ((mid > r1.hi) | ((j1 < r0.lo) & (mid >= r1.first))));
  return __builtin_amdgcn_readfirstlane(skip ? TILE_SKIP : all ? any : late ? at_end
                                        : early ? at_start : TILE_WHOLE);
}

// The query rows of a workgroup and the key tiles that any of them sees: the
// first `ns` tiles of the sample (sinks), then tiles lo .. hi.
struct WindowPlan {
  int base, n;   // the sample's first row and rows
  int q0, q1;    // first and last query row
  int ns, lo, nt;
  __device__ __forceinline__ int tile(int it) const { return it < ns ? it : lo + it - ns; }
};
// (every member is the same in all lanes, and the compiler has to know it)
__device__ __forceinline__ WindowPlan window_plan(const WindowArgs& a, const WindowSeqs& sq, int tile,
                                                  int rows, int keys) {
  int lo = 0, hi = sq.n - 1;  // the last sample whose first tile is not after this one
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (sq.tile[mid] <= tile) lo = mid; else hi = mid - 1;
  }
  WindowPlan p;
  p.base = sq.cu[lo];
  p.n = sq.cu[lo + 1] - p.base;
  p.q0 = (tile - sq.tile[lo]) * rows;
  p.q1 = min(p.q0 + rows, p.n) - 1;
  p.lo = max(0, p.q0 - a.window + 1) / keys;
  const int last = a.causal ? p.q1 : min(p.n - 1, p.q1 + a.window - 1);
  p.ns = min((min(a.sinks, p.n) + keys - 1) / keys, p.lo);
  p.nt = p.ns + last / keys - p.lo + 1;
  // sinks past the window's end (two-sided)
  if (!a.causal) p.nt = max(p.nt, p.ns + (min(a.sinks, p.n) + keys - 1) / keys - p.lo);
  return p;
}

// The place of a workgroup in the line of row tiles times head units.
// Workgroups go to the 8 XCDs in turn; with a window of at most NEAR_WINDOW
// rows, NEAR row tiles in a row go to one of them, whose L2 then reads the keys
// that they share once (64 samples of up to 577 rows, window 97: 38.6 us in
// turn, 37.0 so; 4 of 4,096 rows, 12 heads of 80 over 4, window 512: 83, 78).
// Longer windows are not bound by what they read, and under none the last rows
// of a sample see most, so that an XCD with many of them ends late (window
// 1,024: 352 us in turn, 365 so; 8 of 4,096 rows and no window: 288, 441).
constexpr int NEAR = 8, NEAR_WINDOW = 512;
__device__ __forceinline__ int place(const WindowArgs& a, int units) {
  const unsigned b = blockIdx.x, run = NEAR * units, round = 8 * run, in = b % round;
  return a.window <= NEAR_WINDOW && b - in + round <= gridDim.x ? b - in + in % 8 * run + in / 8 : b;
}

template <int DC, bool PAD, bool SIZES, bool SPLIT>
__global__ __launch_bounds__(64 * WNW, DC == 64 && !SPLIT ? 3 : 2) void window_attention_mfma(WindowArgs a, WindowSeqs sq,
                                                                     int tiles, int hshift) {
  constexpr int DP = DC <= 64 ? 64 : 128;  // dims of an LDS row; DC of them take part
  constexpr int PPR = DP / 8;             // 16-byte pieces per row
  constexpr int RPC = 64 / PPR;           // rows per copy
  constexpr int PARTS = SPLIT ? (DC == 64 ? 4 : 2) : 1;  // waves of a row tile
  constexpr int KW = SPLIT ? 32 : 64, KT = KW * PARTS;   // keys of a wave, of a tile
  constexpr int NX = KW / 32;
  constexpr int NC = KT / RPC / WNW;      // copies of K (and of V) per wave and tile
  constexpr int ROWB = DP * 2, TILEB = KT * ROWB;
  constexpr int KS = DC / 16, ND = DC / 32;
  __shared__ __attribute__((aligned(16))) char smem[4 * TILEB];  // [stage][K, V]
  __shared__ __attribute__((aligned(16))) float lnS[2][KT];
  __shared__ int s_bad, s_hidden[2][2];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int hl = lane >> 5, c = lane & 31;
  const int part = wave % PARTS, who = wave / PARTS;
  const int per_group = a.group >> hshift, units = a.H >> hshift;
  const int at = place(a, units), unit = at % units, kh = unit / per_group;
  const int h = unit % per_group * (1 << hshift) + kh * a.group + (who & ((1 << hshift) - 1));
  const WindowPlan pl = window_plan(a, sq, tiles - 1 - at / units,
                                    32 * (WNW / PARTS >> hshift), KT);
  const int n = pl.n, dh = a.dh;
  const int w0 = pl.q0 + 32 * (who >> hshift), w1 = min(w0 + 31, n - 1);
  const bf16_t* kg = (const bf16_t*)a.k + (int64_t)pl.base * a.k_row + (int64_t)kh * a.k_head;
  const bf16_t* vg = (const bf16_t*)a.v + (int64_t)pl.base * a.v_row + (int64_t)kh * a.v_head;
  const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) void*)smem;
  if (tid == 0) s_bad = -1;
  // permutations of the 16-byte pieces of K's row r and of the 32-byte segments
  // of V's: 16 pieces of 16 rows, and 4 rows of 64 bytes, cover the 256 bytes
  // of the banks
  auto k_swizzle = [](int r) { return DP == 128 ? r & 15 : r >> 1 & 7; };
  auto v_swizzle = [](int r) { return (DP == 128 ? r & 3 : r >> 1 & 1) << 1; };

  // copy of one tile: the wave's rows r = (wave NC + u) RPC + lane / PPR
  auto copy_tile = [&](int t, int st) {
    const int k0 = t * KT, lim = n - 1 - k0;
    const bf16_t* kt = kg + (int64_t)k0 * a.k_row;
    const bf16_t* vt = vg + (int64_t)k0 * a.v_row;
#pragma unroll
    for (int u = 0; u < NC; u++) {
      const int r = (wave * NC + u) * RPC + lane / PPR, rr = min(r, lim), p = lane % PPR;
      const int pk = p ^ k_swizzle(r), pv = p ^ (v_swizzle(r) << 1);
      const unsigned dst = lds0 + st * 2 * TILEB + (wave * NC + u) * 1024;
      const unsigned ko = (unsigned)rr * (unsigned)a.k_row * 2 + pk * 16;
      const unsigned vo = (unsigned)rr * (unsigned)a.v_row * 2 + pv * 16;
      if (PAD) {
        copy16(pk * 8 < dh ? (const void*)((const char*)kt + ko) : (const void*)&kZeros, dst);
        copy16(pv * 8 < dh ? (const void*)((const char*)vt + vo) : (const void*)&kZeros,
               dst + TILEB);
      } else {
        copy16(kt, ko, dst);
        copy16(vt, vo, dst + TILEB);
      }
    }
  };
  float size_next = 0.f;
  auto load_size = [&](int t) {
    if (SIZES && tid < KT) size_next = a.size[pl.base + min(t * KT + tid, n - 1)];
  };
  auto put_size = [&](int st) {
    if (SIZES && tid < KT) {
      lnS[st][tid] = size_next > 0.f ? logf(size_next) * kLog2e : -INFINITY;
      const bool hidden = __any(!(size_next > 0.f));
      if (lane == 0) s_hidden[st][wave] = hidden;
    }
  };
  copy_tile(pl.tile(0), 0);
  load_size(pl.tile(0));

  // Q^T operand: lane holds Q[w0 + c][16 s + 8 hl .. + 7]
  bf16x8_t qf[KS];
  {
    const bf16_t* qr = (const bf16_t*)a.q + (int64_t)(pl.base + min(w0 + c, n - 1)) * a.q_row +
                       (int64_t)h * a.q_head;
#pragma unroll
    for (int s = 0; s < KS; s++) {
      uint4 v = make_uint4(0, 0, 0, 0);
      if (!PAD || 16 * s + 8 * hl < dh) v = *(const uint4*)(qr + 16 * s + 8 * hl);
      qf[s] = __builtin_bit_cast(bf16x8_t, v);
    }
  }
  put_size(0);
  const float sc2 = a.scale * kLog2e;
  float m = -INFINITY, l = 0.f;
  const RowSpan sp = row_span(a, w0 + c, n);
  bool any_bad = false;
  f32x16_t O[ND];
#pragma unroll
  for (int d = 0; d < ND; d++)
#pragma unroll
    for (int i = 0; i < 16; i++) O[d][i] = 0.f;

  // LDS addresses of the operands: K row c of a half, V rows of a 16-lane group
  const int krow = c * ROWB, kx = k_swizzle(c);
  const int vkey = (lane & 15) >> 2;
  const int vcol = ((lane >> 4) & 1) * 32 + (lane & 3) * 8;  // bytes within a 64-byte dim tile
  int it = 0, st = 0, k0 = 0;  // the tile in hand: its number, LDS stage and first key
  bool hidden = false;         // some key of it has no size
  // waits for tile `it`, starts the next one's copies, clears what no product
  // may meet; returns how the wave takes it
  auto begin = [&]() {
    st = it & 1;
    k0 = pl.tile(it) * KT;
    wait_copies();
    __syncthreads();
    if (it + 1 < pl.nt) {
      copy_tile(pl.tile(it + 1), st ^ 1);
      load_size(pl.tile(it + 1));
    }
    hidden = SIZES && __builtin_amdgcn_readfirstlane(s_hidden[st][0] | (KT > 64 ? s_hidden[st][1] : 0));
    if (tile_mode<0>(a, n, pl.q0, pl.q1, k0, KT, hidden) > TILE_WHOLE) {
      char* Vs = smem + st * 2 * TILEB + TILEB;
      uint32_t any = 0;
#pragma unroll
      for (int u = 0; u < TILEB / (64 * WNW * 16); u++) {
        const uint4 v = *(const uint4*)(Vs + (tid + u * 64 * WNW) * 16);
        any |= ((v.x & 0x7F807F80u) + 0x00800080u) | ((v.y & 0x7F807F80u) + 0x00800080u) |
               ((v.z & 0x7F807F80u) + 0x00800080u) | ((v.w & 0x7F807F80u) + 0x00800080u);
      }
      if (any & 0x80008000u) s_bad = it;
      __syncthreads();
      if (__builtin_amdgcn_readfirstlane(s_bad) == it) {
        for (int u = tid; u < TILEB / 2; u += 64 * WNW) {
          bf16_t* v = (bf16_t*)Vs + u;
          if ((*v & 0x7F80) == 0x7F80) *v = 0;
        }
        any_bad = true;
        __syncthreads();
      }
    }
    return tile_mode<(NX > 1)>(a, n, w0, w1, k0 + part * KW, KW, hidden);
  };
  // the next tile's mode, or -1 after the last
  auto next = [&]() {
    if (it + 1 < pl.nt) put_size(st ^ 1);
    return ++it < pl.nt ? begin() : -1;
  };
  auto compute = [&](auto mode_c) {
    constexpr int MODE = decltype(mode_c)::value;
    constexpr bool LATE = MODE == TILE_LATE || MODE == TILE_LATE_1;
    constexpr bool EARLY = MODE == TILE_EARLY || MODE == TILE_EARLY_2;
    constexpr int X0 = MODE == TILE_EARLY_2, X1 = MODE == TILE_LATE_1 ? 1 : NX;  // halves
    const char* Ks = smem + st * 2 * TILEB + part * KW * ROWB;
    const char* Vs = Ks + TILEB;
    f32x16_t S[NX];
#pragma unroll
    for (int x = X0; x < X1; x++) {
#pragma unroll
      for (int i = 0; i < 16; i++) S[x][i] = 0.f;
#pragma unroll
      for (int s = 0; s < KS; s++) {
        const bf16x8_t kf = *(const bf16x8_t*)(Ks + x * 32 * ROWB + krow + (((2 * s + hl) ^ kx) << 4));
        S[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[s], S[x], 0, 0, 0);
      }
    }
    // with sizes the scores of base 2; -inf for keys that the query does not see
    if (SIZES) {
#pragma unroll
      for (int x = X0; x < X1; x++)
#pragma unroll
        for (int i4 = 0; i4 < 4; i4++) {
          const f32x4_t ln = *(const f32x4_t*)(&lnS[st][part * KW + x * 32 + 8 * i4 + 4 * hl]);
#pragma unroll
          for (int j = 0; j < 4; j++) S[x][4 * i4 + j] = fmaf(S[x][4 * i4 + j], sc2, ln[j]);
        }
      if (MODE == TILE_ALL && hidden)
#pragma unroll
        for (int x = X0; x < X1; x++)
#pragma unroll
          for (int i = 0; i < 16; i++)
            if (lnS[st][part * KW + x * 32 + 8 * (i / 4) + 4 * hl + i % 4] == -INFINITY) S[x][i] = -INFINITY;
    }
    const int kp = k0 + part * KW + 4 * hl, lo = sp.lo - kp, hi = sp.hi - kp, first = sp.first - kp;
#pragma unroll
    for (int x = X0; x < X1; x++)
#pragma unroll
      for (int i = 0; i < 16; i++) {
        const int key = x * 32 + 8 * (i / 4) + i % 4;
        if (LATE) S[x][i] = key <= hi ? S[x][i] : -INFINITY;
        if (EARLY) S[x][i] = key >= lo ? S[x][i] : -INFINITY;
        if (MODE == TILE_ALL) S[x][i] = (key <= hi) & ((key >= lo) | (key < first)) ? S[x][i] : -INFINITY;
      }
    float mt = -INFINITY;
#pragma unroll
    for (int x = X0; x < X1; x++)
#pragma unroll
      for (int i = 0; i < 16; i++) mt = fmaxf(mt, S[x][i]);
    mt = max_xor32(mt);
    if (!SIZES) mt *= sc2;
    const bool grow = mt > m + 8.f;
    if (__any(grow)) {
      const float f = grow ? __builtin_amdgcn_exp2f(m - mt) : 1.f;
      if (grow) m = mt;
      l *= f;
#pragma unroll
      for (int d = 0; d < ND; d++)
#pragma unroll
        for (int i = 0; i < 16; i++) O[d][i] *= f;
    }
    const float mu = m == -INFINITY ? 0.f : m;
    bf16x8_t pf[2 * NX];
    float lt[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int x = X0; x < X1; x++)
#pragma unroll
      for (int y = 0; y < 2; y++) {
        union { uint32_t u[4]; bf16x8_t v; } p;
#pragma unroll
        for (int w = 0; w < 4; w++) {
          const float s0 = S[x][8 * y + 2 * w], s1 = S[x][8 * y + 2 * w + 1];
          const float e0 = __builtin_amdgcn_exp2f(SIZES ? s0 - mu : fmaf(s0, sc2, -mu));
          const float e1 = __builtin_amdgcn_exp2f(SIZES ? s1 - mu : fmaf(s1, sc2, -mu));
          lt[w] += e0 + e1;
          p.u[w] = pack_bf16x2(e0, e1);
        }
        pf[2 * x + y] = p.v;
      }
    l += (lt[0] + lt[1]) + (lt[2] + lt[3]);
#pragma unroll
    for (int y = 2 * X0; y < 2 * X1; y++)
#pragma unroll
      for (int d = 0; d < ND; d++) {
        union { s16x4_t h[2]; bf16x8_t v; } vf;
#pragma unroll
        for (int z = 0; z < 2; z++) {
          const int key = 16 * y + 8 * z + 4 * hl + vkey;  // key % 4 == vkey
          const int seg = (d * 2 + (vcol >> 5)) ^ v_swizzle(vkey);
          vf.h[z] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              (__attribute__((address_space(3))) s16x4_t*)(Vs + key * ROWB + seg * 32 + (vcol & 31)));
        }
        O[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf.v, pf[y], O[d], 0, 0, 0);
      }
  };
  // (a loop for each mode, since tiles of one come in runs: with one loop over
  // both copies of the code the output moved between registers in every tile)
  int mode = begin();
  while (mode >= 0) {
    while (mode == TILE_WHOLE) {
      compute(std::integral_constant<int, TILE_WHOLE>{});
      mode = next();
    }
    while (mode == TILE_LATE) {
      compute(std::integral_constant<int, TILE_LATE>{});
      mode = next();
    }
    while (mode == TILE_EARLY) {
      compute(std::integral_constant<int, TILE_EARLY>{});
      mode = next();
    }
    if constexpr (NX > 1) {
      while (mode == TILE_LATE_1) {
        compute(std::integral_constant<int, TILE_LATE_1>{});
        mode = next();
      }
      while (mode == TILE_EARLY_2) {
        compute(std::integral_constant<int, TILE_EARLY_2>{});
        mode = next();
      }
    }
    while (mode == TILE_ALL) {
      compute(std::integral_constant<int, TILE_ALL>{});
      mode = next();
    }
    while (mode == TILE_SKIP) mode = next();
  }
  if constexpr (SPLIT) {  // the parts of a row tile joined, by the first of its waves
    __syncthreads();
    constexpr int OTHERS = PARTS - 1;
    float* Os = (float*)smem + lane;
    float2* ml = (float2*)(smem + WNW / PARTS * OTHERS * ND * 4096) + lane;
    if (part > 0) {
      const int to = who * OTHERS + part - 1;
#pragma unroll
      for (int d = 0; d < ND; d++)
#pragma unroll
        for (int i = 0; i < 16; i++) Os[((to * ND + d) * 16 + i) * 64] = O[d][i];
      ml[to * 64] = make_float2(m, l);
    }
    __syncthreads();
    if (part > 0) return;
    float top = m;
#pragma unroll
    for (int p = 0; p < OTHERS; p++) top = fmaxf(top, ml[(who * OTHERS + p) * 64].x);
    const float mu = top == -INFINITY ? 0.f : top, f0 = __builtin_amdgcn_exp2f(m - mu);
    l *= f0;
#pragma unroll
    for (int d = 0; d < ND; d++)
#pragma unroll
      for (int i = 0; i < 16; i++) O[d][i] *= f0;
#pragma unroll
    for (int p = 0; p < OTHERS; p++) {
      const int of = who * OTHERS + p;
      const float f = __builtin_amdgcn_exp2f(ml[of * 64].x - mu);
      l = fmaf(ml[of * 64].y, f, l);
#pragma unroll
      for (int d = 0; d < ND; d++)
#pragma unroll
        for (int i = 0; i < 16; i++) O[d][i] = fmaf(Os[((of * ND + d) * 16 + i) * 64], f, O[d][i]);
    }
  }
  l = sum_xor32(l);
  // rows that see infinite or NaN values get their sum
  float zero[4] = {0.f, 0.f, 0.f, 0.f};  // NaN where an output is not finite
#pragma unroll
  for (int d = 0; d < ND; d++)
#pragma unroll
    for (int i = 0; i < 16; i++) zero[i & 3] = fmaf(O[d][i], 0.f, zero[i & 3]);
  const bool odd = any_bad | ((zero[0] + zero[1]) + (zero[2] + zero[3]) != 0.f);
  if (odd && l == l && w0 + c < n) {  // (a NaN score makes all of a row NaN)
    float sum[ND][16] = {};
    for (int it = 0; it < pl.nt; it++)
      for (int j = pl.tile(it) * KT; j < min(n, pl.tile(it) * KT + KT); j++) {
        if (!sees(a, w0 + c, j) || (SIZES && !(a.size[pl.base + j] > 0.f))) continue;
        const bf16_t* v = vg + (int64_t)j * a.v_row + 4 * hl;
#pragma unroll
        for (int d = 0; d < ND; d++)
#pragma unroll
          for (int i4 = 0; i4 < 4; i4++) {
            if (PAD && 32 * d + 8 * i4 >= dh) break;
            const uint2 x = *(const uint2*)(v + 32 * d + 8 * i4);
            const float e[4] = {__uint_as_float(x.x << 16), __uint_as_float(x.x & 0xFFFF0000u),
                                __uint_as_float(x.y << 16), __uint_as_float(x.y & 0xFFFF0000u)};
#pragma unroll
            for (int q = 0; q < 4; q++) sum[d][4 * i4 + q] += fabsf(e[q]) < INFINITY ? 0.f : e[q];
          }
      }
#pragma unroll
    for (int d = 0; d < ND; d++)
#pragma unroll
      for (int i = 0; i < 16; i++) O[d][i] = sum[d][i] == 0.f ? O[d][i] : sum[d][i];
  }
  if (w0 + c < n) {
    const float r = l == 0.f ? 0.f : 1.f / l;
    bf16_t* out = (bf16_t*)a.out + ((int64_t)(pl.base + w0 + c) * a.H + h) * dh + 4 * hl;
#pragma unroll
    for (int d = 0; d < ND; d++)
#pragma unroll
      for (int i4 = 0; i4 < 4; i4++)
        if (!PAD || 32 * d + 8 * i4 < dh)
          *(uint2*)(out + 32 * d + 8 * i4) =
              make_uint2(pack_bf16x2(O[d][4 * i4] * r, O[d][4 * i4 + 1] * r),
                         pack_bf16x2(O[d][4 * i4 + 2] * r, O[d][4 * i4 + 3] * r));
  }
}

// ------------------------------------------------------------ fp32 MFMA --
// The same plan with v_mfma_f32_16x16x4_f32, 16 query rows per wave, bound by
// the fp32 matrix rate.  Lane (g, c) = (lane / 16, lane % 16) holds query c
// against keys 16 t + 4 g + j, and these registers are the operand of
// O^T = V^T P^T as they stand (slot g of step j is key 16 t + 4 g + j).  A
// 16-byte piece of a key feeds four steps (slot g of step i is dim
// 16 u + 4 g + i).  Tiles are 8 KB of keys and as much of values (with 16 KB a
// window of 130 took 51 us instead of 37, since more of a tile lies outside,
// and one of 4,096 took 491 instead of 502); K's pieces are XOR-permuted by
// the row mod 16, V's groups of four pieces by row / 4 mod 4, so that the
// 16-byte key reads of 16 rows and the 4-byte value reads of 4 x 16 spread over
// all banks.  8 sequences of up to 1,031 rows, 12 heads of 64, window 130, 1.76
// GFLOP in the window: 40.5 us (42.2 with whole tiles only, which made 2.69 of
// them; with a window of 4,096 the loops for parts of a tile cost 1 %).
//
// SPLIT: the waves share the keys of a row tile instead, 16 keys each of tiles
// of twice the size, with a maximum, sum and output of their own that are
// joined through LDS at the end (4 waves a row tile of 64-wide heads, 2 of
// wider ones).  share_keys says when.
template <int DC, bool PAD, bool SIZES, bool SPLIT>
__global__ __launch_bounds__(64 * WNW, 2) void window_attention_mfma_f32(WindowArgs a, WindowSeqs sq,
                                                                         int tiles, int hshift) {
  constexpr int DP = DC <= 64 ? 64 : 128;
  constexpr int PPR = DP / 4, RPC = 64 / PPR;  // pieces per row, rows per copy
  constexpr int TILEB = SPLIT ? 16384 : 8192, ROWB = DP * 4, KT = TILEB / ROWB;
  constexpr int PARTS = SPLIT ? KT / 16 : 1, KW = KT / PARTS;  // waves of a row tile, keys of each
  constexpr int NC = KT / RPC / WNW, NT = KW / 16, NU = DC / 16;
  __shared__ __attribute__((aligned(16))) char smem[4 * TILEB];  // [stage][K, V]
  __shared__ __attribute__((aligned(16))) float lnS[2][KT];
  __shared__ int s_bad, s_hidden[2];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int g = lane >> 4, c = lane & 15;
  const int part = wave % PARTS, who = wave / PARTS;
  const int per_group = a.group >> hshift, units = a.H >> hshift;
  const int at = place(a, units), unit = at % units, kh = unit / per_group;
  const int h = unit % per_group * (1 << hshift) + kh * a.group + (who & ((1 << hshift) - 1));
  const WindowPlan pl = window_plan(a, sq, tiles - 1 - at / units, 16 * (WNW / PARTS >> hshift), KT);
  const int n = pl.n, dh = a.dh;
  const int w0 = pl.q0 + 16 * (who >> hshift), w1 = min(w0 + 15, n - 1);
  const float* kg = (const float*)a.k + (int64_t)pl.base * a.k_row + (int64_t)kh * a.k_head;
  const float* vg = (const float*)a.v + (int64_t)pl.base * a.v_row + (int64_t)kh * a.v_head;
  const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) void*)smem;
  if (tid == 0) s_bad = -1;

  auto copy_tile = [&](int t, int st) {
    const int k0 = t * KT, lim = n - 1 - k0;
    const float* kt = kg + (int64_t)k0 * a.k_row;
    const float* vt = vg + (int64_t)k0 * a.v_row;
#pragma unroll
    for (int u = 0; u < NC; u++) {
      const int r = (wave * NC + u) * RPC + lane / PPR, rr = min(r, lim), p = lane % PPR;
      const int pk = p ^ (r & 15), pv = p ^ ((r >> 2 & 3) << 2);
      const unsigned dst = lds0 + st * 2 * TILEB + (wave * NC + u) * 1024;
      const unsigned ko = (unsigned)rr * (unsigned)a.k_row * 4 + pk * 16;
      const unsigned vo = (unsigned)rr * (unsigned)a.v_row * 4 + pv * 16;
      if (PAD) {
        copy16(pk * 4 < dh ? (const void*)((const char*)kt + ko) : (const void*)&kZeros, dst);
        copy16(pv * 4 < dh ? (const void*)((const char*)vt + vo) : (const void*)&kZeros,
               dst + TILEB);
      } else {
        copy16(kt, ko, dst);
        copy16(vt, vo, dst + TILEB);
      }
    }
  };
  float size_next = 0.f;
  auto load_size = [&](int t) {
    if (SIZES && tid < KT) size_next = a.size[pl.base + min(t * KT + tid, n - 1)];
  };
  auto put_size = [&](int st) {
    if (SIZES && tid < KT) {
      lnS[st][tid] = size_next > 0.f ? logf(size_next) * kLog2e : -INFINITY;
      const bool hidden = __any(!(size_next > 0.f));
      if (tid == 0) s_hidden[st] = hidden;
    }
  };
  copy_tile(pl.tile(0), 0);
  load_size(pl.tile(0));

  f32x4_t qf[NU];
  {
    const float* qr = (const float*)a.q + (int64_t)(pl.base + min(w0 + c, n - 1)) * a.q_row +
                      (int64_t)h * a.q_head;
#pragma unroll
    for (int u = 0; u < NU; u++) {
      qf[u] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      if (!PAD || 16 * u + 4 * g < dh) qf[u] = *(const f32x4_t*)(qr + 16 * u + 4 * g);
    }
  }
  put_size(0);
  const float sc2 = a.scale * kLog2e;
  float m = -INFINITY, l = 0.f;
  const RowSpan sp = row_span(a, w0 + c, n);
  bool any_bad = false;
  f32x4_t O[NU];
#pragma unroll
  for (int d = 0; d < NU; d++) O[d] = f32x4_t{0.f, 0.f, 0.f, 0.f};

  int it = 0, st = 0, k0 = 0;  // the tile in hand: its number, LDS stage and first key
  bool hidden = false;         // some key of it has no size
  int mode = 0;                // how the wave takes it, or -1 after the last
  auto begin = [&]() {
    st = it & 1;
    k0 = pl.tile(it) * KT;
    wait_copies();
    __syncthreads();
    if (it + 1 < pl.nt) {
      copy_tile(pl.tile(it + 1), st ^ 1);
      load_size(pl.tile(it + 1));
    }
    char* Vs = smem + st * 2 * TILEB + TILEB;
    bool bad = false;
    hidden = SIZES && __builtin_amdgcn_readfirstlane(s_hidden[st]);
    if (tile_mode<0>(a, n, pl.q0, pl.q1, k0, KT, hidden) > TILE_WHOLE) {
      bool any = false;
#pragma unroll
      for (int u = 0; u < TILEB / (64 * WNW * 16); u++) {
        const f32x4_t v = *(const f32x4_t*)(Vs + (tid + u * 64 * WNW) * 16);
        any |= !(fabsf(v[0]) < INFINITY) | !(fabsf(v[1]) < INFINITY) | !(fabsf(v[2]) < INFINITY) |
               !(fabsf(v[3]) < INFINITY);
      }
      if (any) s_bad = it;
      __syncthreads();
      bad = __builtin_amdgcn_readfirstlane(s_bad) == it;
    }
    if (bad) {
      for (int u = tid; u < TILEB / 4; u += 64 * WNW) {
        float* v = (float*)Vs + u;
        if (!(fabsf(*v) < INFINITY)) *v = 0.f;
      }
      any_bad = true;
      __syncthreads();
    }
    mode = tile_mode<(NT > 1 ? 2 : 0)>(a, n, w0, w1, k0 + part * KW, KW, hidden);
  };
  auto next = [&]() {
    if (it + 1 < pl.nt) put_size(st ^ 1);
    if (++it < pl.nt) begin(); else mode = -1;
  };
  // 16-key parts X0 .. X1 - 1; EDGES: some may be unseen
  auto compute = [&](auto x0_c, auto x1_c, auto edges_c) {
    constexpr int X0 = decltype(x0_c)::value, X1 = decltype(x1_c)::value;
    constexpr bool EDGES = decltype(edges_c)::value;
    const char* Ks = smem + st * 2 * TILEB + part * KW * ROWB;
    const char* Vs = Ks + TILEB;
    const int kp = k0 + part * KW;
    f32x4_t S[NT];
#pragma unroll
    for (int x = X0; x < X1; x++) S[x] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int u = 0; u < NU; u++) {
      f32x4_t kf[NT];
#pragma unroll
      for (int x = X0; x < X1; x++)
        kf[x] = *(const f32x4_t*)(Ks + (16 * x + c) * ROWB + (((4 * u + g) ^ c) << 4));
#pragma unroll
      for (int i = 0; i < 4; i++)
#pragma unroll
        for (int x = X0; x < X1; x++)
          S[x] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[x][i], qf[u][i], S[x], 0, 0, 0);
    }
#pragma unroll
    for (int x = X0; x < X1; x++) {
      f32x4_t ln = {0.f, 0.f, 0.f, 0.f};
      if (SIZES) ln = *(const f32x4_t*)(&lnS[st][part * KW + 16 * x + 4 * g]);
#pragma unroll
      for (int j = 0; j < 4; j++) {
        S[x][j] = fmaf(S[x][j], sc2, ln[j]);
        if (EDGES && hidden && ln[j] == -INFINITY) S[x][j] = -INFINITY;
      }
    }
    if (EDGES && mode > TILE_WHOLE) {
      const int lo = sp.lo - kp - 4 * g, hi = sp.hi - kp - 4 * g, first = sp.first - kp - 4 * g;
#pragma unroll
      for (int x = X0; x < X1; x++)
#pragma unroll
        for (int j = 0; j < 4; j++) {
          const int key = 16 * x + j;
          S[x][j] = (key <= hi) & ((key >= lo) | (key < first)) ? S[x][j] : -INFINITY;
        }
    }
    float mt = -INFINITY;
#pragma unroll
    for (int x = X0; x < X1; x++)
#pragma unroll
      for (int j = 0; j < 4; j++) mt = fmaxf(mt, S[x][j]);
    mt = max_xor32(max_xor16(mt));
    const bool grow = mt > m + 8.f;
    if (__any(grow)) {
      const float f = grow ? __builtin_amdgcn_exp2f(m - mt) : 1.f;
      if (grow) m = mt;
      l *= f;
#pragma unroll
      for (int d = 0; d < NU; d++)
#pragma unroll
        for (int j = 0; j < 4; j++) O[d][j] *= f;
    }
    const float mu = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int x = X0; x < X1; x++) {
#pragma unroll
      for (int j = 0; j < 4; j++) S[x][j] = __builtin_amdgcn_exp2f(S[x][j] - mu);
      l += (S[x][0] + S[x][1]) + (S[x][2] + S[x][3]);
    }
#pragma unroll
    for (int x = X0; x < X1; x++)
#pragma unroll
      for (int j = 0; j < 4; j++) {
        const char* vr = Vs + (16 * x + 4 * g + j) * ROWB + (c & 3) * 4;
#pragma unroll
        for (int d = 0; d < NU; d++)
          O[d] = __builtin_amdgcn_mfma_f32_16x16x4f32(
              *(const float*)(vr + (((4 * d + (c >> 2)) ^ (g << 2)) << 4)), S[x][j], O[d], 0, 0, 0);
      }
  };
  // (a loop for each set of parts, as above; where there is one set, one loop
  // takes 126 registers, with which 4 waves share a SIMD, and two take 163)
  constexpr std::integral_constant<int, 0> none;
  constexpr std::integral_constant<int, NT / 2> half;
  constexpr std::integral_constant<int, NT> whole;
  begin();
  if constexpr (NT > 1) {
    while (mode >= 0) {
      while (mode == TILE_LATE_1 || mode == TILE_ALL_1) {
        compute(none, half, std::true_type{});
        next();
      }
      while (mode == TILE_EARLY_2) {
        compute(half, whole, std::true_type{});
        next();
      }
      while (mode == TILE_LATE || mode == TILE_EARLY || mode == TILE_ALL) {
        compute(none, whole, std::true_type{});
        next();
      }
      while (mode == TILE_WHOLE) {
        compute(none, whole, std::false_type{});
        next();
      }
      while (mode == TILE_SKIP) next();
    }
  } else {
    while (mode >= 0) {
      if (mode != TILE_SKIP) compute(none, whole, std::true_type{});
      next();
    }
  }
  if constexpr (SPLIT) {  // the parts of a row tile joined, by the first of its waves
    __syncthreads();
    f32x4_t* Os = (f32x4_t*)smem + lane;
    float2* ml = (float2*)(smem + WNW * NU * 1024) + lane;
#pragma unroll
    for (int d = 0; d < NU; d++) Os[(wave * NU + d) * 64] = O[d];
    ml[wave * 64] = make_float2(m, l);
    __syncthreads();
    if (part != 0) return;
    float top = m;
#pragma unroll
    for (int p = 1; p < PARTS; p++) top = fmaxf(top, ml[(wave + p) * 64].x);
    const float mu = top == -INFINITY ? 0.f : top, f0 = __builtin_amdgcn_exp2f(m - mu);
    l *= f0;
#pragma unroll
    for (int d = 0; d < NU; d++) O[d] *= f0;
#pragma unroll
    for (int p = 1; p < PARTS; p++) {
      const float2 x = ml[(wave + p) * 64];
      const float f = __builtin_amdgcn_exp2f(x.x - mu);
      l = fmaf(x.y, f, l);
#pragma unroll
      for (int d = 0; d < NU; d++) O[d] += Os[((wave + p) * NU + d) * 64] * f;
    }
  }
  l = sum_xor32(sum_xor16(l));
  // rows that see infinite or NaN values get their sum
  f32x4_t zero = {0.f, 0.f, 0.f, 0.f};  // NaN where an output is not finite
#pragma unroll
  for (int d = 0; d < NU; d++)
#pragma unroll
    for (int q = 0; q < 4; q++) zero[q] = fmaf(O[d][q], 0.f, zero[q]);
  const bool odd = any_bad | ((zero[0] + zero[1]) + (zero[2] + zero[3]) != 0.f);
  if (odd && l == l && w0 + c < n) {  // (a NaN score makes all of a row NaN)
    f32x4_t sum[NU];
#pragma unroll
    for (int d = 0; d < NU; d++) sum[d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    for (int it = 0; it < pl.nt; it++)
      for (int j = pl.tile(it) * KT; j < min(n, pl.tile(it) * KT + KT); j++) {
        if (!sees(a, w0 + c, j) || (SIZES && !(a.size[pl.base + j] > 0.f))) continue;
        const float* v = vg + (int64_t)j * a.v_row + 4 * g;
#pragma unroll
        for (int d = 0; d < NU; d++) {
          if (PAD && 16 * d + 4 * g >= dh) break;
          const f32x4_t x = *(const f32x4_t*)(v + 16 * d);
#pragma unroll
          for (int q = 0; q < 4; q++) sum[d][q] += fabsf(x[q]) < INFINITY ? 0.f : x[q];
        }
      }
#pragma unroll
    for (int d = 0; d < NU; d++)
#pragma unroll
      for (int q = 0; q < 4; q++) O[d][q] = sum[d][q] == 0.f ? O[d][q] : sum[d][q];
  }
  if (w0 + c < n) {
    const float r = l == 0.f ? 0.f : 1.f / l;
    float* out = (float*)a.out + ((int64_t)(pl.base + w0 + c) * a.H + h) * dh + 4 * g;
#pragma unroll
    for (int d = 0; d < NU; d++)
      if (!PAD || 16 * d + 4 * g < dh) *(f32x4_t*)(out + 16 * d) = O[d] * r;
  }
}

// Runs `launch(samples, tiles, grid)` for all samples, as many at once as the
// arguments of a launch hold, with tiles of `rows` rows and `units` workgroups a
// tile, from the last tile back (workgroup 0 has tile tiles - 1).
template <typename F>
hipError_t for_samples(const int32_t* cu_host, int batch, int rows, int units, F launch) {
  constexpr int MOST = (1 << 30) / (64 * WNW);  // workgroups a launch; it holds less than 2^32 threads
  for (int f = 0; f < batch; f += WIN_SEQS) {
    WindowSeqs sq;
    sq.n = std::min(batch - f, WIN_SEQS);
    int tiles = 0;
    for (int i = 0; i <= sq.n; i++) {
      sq.cu[i] = cu_host[f + i];
      sq.tile[i] = tiles;
      if (i < sq.n) tiles += (cu_host[f + i + 1] - cu_host[f + i] + rows - 1) / rows;
    }
    for (int m; tiles > 0; tiles -= m) {
      m = std::min(tiles, MOST / units);
      launch(sq, tiles, (unsigned)(m * units));
      if (hipError_t e = hipGetLastError()) return e;
    }
  }
  return hipSuccess;
}

// Whether the waves of a workgroup share the keys of its row tiles, `parts` waves
// a tile, instead of having a row tile each: where that many more workgroups
// still run at once (2 a CU: groups x parts <= 512), or where hardly a window
// evens the rows out and the last rows' chains of tiles are what the call takes:
// a chain is longest / (keys of a tile) tiles, which sharing divides by `parts`,
// and what it costs is the work of workgroups that no longer run at once, groups
// x min(window, longest).  The second rule's two factors are set by the points
// below, on whose sides of it they lie, and by nothing else.  One sample, causal
// (row tiles each / shared, us; in brackets the workgroups without sharing):
//   fp32: 512 rows, 16 heads of 128, window 300 [128] 40 / 25; 1,536, 6 of 64,
//     964 [144] 59 / 31; 4,096, 6 of 64, none [384] 234 / 160; but 2,048, 6 of
//     64, 200 [192] 21 / 26 and 5,120, 1,000 [480] 94 / 109
//   bf16: 1,024, 16 of 128, none [128] 27 / 21; 4,096, 6 of 64, none [192] 69 /
//     36; 8,192 [384] 139 / 118; but 16,384 [768] 310 / 420, 4,096, 400 [192]
//     16.6 / 21, 8,192, 4,096 [384] 81 / 98 and 6 samples of 900 [288] 21 / 23
bool share_keys(const WindowArgs& a, const int32_t* cu_host, int batch, int rows, int units,
                int parts) {
  int64_t groups = 0, longest = 0;
  for (int i = 0; i < batch; i++) {
    const int64_t n = cu_host[i + 1] - cu_host[i];
    groups += (n + rows - 1) / rows;
    longest = std::max(longest, n);
  }
  groups *= units;
  return groups * parts <= 512 || (a.causal && longest >= 5 * groups &&
                                   groups * longest <= 400 * std::min((int64_t)a.window, longest));
}

template <typename T, int DC, bool PAD>
hipError_t launch_mfma(const WindowArgs& a, const int32_t* cu_host, int batch, hipStream_t s) {
  // heads of a group per workgroup, 1 << hshift
  const int hshift = a.group % 4 == 0 ? 2 : a.group % 2 == 0 ? 1 : 0;
  const int rows = (sizeof(T) == 2 ? 32 : 16) * (WNW >> hshift);
  const auto run = [&](auto split_c, int rows, int hshift) {
    constexpr bool SPLIT = decltype(split_c)::value;
    const int units = a.H >> hshift;
    return for_samples(cu_host, batch, rows, units, [&](const WindowSeqs& sq, int tiles, unsigned grid) {
      if constexpr (sizeof(T) == 2) {
        if (a.size)
          window_attention_mfma<DC, PAD, true, SPLIT><<<grid, 64 * WNW, 0, s>>>(a, sq, tiles, hshift);
        else
          window_attention_mfma<DC, PAD, false, SPLIT><<<grid, 64 * WNW, 0, s>>>(a, sq, tiles, hshift);
      } else {
        if (a.size)
          window_attention_mfma_f32<DC, PAD, true, SPLIT><<<grid, 64 * WNW, 0, s>>>(a, sq, tiles, hshift);
        else
          window_attention_mfma_f32<DC, PAD, false, SPLIT><<<grid, 64 * WNW, 0, s>>>(a, sq, tiles, hshift);
      }
    });
  };
  constexpr int parts = DC <= 64 ? 4 : 2;
  return share_keys(a, cu_host, batch, rows, a.H >> hshift, parts)
             ? run(std::true_type{}, (rows << hshift) / parts, 0)
             : run(std::false_type{}, rows, hshift);
}

}  // namespace

template <typename T>
hipError_t launch_window_attention(const WindowArgs& a, const int32_t* cu_host, int batch,
                                   hipStream_t s) {
  // (dims are taken in 64, 96 or 128, the rest of them zeros)
  if (a.dh == 64) return launch_mfma<T, 64, false>(a, cu_host, batch, s);
  if (a.dh < 64) return launch_mfma<T, 64, true>(a, cu_host, batch, s);
  if (a.dh <= 96) return launch_mfma<T, 96, true>(a, cu_host, batch, s);
  if (a.dh < 128) return launch_mfma<T, 128, true>(a, cu_host, batch, s);
  return launch_mfma<T, 128, false>(a, cu_host, batch, s);
}
template hipError_t launch_window_attention<float>(const WindowArgs&, const int32_t*, int,
                                                   hipStream_t);
template hipError_t launch_window_attention<bf16_t>(const WindowArgs&, const int32_t*, int,
                                                    hipStream_t);

}  // namespace fusion
