// Attention of one new token per sequence over a paged cache: the kernels, for
// caches of bf16, fp32 and 4 bits, over all tokens or chosen pages, and what
// launches them.
#pragma once
#include "kernels.h"

#include <algorithm>
#include <type_traits>

namespace fusion {
namespace {

inline size_t round256(size_t v) { return (v + 255) & ~(size_t)255; }

// Page of a sequence's slot, or -1 where the table holds none.
__device__ __forceinline__ int page_of(const CacheArgs& c, int b, uint32_t pg) {
  const int p = c.table[(int64_t)b * c.max_pages + pg];
  return (unsigned)p < (unsigned)c.pages ? p : -1;
}
__device__ __forceinline__ int held(const CacheArgs& c, int b) {
  return max(0, min(c.len[b], c.cap));
}

// Inclusive sum over the lanes of a wave, by DPP shifts within rows of 16 and
// the two row broadcasts.
__device__ __forceinline__ int wave_scan(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);  // row_shr 1
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);  // row_shr 2
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);  // row_shr 4
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);  // row_shr 8
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);  // row_bcast 15
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);  // row_bcast 31
  return v;
}

// Eight neighbouring values of a row.
template <typename T>
__device__ __forceinline__ void load8(const T* p, float* x) {
  if constexpr (sizeof(T) == 2) {
    const uint4 u = *(const uint4*)p;
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; i++) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  } else {
    const float4 a = *(const float4*)p, b = *(const float4*)(p + 4);
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
    x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
  }
}
template <typename T>
__device__ __forceinline__ void store8(T* p, const float* x) {
  if constexpr (sizeof(T) == 2) {
    *(uint4*)p = make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]),
                            pack_bf16x2(x[6], x[7]));
  } else {
    *(float4*)p = make_float4(x[0], x[1], x[2], x[3]);
    *(float4*)(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
  }
}

// Offsets of the samples of one launch as kernel arguments.
constexpr int APPEND_SEQS = 256;
struct AppendSeqs {
  int n, first;  // samples, the first one's index
  int cu[APPEND_SEQS + 1];
};
struct OneRowEach {};
constexpr int APPEND_FEW = 8;  // rows of a sample up to which one workgroup takes them
constexpr int APPEND_BLOCKS = 1 << 22;  // workgroups of a launch (2^32 threads are too many for one)

// ------------------------------------------------------ paged attention --
// One new token per sequence: bound by the bytes of the visible keys and
// values, which are read once.  The visible tokens of a sequence form tiles of
// KT (32 bf16, 16 fp32: 16 KB of keys and values at 128-wide heads), the tiles
// of all sequences one line, and the waves of a unit (a key head and up to 16
// of its query heads) take equal parts of that line, wherever sequences begin
// and end; a wave is on its own, with no barrier, and the 4 waves of a
// workgroup take neighbouring heads of the same tokens.  With more sequences
// than PAGED_SPLIT each is one part, since they fill the chip by themselves.
//
// Lane (g, c) = (lane / 16, lane % 16) reads the 16-byte pieces 4s + g of the
// keys and values of token c of each 16 (64 contiguous bytes per token and
// instruction).  The key registers are the operand of S^T = K Q^T as they
// stand; lane (g, c) then holds query c against tokens 4g + j.  The values go
// through the wave's own LDS tile, from which O^T = V^T P^T takes them
// transposed.  The next tile's keys and values are under way from the moment
// the current ones are in LDS and S, its page numbers one tile earlier.
// Values of hidden tokens are cleared, so that 0 times infinity or NaN does
// not arise.  Of a visible token it does: where a weight underflows, and where
// the second of the two bf16 numbers that stand for it is 0 or negative; the
// join mends it.  (Weights refer to a maximum that is raised only when it is passed by
// 8 in base 2, so they reach 2^8: finite values whose sum times 2^8 passes fp32's range
// overflow, in all types.)
//
// With a window over a cache whose slots are out of order a wave gathers the
// visible ones of its part first, LIST at a time (16 sequences of up to 4,099
// tokens, of which an eighth are visible, 12 fp32 heads of 64: 34.7 us with all
// slots in the tiles, 30.0 with those gathered, the join included).
//
// Each part of a sequence leaves its maximum, sum and unnormalised output;
// paged_join adds the parts up and turns the scores, kept in fp32, into the
// weight that every token drew.
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef unsigned u32x4_t __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr int PAGED_SPLIT = 1024;  // sequences up to which the work is split over their lengths
// Parts in all, about: the waves that the registers let run at once (64-wide
// heads, 64 sequences of 4,096 tokens, 12 heads: with 2,048 parts 2.5 % slower,
// with 4,096 4 %).
constexpr int PAGED_WAVES = 2048, PAGED_WAVES_64 = 3 * 1024;
// Waves of a SIMD over a cache in 4 bits, as the registers allow without spills: 16
// windowed sequences of fp32 queries with 96-wide heads take 18.4 us with 2, 20.1 with
// 3; the bf16 ones of paged4_flat's comment, by paged_attention, 77 with 3, 86 with 2.
template <typename T, int DP> constexpr int four_waves() { return sizeof(T) == 4 && DP == 128 ? 2 : 3; }

constexpr int LIST = 512;  // tokens of a part that are gathered at a time

// The values of a lane's 16 or 8 bytes of e2m1 codes, in bf16 (exact, since the
// scale is a power of two; 255 is NaN).  The scaled matrix instruction takes codes and
// scales as they lie in memory, but brings the 128 products that it adds to the
// largest one's exponent: off by 7e-5 of it on average, where the bf16 instruction is
// by 4e-9 of their sum, so the weights would lose half their bits.
__device__ __forceinline__ uint32_t four_pair(uint32_t codes, float scale, int at) {
  typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
  bf16x2_t r;
  switch (at) {
    case 0: r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0); break;
    case 1: r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1); break;
    case 2: r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2); break;
    default: r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3);
  }
  return __builtin_bit_cast(uint32_t, r);
}
__device__ __forceinline__ uint4 four_word(uint32_t codes, float scale) {
  return make_uint4(four_pair(codes, scale, 0), four_pair(codes, scale, 1), four_pair(codes, scale, 2),
                    four_pair(codes, scale, 3));
}
__device__ __forceinline__ void four_values(uint2 c, uint32_t scale, uint4* v) {
  const float s = __uint_as_float(scale << 23);
  v[0] = four_word(c.x, s);
  v[1] = four_word(c.y, s);
}
__device__ __forceinline__ void four_values(uint4 c, uint32_t scale, uint4* v) {
  four_values(make_uint2(c.x, c.y), scale, v);
  four_values(make_uint2(c.z, c.w), scale, v + 2);
}
// Columns of 16 lanes: `from`'s first W into the x-th W of `to`, and back (the others
// of the result hold anything).
template <int W>
__device__ __forceinline__ float columns_right(int x, float to, float from) {
  const int t = __float_as_int(to), f = __float_as_int(from);
  int r = t;
  if (W == 8) r = __builtin_amdgcn_update_dpp(t, f, 0x118, 0xF, 0xC, false);  // row_shr 8
  if (W == 4 && x == 1) r = __builtin_amdgcn_update_dpp(t, f, 0x114, 0xF, 0x2, false);
  if (W == 4 && x == 2) r = __builtin_amdgcn_update_dpp(t, f, 0x118, 0xF, 0x4, false);
  if (W == 4 && x == 3) r = __builtin_amdgcn_update_dpp(t, f, 0x11C, 0xF, 0x8, false);
  return __int_as_float(r);
}
template <int W>
__device__ __forceinline__ uint32_t columns_left(int x, uint32_t v) {
  if (W == 8 && x) return __builtin_amdgcn_mov_dpp(v, 0x108, 0xF, 0xF, true);  // row_shl 8
  if (W == 4 && x == 1) return __builtin_amdgcn_mov_dpp(v, 0x104, 0xF, 0xF, true);
  if (W == 4 && x == 2) return __builtin_amdgcn_mov_dpp(v, 0x108, 0xF, 0xF, true);
  if (W == 4 && x == 3) return __builtin_amdgcn_mov_dpp(v, 0x10C, 0xF, 0xF, true);
  return v;
}
// Eight fp32 numbers as sums of three bf16 numbers.
__device__ __forceinline__ void bf16_parts(float4 a, float4 b, uint4* part) {
#pragma unroll
  for (int i = 0; i < 3; i++) {
    part[i] = make_uint4(pack_bf16x2(a.x, a.y), pack_bf16x2(a.z, a.w), pack_bf16x2(b.x, b.y),
                         pack_bf16x2(b.z, b.w));
    auto low = [](uint32_t u) { return __uint_as_float(u << 16); };
    auto high = [](uint32_t u) { return __uint_as_float(u & 0xFFFF0000u); };
    a.x -= low(part[i].x); a.y -= high(part[i].x); a.z -= low(part[i].y); a.w -= high(part[i].y);
    b.x -= low(part[i].z); b.y -= high(part[i].z); b.z -= low(part[i].w); b.w -= high(part[i].w);
  }
}

struct PagedSpace {
  int2* plan;    // [B]: first part, number of parts
  float2* ml;    // [parts][H]: maximum (base 2), sum
  float* o;      // [parts][H][DP]
  float* score;  // [B][units][tiles][heads][KT], base 2, by visible token
  int ranges;    // parts per unit
  int units, qtiles, tiles, heads;  // (heads of a unit, at most 16)
  int block0;    // number of the launch's first workgroup
  const int* sel;  // [B][Hkv][blocks]: pages of the chosen blocks, in order
  FastDiv by_group;
};
// Tokens of a tile.
template <typename T, bool FOUR> __host__ __device__ constexpr int tile_tokens() {
  return sizeof(T) == 2 || FOUR ? 32 : 16;
}

// The visible tokens of a sequence: x-th visible token -> slot.  In a cache
// whose slots are in order a window is a range of them; else positions decide.
struct Visible {
  int n;      // slots in use
  int nv;     // candidates
  int head;   // the first `head` candidates are slots 0 .. head-1
  int gap;    // the others are that many slots further on
  int oldest; // by_pos: the smallest position in the window
  bool by_pos;
  __device__ __forceinline__ int slot(int x) const { return x < head ? x : x + gap; }
  __device__ __forceinline__ bool by_position(const int* pos, int x, int sinks) const {
    return !by_pos || pos[x] >= oldest || pos[x] < sinks;
  }
};
template <bool SEL>
__device__ __forceinline__ Visible visible(const CacheArgs& c, const PagedArgs& a, int b) {
  Visible v;
  v.n = v.nv = held(c, b);
  v.head = v.gap = 0;
  if constexpr (SEL) {  // the chosen pages are full but for the last, which is the sequence's last
    const int pages = (int)quot((uint32_t)v.n + c.page.d - 1, c.page);
    v.nv -= max(0, pages - a.blocks) * (int)c.page.d;
    v.by_pos = false;
    v.oldest = 0;
    return v;
  }
  const int seen = c.seen[b];
  v.by_pos = a.window > 0 && seen != v.n;
  v.oldest = (int)max((int64_t)seen - a.window, (int64_t)INT32_MIN);
  if (a.window > 0 && !v.by_pos && v.n - a.window > a.sinks) {
    v.head = a.sinks;
    v.nv = a.sinks + a.window;
    v.gap = v.n - v.nv;
  }
  return v;
}

// The wave's part of the line of tiles: runs segment(sequence, its first tile, the
// one past its last, part) for each piece of it, and leaves the plan of the parts
// (the first wave of each line).
template <int KT, bool SEL, typename F>
__device__ __forceinline__ void paged_walk(const CacheArgs& c, const PagedArgs& a, const PagedSpace& ws,
                                           int unit, int range, int lane, F segment) {
  // the sequences whose tiles form the line: all, or the part's own
  const bool split = c.B <= PAGED_SPLIT;
  const int b0 = split ? 0 : range, b1 = split ? c.B : range + 1;
  auto tiles_of = [&](int b) { return b < b1 ? (visible<SEL>(c, a, b).nv + KT - 1) / KT : 0; };
  const int head = tiles_of(b0 + lane);  // of the first 64 sequences, kept
  int total = __builtin_amdgcn_readfirstlane(wave_sum_i(head));
  for (int b = b0 + 64; b < b1; b += 64)
    total += __builtin_amdgcn_readfirstlane(wave_sum_i(tiles_of(b + lane)));
  const int per = max(1, split ? (total + ws.ranges - 1) / ws.ranges : total);
  const int first = split ? range * per : 0, last = min(first + per, total);
  const bool planner = unit == 0 && (range == 0 || !split);
  if (first >= total && !planner) return;
  int before = 0;  // tiles of the sequences before b
  for (int b = b0; b < b1 && (before < last || planner); b += 64) {
    const int t = b == b0 ? head : tiles_of(b + lane);
    int p = wave_scan(t);  // inclusive, then exclusive sum over the lanes
    const int sum = __builtin_amdgcn_readlane(p, 63);
    p += before - t;
    before += sum;
    if (planner && b + lane < b1)
      ws.plan[b + lane] = make_int2(p / per + b + lane, t > 0 ? (p + t - 1) / per - p / per + 1 : 0);
    for (uint64_t mine = __ballot(t > 0 && p < last && p + t > first); mine; mine &= mine - 1) {
      const int i = __builtin_ctzll(mine);
      const int tp = __builtin_amdgcn_readlane(p, i), tn = __builtin_amdgcn_readlane(t, i);
      segment(b + i, max(first - tp, 0), min(last - tp, tn), split ? range + b + i : range);
    }
  }
}

template <typename T, int DP, bool PAD, bool ACC, bool FOUR, bool SEL>
__global__ __launch_bounds__(256, (FOUR ? four_waves<T, DP>() : 2)) void paged_attention(CacheArgs c, PagedArgs a,
                                                                              PagedSpace ws) {
  constexpr bool BF = sizeof(T) == 2 || FOUR;  // values are bf16 in LDS
  constexpr int KT = BF ? 32 : 16, NSUB = KT / 16;
  constexpr int EPP = BF ? 8 : 4;           // values per 16-byte piece
  constexpr int NL = DP / EPP / 4;          // pieces per lane and token
  constexpr int ND = DP / 16;
  constexpr int VROW = BF ? DP * 2 : (DP + 4) * 4;  // bytes of a token's values in LDS
  constexpr int NQ = FOUR && sizeof(T) == 4 ? 3 : 1;  // bf16 numbers that stand for a query's
  constexpr int NP = sizeof(T) == 4 ? 3 : 2;          // and for a weight
  constexpr int BL = DP / 8;                // bytes of a token's 4-bit values that a lane reads
  __shared__ __attribute__((aligned(16))) char v_all[4 * KT * VROW];
  // LDS that a wave's values leave free: scores held back, or a list of tokens
  // (allocated in units of 1280 bytes, 160 KB a CU, for the workgroups that run at once)
  constexpr int SHARE = 160 * 1024 / (FOUR ? four_waves<T, DP>() : DP <= 64 ? 3 : 2) / 1280 * 1280 / 4;
  constexpr int SCORE_BYTES = (SHARE - KT * VROW) / 1024 * 1024;
  static_assert(SCORE_BYTES >= 2048 && SCORE_BYTES >= LIST * 4, "a tile of 16 heads, a list");
  constexpr int SPARE = ACC ? SCORE_BYTES : LIST * 4;
  __shared__ __attribute__((aligned(16))) char s_all[4 * SPARE];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int g = lane >> 4, cl = lane & 15;
  const int id = (blockIdx.x + ws.block0) * 4 + wave, unit = id % ws.units, range = id / ws.units;
  if (range >= ws.ranges) return;
  char* Vs = v_all + wave * KT * VROW;
  char* Ss = s_all + wave * SPARE;
  int* list = (int*)Ss;
  const int kh = unit / ws.qtiles, qt = unit % ws.qtiles;
  const int h0 = kh * a.group + qt * 16, nq = min(16, a.group - qt * 16);
  const int dh = c.dh;
  const float sc2 = a.scale * kLog2e;
  // place of the 32-byte segment of a token's values in LDS (bf16): permuted so
  // that 8 tokens cover the banks, and the halves of a segment swapped every 8
  // tokens, so that 16 tokens' 16-byte pieces do
  auto v_at = [](int r, int seg) {
    return r * VROW + ((seg ^ (DP == 128 ? r & 7 : r >> 1 & 3)) << 5);
  };

  auto segment = [&](int b, int ta, int tb, int part) {
    Visible vis = visible<SEL>(c, a, b);
    vis.nv = __builtin_amdgcn_readfirstlane(vis.nv);
    vis.head = __builtin_amdgcn_readfirstlane(vis.head);
    vis.gap = __builtin_amdgcn_readfirstlane(vis.gap);
    vis.oldest = __builtin_amdgcn_readfirstlane(vis.oldest);
    const bool by_pos = __builtin_amdgcn_readfirstlane(vis.by_pos);
    // Q^T operand
    uint4 q[NQ][NL];
#pragma unroll
    for (int s = 0; s < NL; s++) {
#pragma unroll
      for (int i = 0; i < NQ; i++) q[i][s] = make_uint4(0, 0, 0, 0);
      const int d = FOUR ? (NL * g + s) * 8 : (4 * s + g) * EPP;
      if (cl < nq && (!PAD || d < dh)) {
        const T* qp = (const T*)a.q + (int64_t)b * a.q_row + (int64_t)(h0 + cl) * a.q_head + d;
        if constexpr (NQ == 1) {
          q[0][s] = *(const uint4*)qp;
        } else {
          uint4 part[3];
          bf16_parts(*(const float4*)qp, *(const float4*)(qp + 4), part);
#pragma unroll
          for (int i = 0; i < NQ; i++) q[i][s] = part[i];
        }
      }
    }
    const int* table = SEL ? ws.sel + ((int64_t)b * c.Hkv + kh) * a.blocks
                           : c.table + (int64_t)b * c.max_pages;
    // tiles t0 .. t1 - 1 of the tokens in hand, `limit` of them: the part's own,
    // or those of its tokens that are visible by position
    int t0 = ta, t1 = tb, limit = vis.nv;
    // page and place of the lane's tokens of a tile
    struct Tokens {
      int page[NSUB], place[NSUB];
    };
    auto look_up = [&](int t) {
      Tokens k;
#pragma unroll
      for (int u = 0; u < NSUB; u++) {
        const int i = min(t * KT + 16 * u + cl, limit - 1), x = by_pos ? list[by_pos ? i : 0] : vis.slot(i);
        const uint32_t pg = quot((uint32_t)x, c.page);
        k.page[u] = table[pg];
        k.place[u] = x - (int)(pg * c.page.d);
      }
      return k;
    };
    // keys and values of the lane's tokens; hidden ones read the cache's first row
    typedef typename std::conditional<FOUR, uint8_t, T>::type Held;
    typedef typename std::conditional<DP == 128, uint4, uint2>::type Four;
    uint4 kr[NSUB][NL], vr[NSUB][NL];
    Four k4[NSUB], v4[NSUB];         // 4 bits: the lane's block (a half of one at 64 dims), its scale
    uint32_t ks[NSUB], vs[NSUB];
    uint32_t mask_next;  // visible tokens of the tile, one bit each
    bool see[NSUB];
    const Held* kp[NSUB];
    const Held* vp[NSUB];
    const uint8_t* ksp[NSUB];
    const uint8_t* vsp[NSUB];
    auto point = [&](int t, const Tokens& tk) {
      mask_next = 0;
#pragma unroll
      for (int u = 0; u < NSUB; u++) {
        see[u] = (t * KT + 16 * u + cl < limit) & ((unsigned)tk.page[u] < (unsigned)c.pages);
        mask_next |= (uint32_t)(__ballot(see[u]) & 0xFFFF) << (16 * u);
        const int64_t p = see[u] ? tk.page[u] : 0, r = see[u] ? tk.place[u] : 0;
        kp[u] = (const Held*)c.k + p * c.k_page + r * c.k_row + kh * c.k_head;
        vp[u] = (const Held*)c.v + p * c.v_page + r * c.v_row + kh * c.v_head;
        if constexpr (FOUR) {
          ksp[u] = c.ks + p * c.ks_page + r * c.ks_row + kh * c.ks_head;
          vsp[u] = c.vs + p * c.vs_page + r * c.vs_row + kh * c.vs_head;
        }
      }
    };
    auto load_four = [&]() {
      const bool in = !PAD || g * BL * 2 < dh;
      const int at = in ? g * BL : 0, block = at >> 4;
#pragma unroll
      for (int u = 0; u < NSUB; u++) {
        k4[u] = *(const Four*)(kp[u] + at);
        ks[u] = ksp[u][block];
      }
#pragma unroll
      for (int u = 0; u < NSUB; u++) {
        v4[u] = *(const Four*)(vp[u] + at);
        vs[u] = vsp[u][block];
      }
    };
    auto load_kv = [&]() {
      if constexpr (FOUR) {
        load_four();
        return;
      }
#pragma unroll
      for (int u = 0; u < NSUB; u++)
#pragma unroll
        for (int s = 0; s < NL; s++) {
          const int d = (4 * s + g) * EPP;
          kr[u][s] = make_uint4(0, 0, 0, 0);
          if (!PAD || d < dh) kr[u][s] = *(const uint4*)(kp[u] + d);
        }
#pragma unroll
      for (int u = 0; u < NSUB; u++)
#pragma unroll
        for (int s = 0; s < NL; s++) {
          const int d = (4 * s + g) * EPP;
          vr[u][s] = make_uint4(0, 0, 0, 0);
          if (!PAD || d < dh) vr[u][s] = *(const uint4*)(vp[u] + d);
        }
    };
    float m = -INFINITY, l = 0.f;
    f32x4_t O[ND];
#pragma unroll
    for (int d = 0; d < ND; d++) O[d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    // Scores wait in LDS until they fill SCORE_BYTES and then leave in whole
    // 1-KB stores: writes among the reads cost the memory more than their bytes
    // do, so they come together and seldom (64 sequences of 4,096 tokens, 4
    // heads a unit, 33 MB written beside 1.07 GB read: 230 us with 12 KB held back,
    // 239 with 2 KB, 209 without any scores written).
    // (a tile's rows in LDS: the next power of two from nq on)
    const int tile_shift = 31 - __builtin_clz(2 * nq - 1) + (BF ? 7 : 6);  // bytes of a tile
    const int slots = SCORE_BYTES >> tile_shift;
    int held_from = ta;
    auto store_scores = [&](int t) {  // tiles held_from .. t
#pragma unroll(FOUR ? 1 : SCORE_BYTES / 1024)
      for (int i = 0; i < SCORE_BYTES / 1024; i++) {
        const int at = (i * 64 + lane) * 16, x = held_from + (at >> tile_shift);
        const int in = at & ((1 << tile_shift) - 1);
        if (x <= t && in < nq * KT * 4)
          *(uint4*)((char*)(ws.score + (((int64_t)b * ws.units + unit) * ws.tiles + x) * ws.heads * KT) +
                    in) = *(const uint4*)(Ss + at);
      }
      held_from = t + 1;
    };
    // Scores of visible tokens to the places of their slots (the join does not
    // read those of the others).
    auto scatter_scores = [&](int t, const f32x4_t* S) {
      if (cl >= nq) return;
#pragma unroll
      for (int u = 0; u < NSUB; u++) {
        const int i = t * KT + 16 * u + 4 * g;
#pragma unroll
        for (int j = 0; j < 4; j++)
          if (i + j < limit) {
            const int x = list[i + j];
            ws.score[((((int64_t)b * ws.units + unit) * ws.tiles + x / KT) * ws.heads + cl) * KT + x % KT] =
                S[u][j];
          }
      }
    };
    // One tile in straight line, with its memory operations in a fixed order
    // (look-ups two tiles ahead, the next tile's keys, its values, scores now
    // and then), so that each wait counts the operations after the one it
    // needs.  LAST: no tile follows.
    auto tile = [&](int t, Tokens& ahead, auto last_c) {
      constexpr bool LAST = decltype(last_c)::value;
      const uint32_t mask = mask_next;
      f32x4_t S[NSUB];
#pragma unroll
      for (int u = 0; u < NSUB; u++) {
        if constexpr (FOUR) {
          // (what a hidden token's place holds is masked below, and its values are cleared)
          const bool in = !PAD || g * BL * 2 < dh;
          four_values(k4[u], in ? ks[u] : 0, kr[u]);
          if (!see[u] || !in) v4[u] = Four{};
          vs[u] = see[u] && in ? vs[u] : 0;
        }
        S[u] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < NL; s++) {
          if constexpr (BF) {
#pragma unroll
            for (int i = NQ - 1; i >= 0; i--)
              S[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, kr[u][s]),
                                                             __builtin_bit_cast(bf16x8_t, q[i][s]),
                                                             S[u], 0, 0, 0);
          } else {
            const f32x4_t kf = __builtin_bit_cast(f32x4_t, kr[u][s]);
            const f32x4_t qf = __builtin_bit_cast(f32x4_t, q[0][s]);
#pragma unroll
            for (int i = 0; i < 4; i++)
              S[u] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[i], qf[i], S[u], 0, 0, 0);
          }
        }
      }
#pragma unroll
      for (int u = 0; u < NSUB; u++) {
        if constexpr (FOUR) four_values(v4[u], vs[u], vr[u]);
#pragma unroll
        for (int s = 0; s < NL; s++) {
          const uint4 x = vr[u][s];
          const uint4 v = FOUR ? x
                               : make_uint4(see[u] ? x.x : 0, see[u] ? x.y : 0, see[u] ? x.z : 0,
                                            see[u] ? x.w : 0);
          const int r = 16 * u + cl, p = FOUR ? NL * g + s : 4 * s + g;
          if constexpr (BF)
            *(uint4*)(Vs + v_at(r, p >> 1) + ((p & 1) << 4 ^ (r >> 3 & 1) << 4)) = v;
          else
            *(uint4*)(Vs + r * VROW + p * 16) = v;
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (!LAST) {
        point(t + 1, ahead);
        __builtin_amdgcn_sched_barrier(0);
        ahead = look_up(min(t + 2, t1 - 1));
        __builtin_amdgcn_sched_barrier(0);
        load_kv();
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int u = 0; u < NSUB; u++)
#pragma unroll
        for (int j = 0; j < 4; j++)
          S[u][j] = mask >> (16 * u + 4 * g + j) & 1 ? S[u][j] * sc2 : -INFINITY;
      if constexpr (ACC) {
        if (by_pos) {
          scatter_scores(t, S);
        } else {
          if (cl < nq) {
#pragma unroll
            for (int u = 0; u < NSUB; u++)
              *(f32x4_t*)(Ss + ((t - held_from) << tile_shift) + (cl * KT + 16 * u + 4 * g) * 4) = S[u];
          }
          if (LAST || t - held_from == slots - 1) store_scores(t);
        }
      }
      float mt = fmaxf(fmaxf(S[0][0], S[0][1]), fmaxf(S[0][2], S[0][3]));
      if (NSUB > 1)
        mt = fmaxf(mt, fmaxf(fmaxf(S[NSUB - 1][0], S[NSUB - 1][1]), fmaxf(S[NSUB - 1][2], S[NSUB - 1][3])));
      mt = max_xor32(max_xor16(mt));
      const bool grow = mt > m + 8.f;
      const float f = grow ? __builtin_amdgcn_exp2f(m - mt) : 1.f;
      m = grow ? mt : m;
      if (!FOUR || __any(grow)) {
        l *= f;
#pragma unroll
        for (int d = 0; d < ND; d++)
#pragma unroll
          for (int j = 0; j < 4; j++) O[d][j] *= f;
      }
      const float mu = m == -INFINITY ? 0.f : m;
#pragma unroll
      for (int u = 0; u < NSUB; u++) {
#pragma unroll
        for (int j = 0; j < 4; j++) S[u][j] = __builtin_amdgcn_exp2f(S[u][j] - mu);
        l += (S[u][0] + S[u][1]) + (S[u][2] + S[u][3]);
      }
      if constexpr (BF) {
        // P as the sum of two bf16 numbers, 16 bits of precision (of three for
        // fp32): the second product costs nothing beside the loads
        union { uint32_t u[4]; bf16x8_t v; } p[NP];
#pragma unroll
        for (int w = 0; w < 4; w++) {
          float e0 = S[w / 2 * (NSUB - 1)][w % 2 * 2], e1 = S[w / 2 * (NSUB - 1)][w % 2 * 2 + 1];
#pragma unroll
          for (int i = 0; i < NP; i++) {
            p[i].u[w] = pack_bf16x2(e0, e1);
            e0 -= __uint_as_float(p[i].u[w] << 16);
            e1 -= __uint_as_float(p[i].u[w] & 0xFFFF0000u);
          }
        }
        // V^T: dims 16 d + cl, tokens 4g .. + 3 and 16 + 4g .. + 3
#pragma unroll
        for (int d = 0; d < ND; d++) {
          union { s16x4_t h[2]; bf16x8_t v; } vf;
#pragma unroll
          for (int z = 0; z < 2; z++) {
            const int r = 16 * z + 4 * g + (cl >> 2);
            vf.h[z] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (__attribute__((address_space(3))) s16x4_t*)(
                    Vs + v_at(r, d) + ((cl & 3) << 3 ^ (r >> 3 & 1) << 4)));
          }
#pragma unroll
          for (int i = 0; i < NP; i++)
            O[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf.v, p[i].v, O[d], 0, 0, 0);
        }
      } else {
#pragma unroll
        for (int j = 0; j < 4; j++)
#pragma unroll
          for (int d = 0; d < ND; d++)
            O[d] = __builtin_amdgcn_mfma_f32_16x16x4f32(
                *(const float*)(Vs + (4 * g + j) * VROW + (16 * d + cl) * 4), S[0][j], O[d], 0, 0, 0);
      }
    };
    int next = ta * KT;
    const int end = min(tb * KT, vis.nv);
    const int* pos = c.pos + (int64_t)b * c.cap;
    do {
      if (by_pos) {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // (its last reader is done)
        __builtin_amdgcn_wave_barrier();
        int count = 0;
        for (; next < end && count <= LIST - 256; next += 256) {
          int at[4];
#pragma unroll
          for (int k = 0; k < 4; k++) at[k] = pos[min(next + 64 * k + lane, end - 1)];
#pragma unroll
          for (int k = 0; k < 4; k++) {
            const int x = next + 64 * k + lane;
            const bool in = (x < end) & ((at[k] >= vis.oldest) | (at[k] < a.sinks));
            const uint64_t m = __ballot(in);
            if (in) list[count + __popcll(m & ((1ull << lane) - 1))] = x;
            count += __popcll(m);
          }
        }
        // (the list is the wave's own, and its LDS operations stay in order)
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        if (count == 0) continue;
        t0 = 0;
        t1 = (count + KT - 1) / KT;
        limit = count;
      }
      Tokens ahead = look_up(t0);
      point(t0, ahead);
      ahead = look_up(min(t0 + 1, t1 - 1));
      load_kv();
      for (int t = t0; t < t1 - 1; t++) tile(t, ahead, std::false_type{});
      tile(t1 - 1, ahead, std::true_type{});
    } while (by_pos && next < end);
    l = sum_xor32(sum_xor16(l));
    if (cl < nq) {
      const int64_t o = (int64_t)part * a.H + h0 + cl;
      if (g == 0) ws.ml[o] = make_float2(m, l);
#pragma unroll
      for (int d = 0; d < ND; d++) *(f32x4_t*)(ws.o + o * DP + 16 * d + 4 * g) = O[d];
    }
  };

  paged_walk<KT, SEL>(c, a, ws, unit, range, lane, segment);
}

// The same over 4 bits without a window, in pages of whole 16 tokens: tiles of 64
// tokens whose sub-tiles of 16 lie in a page each (ONE: pages of whole tiles), so that
// addresses are the wave's and a lane adds what it always adds, where paged_attention
// spends as much on addresses as on arithmetic.  Rows past the end are read (their
// page has them) and masked.
//
// A key head of up to 16 / R query heads fills 16 / R of the 16 columns of the
// scores.  R sub-tiles are moved side by side, so that the softmax works on 64 tokens
// in 16 / R registers where it took 16, and the weights move back for the product
// with the values.  Keys are on their way while the softmax and the values are worked
// on, values while the next scores are; the halves of a tile's values share the LDS.
//
// 64 sequences of up to 8,192 tokens, 32 bf16 heads of 128 over 8 (290 MB of cache, 33 of
// scores): 69 us, 4.7 TB/s, by paged_attention 77.  When it took 71: 63 if the cache
// came from the last level, 52 without scores; with every tile read from L2 54 and 47,
// of which 14 were the product with the values.  Memory and the issue of instructions
// bound it together: vector instructions 19 us, matrix 10, LDS 28; a quarter of the
// waves' cycles wait for memory, half for issue.  Scores written past the caches gain
// nothing.
constexpr int FLAT_KT = 64;
template <typename T, int DP, int R> constexpr int flat_waves() { return R < 4 && DP == 128 ? 2 : four_waves<T, DP>(); }
template <typename T, int DP, bool PAD, bool ACC, bool SEL, int R, bool ONE>
__global__ __launch_bounds__(256, (flat_waves<T, DP, R>())) void paged4_flat(CacheArgs c, PagedArgs a,
                                                                        PagedSpace ws) {
  constexpr int KT = FLAT_KT, NSUB = 4, NS = NSUB / R, W = 16 / R;
  constexpr int NL = DP / 32, ND = DP / 16, VROW = DP * 2, BL = DP / 8;
  constexpr int NQ = sizeof(T) == 4 ? 3 : 1, NP = sizeof(T) == 4 ? 3 : 2;
  typedef typename std::conditional<DP == 128, uint4, uint2>::type Four;
  __shared__ __attribute__((aligned(16))) char v_all[4 * 32 * VROW];
  constexpr int SHARE = 160 * 1024 / flat_waves<T, DP, R>() / 1280 * 1280 / 4;
  constexpr int SCORE_BYTES = (SHARE - 32 * VROW) / 1024 * 1024;
  static_assert(SCORE_BYTES >= 16 * KT * 4, "a tile of 16 heads");
  __shared__ __attribute__((aligned(16))) char s_all[ACC ? 4 * SCORE_BYTES : 16];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int g = lane >> 4, cl = lane & 15;
  const int id = (blockIdx.x + ws.block0) * 4 + wave, unit = id % ws.units, range = id / ws.units;
  if (range >= ws.ranges) return;
  char* Vs = v_all + wave * 32 * VROW;
  char* Ss = s_all + (ACC ? wave * SCORE_BYTES : 0);
  const int kh = unit / ws.qtiles, qt = unit % ws.qtiles;
  const int h0 = kh * a.group + qt * 16, nq = min(16, a.group - qt * 16);
  const float sc2 = a.scale * kLog2e;
  const bool in = !PAD || g * BL * 2 < c.dh;
  const uint32_t at4 = in ? g * BL : 0, block4 = at4 >> 4;
  const uint32_t k_lane = cl * (uint32_t)c.k_row + at4, v_lane = cl * (uint32_t)c.v_row + at4;
  const uint32_t ks_lane = cl * (uint32_t)c.ks_row + block4, vs_lane = cl * (uint32_t)c.vs_row + block4;
  const uint8_t* k_base = (const uint8_t*)c.k + kh * c.k_head;
  const uint8_t* v_base = (const uint8_t*)c.v + kh * c.v_head;
  const uint8_t* ks_base = c.ks + kh * c.ks_head;
  const uint8_t* vs_base = c.vs + kh * c.vs_head;
  auto v_at = [](int r, int seg) {  // (as in paged_attention)
    return r * VROW + ((seg ^ (DP == 128 ? r & 7 : r >> 1 & 3)) << 5);
  };
  const int tile_shift = 31 - __builtin_clz(2 * nq - 1) + 8, slots = SCORE_BYTES >> tile_shift;

  auto segment = [&](int b, int t0, int t1, int part) {
    const int limit = __builtin_amdgcn_readfirstlane(visible<SEL>(c, a, b).nv);
    uint4 q[NQ][NL];
#pragma unroll
    for (int s = 0; s < NL; s++) {
#pragma unroll
      for (int i = 0; i < NQ; i++) q[i][s] = make_uint4(0, 0, 0, 0);
      const int d = (NL * g + s) * 8;
      if (cl < nq && (!PAD || d < c.dh)) {
        const T* qp = (const T*)a.q + (int64_t)b * a.q_row + (int64_t)(h0 + cl) * a.q_head + d;
        if constexpr (NQ == 1) {
          q[0][s] = *(const uint4*)qp;
        } else {
          uint4 parts[3];
          bf16_parts(*(const float4*)qp, *(const float4*)(qp + 4), parts);
#pragma unroll
          for (int i = 0; i < NQ; i++) q[i][s] = parts[i];
        }
      }
    }
    const int* table = SEL ? ws.sel + ((int64_t)b * c.Hkv + kh) * a.blocks
                           : c.table + (int64_t)b * c.max_pages;
    Four k4[NSUB], v4[NSUB];
    uint32_t ks[NSUB], vs[NSUB];
    // addresses of the sub-tiles (ONE: of the tile, which lies in one page)
    constexpr int NA = ONE ? 1 : NSUB;
    const uint8_t *kp[NA], *vp[NA], *ksp[NA], *vsp[NA];
    int here;  // sub-tiles whose page is there, one bit each
    // pages of the sub-tiles, in the first lanes
    auto find = [&](int t) {
      const int x = t * KT + (ONE ? 0 : 16 * (lane & 3));
      return table[quot((uint32_t)min(x, limit - 1), c.page)];
    };
    auto aim = [&](int t, int found) {
      here = 0;
#pragma unroll
      for (int u = 0; u < NA; u++) {
        const int x = t * KT + 16 * u, page = __builtin_amdgcn_readlane(found, u);
        const bool h = x < limit && (unsigned)page < (unsigned)c.pages;
        const uint32_t p = h ? page : 0;
        const uint32_t r = h ? x - quot((uint32_t)x, c.page) * c.page.d : 0;
        here |= (ONE ? h * ((1 << NSUB) - 1) : h << u);
        kp[u] = k_base + (uint64_t)p * (uint32_t)c.k_page + (uint64_t)r * (uint32_t)c.k_row;
        vp[u] = v_base + (uint64_t)p * (uint32_t)c.v_page + (uint64_t)r * (uint32_t)c.v_row;
        ksp[u] = ks_base + (uint64_t)p * (uint32_t)c.ks_page + (uint64_t)r * (uint32_t)c.ks_row;
        vsp[u] = vs_base + (uint64_t)p * (uint32_t)c.vs_page + (uint64_t)r * (uint32_t)c.vs_row;
      }
    };
    // (the lanes' offsets are made anew for every tile: sixteen of them kept would spill)
    auto load_k = [&]() {
      uint32_t kl = k_lane, sl = ks_lane;
      if (ONE) asm volatile("" : "+v"(kl), "+v"(sl));
#pragma unroll
      for (int u = 0; u < NSUB; u++) {
        k4[u] = *(const Four*)(kp[u % NA] + (kl + (ONE ? 16 * u * (uint32_t)c.k_row : 0)));
        ks[u] = ksp[u % NA][sl + (ONE ? 16 * u * (uint32_t)c.ks_row : 0)];
      }
    };
    auto load_v = [&]() {
      uint32_t vl = v_lane, sl = vs_lane;
      if (ONE) asm volatile("" : "+v"(vl), "+v"(sl));
#pragma unroll
      for (int u = 0; u < NSUB; u++) {
        v4[u] = *(const Four*)(vp[u % NA] + (vl + (ONE ? 16 * u * (uint32_t)c.v_row : 0)));
        vs[u] = vsp[u % NA][sl + (ONE ? 16 * u * (uint32_t)c.vs_row : 0)];
      }
    };
    float m = -INFINITY, l = 0.f;
    f32x4_t O[ND];
#pragma unroll
    for (int d = 0; d < ND; d++) O[d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    int held_from = t0;
    auto store_scores = [&](int t) {  // tiles held_from .. t
#pragma unroll 1
      for (int i = 0; i < SCORE_BYTES / 1024; i++) {
        const int at = (i * 64 + lane) * 16, x = held_from + (at >> tile_shift);
        const int in_tile = at & ((1 << tile_shift) - 1);
        if (x <= t && in_tile < nq * KT * 4)
          *(uint4*)((char*)(ws.score + (((int64_t)b * ws.units + unit) * ws.tiles + x) * ws.heads * KT) +
                    in_tile) = *(const uint4*)(Ss + at);
      }
      held_from = t + 1;
    };
    auto tile = [&](int t, int& ahead, auto last_c) {
      constexpr bool LAST = decltype(last_c)::value;
      const int left = limit - t * KT, there = here;
      const bool whole = left >= KT && there == (1 << NSUB) - 1;
      if (!whole) {
#pragma unroll
        for (int u = 0; u < NSUB; u++) {
          const bool seen = 16 * u + cl < left && (there >> u & 1);
          if (!seen) v4[u] = Four{};
          vs[u] = seen ? vs[u] : 0;
        }
      }
      if (PAD && !in) {
#pragma unroll
        for (int u = 0; u < NSUB; u++) {
          v4[u] = Four{};
          vs[u] = ks[u] = 0;
        }
      }
      // scores: sub-tile i R + x of the columns x W .. x W + W - 1 of set i
      f32x4_t S[NS];
#pragma unroll
      for (int u = 0; u < NSUB; u++) {
        uint4 kr[NL];
        four_values(k4[u], ks[u], kr);
        f32x4_t x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < NL; s++)
#pragma unroll
          for (int i = NQ - 1; i >= 0; i--)
            x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, kr[s]),
                                                        __builtin_bit_cast(bf16x8_t, q[i][s]), x, 0, 0, 0);
        if (u % R == 0) {
          S[u / R] = x;
        } else {
#pragma unroll
          for (int j = 0; j < 4; j++) S[u / R][j] = columns_right<W>(u % R, S[u / R][j], x[j]);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (!LAST) {
        aim(t + 1, ahead);
        __builtin_amdgcn_sched_barrier(0);
        ahead = find(min(t + 2, t1 - 1));
        load_k();
      }
      __builtin_amdgcn_sched_barrier(0);
      const int col = cl / W;  // sub-tile of the lane's column within its set
#pragma unroll
      for (int i = 0; i < NS; i++)
#pragma unroll
        for (int j = 0; j < 4; j++) S[i][j] *= sc2;
      if (!whole) {
#pragma unroll
        for (int i = 0; i < NS; i++) {
          const int u = i * R + col;
#pragma unroll
          for (int j = 0; j < 4; j++)
            S[i][j] = 16 * u + 4 * g + j < left && (there >> u & 1) ? S[i][j] : -INFINITY;
        }
      }
      if constexpr (ACC) {
        if (cl % W < nq) {
#pragma unroll
          for (int i = 0; i < NS; i++)
            *(f32x4_t*)(Ss + ((t - held_from) << tile_shift) +
                        (cl % W * KT + 16 * (i * R + col) + 4 * g) * 4) = S[i];
        }
        if (LAST || t - held_from == slots - 1) store_scores(t);
      }
      float mt = -INFINITY;
#pragma unroll
      for (int i = 0; i < NS; i++)
        mt = fmaxf(mt, fmaxf(fmaxf(S[i][0], S[i][1]), fmaxf(S[i][2], S[i][3])));
      if (R == 4) mt = fmaxf(mt, dpp_peer<0x124>(mt));  // row_ror 4
      if (R >= 2) mt = fmaxf(mt, dpp_peer<0x128>(mt));  // row_ror 8
      mt = max_xor32(max_xor16(mt));
      const bool grow = mt > m + 8.f;
      if (__any(grow)) {
        const float f = grow ? __builtin_amdgcn_exp2f(m - mt) : 1.f;
        m = grow ? mt : m;
        l *= f;
        // (a lane's column of O is that of its own number: the factor of a head is the
        // same in all its columns)
#pragma unroll
        for (int d = 0; d < ND; d++)
#pragma unroll
          for (int j = 0; j < 4; j++) O[d][j] *= f;
      }
      const float mu = m == -INFINITY ? 0.f : m;
      uint32_t p[NS][NP][2];
#pragma unroll
      for (int i = 0; i < NS; i++) {
        float e[4];
#pragma unroll
        for (int j = 0; j < 4; j++) e[j] = __builtin_amdgcn_exp2f(S[i][j] - mu);
        l += (e[0] + e[1]) + (e[2] + e[3]);
#pragma unroll
        for (int w = 0; w < 2; w++)
#pragma unroll
          for (int k = 0; k < NP; k++) {
            p[i][k][w] = pack_bf16x2(e[2 * w], e[2 * w + 1]);
            e[2 * w] -= __uint_as_float(p[i][k][w] << 16);
            e[2 * w + 1] -= __uint_as_float(p[i][k][w] & 0xFFFF0000u);
          }
      }
#pragma unroll
      for (int half = 0; half < 2; half++) {
#pragma unroll
        for (int z = 0; z < 2; z++) {
          const int u = 2 * half + z, r = 16 * z + cl;
          uint4 vr[NL];
          four_values(v4[u], vs[u], vr);
#pragma unroll
          for (int s = 0; s < NL; s++) {
            const int piece = NL * g + s;
            *(uint4*)(Vs + v_at(r, piece >> 1) + ((piece & 1) << 4 ^ (r >> 3 & 1) << 4)) = vr[s];
          }
        }
        union { uint32_t w[4]; bf16x8_t v; } pb[NP];
#pragma unroll
        for (int k = 0; k < NP; k++)
#pragma unroll
          for (int z = 0; z < 2; z++)
#pragma unroll
            for (int w = 0; w < 2; w++) {
              const int u = 2 * half + z;
              pb[k].w[2 * z + w] = columns_left<W>(u % R, p[u / R][k][w]);
            }
#pragma unroll
        for (int d = 0; d < ND; d++) {
          union { s16x4_t h[2]; bf16x8_t v; } vf;
#pragma unroll
          for (int z = 0; z < 2; z++) {
            const int r = 16 * z + 4 * g + (cl >> 2);
            vf.h[z] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (__attribute__((address_space(3))) s16x4_t*)(
                    Vs + v_at(r, d) + ((cl & 3) << 3 ^ (r >> 3 & 1) << 4)));
          }
#pragma unroll
          for (int k = 0; k < NP; k++)
            O[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf.v, pb[k].v, O[d], 0, 0, 0);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (!LAST) load_v();
      __builtin_amdgcn_sched_barrier(0);
    };
    int ahead = find(t0);
    aim(t0, ahead);
    ahead = find(min(t0 + 1, t1 - 1));
    load_k();
    load_v();
    for (int t = t0; t < t1 - 1; t++) tile(t, ahead, std::false_type{});
    tile(t1 - 1, ahead, std::true_type{});
    if (R == 4) l += dpp_peer<0x124>(l);
    if (R >= 2) l += dpp_peer<0x128>(l);
    l = sum_xor32(sum_xor16(l));
    if (cl < nq) {
      const int64_t o = (int64_t)part * a.H + h0 + cl;
      if (g == 0) ws.ml[o] = make_float2(m, l);
#pragma unroll
      for (int d = 0; d < ND; d++) *(f32x4_t*)(ws.o + o * DP + 16 * d + 4 * g) = O[d];
    }
  };
  paged_walk<KT, SEL>(c, a, ws, unit, range, lane, segment);
}

// The parts of every sequence joined: the last workgroups add the weights of
// 1024 visible tokens of a sequence each (4 tokens a lane, a fourth of the
// heads a wave, summed over the waves in order), the first write the output
// rows, `wpr` waves a row.  Bound by a chain of dependent loads, so they go out
// JOIN_AHEAD at a time, the scores before the statistics that they wait for:
// one stream alone has hundreds of parts (two of 131,072 tokens took 37 us with
// one part after the other, 23 with the statistics first).
//
// Where parts of a row are not finite its waves look through the visible values:
// the output of a dimension with infinite or NaN ones is their sum, since weights
// are positive.
constexpr int JOIN_HEADS = 128;
// (8 leave registers for one workgroup a CU: two sequences of 131,072 tokens, 32 heads, 23.3
// us instead of 14.0)
constexpr int JOIN_AHEAD = 4;
// (maximum, sum) of two parts
__device__ __forceinline__ float2 join_ml(float2 a, float2 b) {
  const float m = fmaxf(a.x, b.x), mu = m == -INFINITY ? 0.f : m;
  return make_float2(m, a.y * __builtin_amdgcn_exp2f(a.x - mu) + b.y * __builtin_amdgcn_exp2f(b.x - mu));
}

template <typename T, int DP, int KT, bool FOUR, bool SEL>
__global__ __launch_bounds__(1024, 8) void paged_join(CacheArgs c, PagedArgs a, PagedSpace ws,
                                                   int rows, int chunks, int wpr) {
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  __shared__ __attribute__((aligned(16))) float part[16][256];
  __shared__ float2 s_ml[JOIN_HEADS];
  __shared__ __attribute__((aligned(16))) char s_odd[16];
  const int block = blockIdx.x + ws.block0;
  if (block < rows) {
    const int64_t row = (int64_t)block * (16 / wpr) + wave / wpr;
    const bool real = row < (int64_t)c.B * a.H;
    const int b = real ? (int)(row / a.H) : 0, h = real ? (int)(row % a.H) : 0;
    const int2 plan = ws.plan[b];
    float o0 = 0.f, o1 = 0.f, l = 0.f, m = -INFINITY;
    for (int i = wave % wpr; i < plan.y; i += wpr * JOIN_AHEAD) {
      float2 ml[JOIN_AHEAD];
      float x0[JOIN_AHEAD], x1[JOIN_AHEAD];
      float m2 = m;
#pragma unroll
      for (int u = 0; u < JOIN_AHEAD; u++) {
        const int64_t p = (int64_t)(plan.x + min(i + wpr * u, plan.y - 1)) * a.H + h;
        ml[u] = ws.ml[p];
        x0[u] = ws.o[p * DP + lane];
        x1[u] = DP > 64 ? ws.o[p * DP + 64 + lane] : 0.f;
      }
#pragma unroll
      for (int u = 0; u < JOIN_AHEAD; u++) m2 = fmaxf(m2, ml[u].x);
      const float mu = m2 == -INFINITY ? 0.f : m2, f0 = __builtin_amdgcn_exp2f(m - mu);
      l *= f0;
      o0 *= f0;
      o1 *= f0;
      m = m2;
#pragma unroll
      for (int u = 0; u < JOIN_AHEAD; u++) {
        const float f = i + wpr * u < plan.y ? __builtin_amdgcn_exp2f(ml[u].x - mu) : 0.f;
        l = fmaf(ml[u].y, f, l);
        o0 = fmaf(x0[u], f, o0);
        o1 = fmaf(x1[u], f, o1);
      }
    }
    part[wave][lane] = o0;
    if (DP > 64) part[wave][64 + lane] = o1;
    // (where a score is NaN, the row is, whatever the values)
    const bool odd = __any(!(fabsf(o0) < INFINITY) | !(fabsf(o1) < INFINITY)) && l == l;
    if (lane == 0) {
      s_ml[wave] = make_float2(m, l);
      s_odd[wave] = odd;
    }
    __syncthreads();
    // the row's first waves join its parts
    const int d = tid % (wpr * 64), w0 = wave / wpr * wpr;
    float o = 0.f, sum = 0.f;
    if (real && d < c.dh) {
      float top = -INFINITY;
      for (int w = 0; w < wpr; w++) top = fmaxf(top, s_ml[w0 + w].x);
      top = top == -INFINITY ? 0.f : top;
      for (int w = 0; w < wpr; w++) {
        const float f = __builtin_amdgcn_exp2f(s_ml[w0 + w].x - top);
        sum = fmaf(s_ml[w0 + w].y, f, sum);
        o = fmaf(part[w0 + w][d], f, o);
      }
      o = sum == 0.f ? 0.f : o / sum;
    }
    const uint4 odds = *(const uint4*)s_odd;
    // (4 bits hold no infinities, and the NaN that they hold reach the sums as they stand)
    if (!FOUR && __builtin_amdgcn_readfirstlane(odds.x | odds.y | odds.z | odds.w)) {
      __syncthreads();
      float e0 = 0.f, e1 = 0.f;
      if (real) {
        const Visible vis = visible<SEL>(c, a, b);
        const int* table = SEL ? ws.sel + ((int64_t)b * c.Hkv + h / a.group) * a.blocks
                               : c.table + (int64_t)b * c.max_pages;
        const int d1 = 64 + lane;
        for (int i = wave % wpr; i < vis.nv; i += wpr * 2) {
#pragma unroll
          for (int u = 0; u < 2; u++) {
            const int x = vis.slot(min(i + wpr * u, vis.nv - 1));  // (twice the last one: the same sum)
            const uint32_t pg = quot((uint32_t)x, c.page);
            const int page = table[pg];
            const bool see = ((unsigned)page < (unsigned)c.pages) & vis.by_position(c.pos + (int64_t)b * c.cap, x, a.sinks);
            const int64_t p = see ? page : 0, r = see ? x - (int)(pg * c.page.d) : 0;
            const T* v = (const T*)c.v + p * c.v_page + r * c.v_row + h / a.group * c.v_head;
            const float x0 = lane < c.dh ? St<T>::get(v[lane]) : 0.f;
            const float x1 = d1 < c.dh ? St<T>::get(v[d1]) : 0.f;
            e0 += see & !(fabsf(x0) < INFINITY) ? x0 : 0.f;
            e1 += see & !(fabsf(x1) < INFINITY) ? x1 : 0.f;
          }
          // (NaN in all dimensions: nothing changes any more)
          if (__all((lane >= c.dh || e0 != e0) & (d1 >= c.dh || e1 != e1))) break;
        }
      }
      part[wave][lane] = e0;
      part[wave][64 + lane] = e1;
      __syncthreads();
      float e = 0.f;
      if (d < c.dh)
        for (int w = 0; w < wpr; w++) e += part[w0 + w][d];
      o = e == 0.f || sum != sum ? o : e;
    }
    if (real && d < c.dh) ((T*)a.out)[row * c.dh + d] = St<T>::put(o);
    return;
  }
  const int b = (block - rows) / chunks, first = (block - rows) % chunks * 1024;
  // (a chain of loads, so what does not wait for another goes out at once: the plan
  // with the lengths, the old weights with the scores)
  const int2 plan = ws.plan[b];
  const Visible vis = visible<SEL>(c, a, b);
  if (first >= vis.nv) return;
  const int h0 = __builtin_amdgcn_readfirstlane(wave >> 2);  // the wave's heads: h0, h0 + 4, ..
  float* old = c.weight + (int64_t)b * c.cap + vis.slot(min(first + tid, vis.nv - 1));
  // scores of 4 tokens from x on under JOIN_AHEAD of the wave's heads from h on
  auto load_scores = [&](int x, int h, f32x4_t* s) {
    const float* sp = ws.score + (int64_t)b * ws.units * ws.tiles * ws.heads * KT +
                      (int64_t)(min(x, vis.nv - 1) / KT) * ws.heads * KT + x % KT;
#pragma unroll
    for (int u = 0; u < JOIN_AHEAD; u++) {
      const int hu = min(h + 4 * u, a.H - 1), kh = quot(hu, ws.by_group), r = hu - kh * a.group;
      s[u] = *(const f32x4_t*)(sp + ((int64_t)(kh * ws.qtiles + r / 16) * ws.tiles * ws.heads + r % 16) * KT);
    }
  };
  for (int hc = 0; hc < a.H; hc += JOIN_HEADS) {
    const int nh = min(JOIN_HEADS, a.H - hc);
    f32x4_t s[JOIN_AHEAD];
    load_scores(first + (wave & 3) * 256 + lane * 4, hc + h0, s);
    float weight = *old;
    __syncthreads();
    // maximum and 1 / (sum H) of the heads, 32 lanes a head
    for (int h = tid >> 5; h < nh; h += 32) {
      float2 t = make_float2(-INFINITY, 0.f);
      for (int i = tid & 31; i < plan.y; i += 32 * JOIN_AHEAD) {
        float2 ml[JOIN_AHEAD];
#pragma unroll
        for (int u = 0; u < JOIN_AHEAD; u++) {
          ml[u] = ws.ml[(int64_t)(plan.x + min(i + 32 * u, plan.y - 1)) * a.H + hc + h];
          if (i + 32 * u >= plan.y) ml[u].x = -INFINITY;
        }
        float m2 = t.x;
#pragma unroll
        for (int u = 0; u < JOIN_AHEAD; u++) m2 = fmaxf(m2, ml[u].x);
        const float mu = m2 == -INFINITY ? 0.f : m2;
        t.y *= __builtin_amdgcn_exp2f(t.x - mu);
#pragma unroll
        for (int u = 0; u < JOIN_AHEAD; u++)
          t.y = fmaf(ml[u].y, __builtin_amdgcn_exp2f(ml[u].x - mu), t.y);
        t.x = m2;
      }
      for (int o = 16; o; o >>= 1)
        t = join_ml(t, make_float2(__shfl_xor(t.x, o, 32), __shfl_xor(t.y, o, 32)));
      if ((tid & 31) == 0)
        s_ml[h] = make_float2(t.x == -INFINITY ? 0.f : t.x, t.y == 0.f ? 0.f : 1.f / (t.y * (float)a.H));
    }
    __syncthreads();
    for (int x0 = first; x0 < vis.nv; x0 += chunks * 1024) {
      const int x = x0 + (wave & 3) * 256 + lane * 4;
      f32x4_t w = {0.f, 0.f, 0.f, 0.f};
      for (int h = h0; h < nh; h += 4 * JOIN_AHEAD) {
        if (x0 != first || h != h0) load_scores(x, hc + h, s);
#pragma unroll
        for (int u = 0; u < JOIN_AHEAD; u++) {
          const float2 ml = s_ml[min(h + 4 * u, nh - 1)];
          const float r = h + 4 * u < nh ? ml.y : 0.f;
#pragma unroll
          for (int j = 0; j < 4; j++) w[j] = fmaf(__builtin_amdgcn_exp2f(s[u][j] - ml.x), r, w[j]);
        }
      }
      *(f32x4_t*)&part[wave][lane * 4] = w;
      __syncthreads();
      const int xt = x0 + tid;
      if (xt < vis.nv && vis.by_position(c.pos + (int64_t)b * c.cap, xt, a.sinks)) {
        const int t = tid >> 8, i = tid & 255;
        float* w = c.weight + (int64_t)b * c.cap + vis.slot(xt);
        *w = (x0 == first ? weight : *w) +
             ((part[t][i] + part[4 + t][i]) + (part[8 + t][i] + part[12 + t][i]));
      }
      __syncthreads();
    }
  }
}

// Layout of the workspace; `space` null: its size alone.
// (4 bits: large enough for tiles of either kind)
template <typename T, bool FOUR>
size_t paged_space(const CacheArgs& c, int H, int accumulate, char* ws, PagedSpace* space, int KT) {
  PagedSpace p{};
  const int group = H / c.Hkv, DP = c.dh <= 64 ? 64 : 128;
  p.qtiles = (group + 15) / 16;
  p.units = c.Hkv * p.qtiles;
  const bool split = c.B <= PAGED_SPLIT;
  // (4 bits: by four_waves also where paged4_flat runs with fewer, flat_waves: of bf16
  // queries of more than 4 heads a key head, wider than 64, two of three parts run at once)
  const int waves = FOUR ? 1024 * (DP == 64 ? four_waves<T, 64>() : four_waves<T, 128>())
                         : DP == 64 ? PAGED_WAVES_64 : PAGED_WAVES;
  p.ranges = split ? std::max(1, waves / p.units) : c.B;
  p.tiles = (c.cap + KT - 1) / KT;
  const int64_t most = FOUR ? FLAT_KT : KT;
  p.heads = std::min(group, 16);
  p.by_group = fast_div((uint32_t)group);
  const size_t parts = (size_t)p.ranges + (split ? c.B : 0);
  size_t n = 0;
  auto take = [&](size_t bytes) {
    const size_t at = n;
    n += round256(bytes);
    return ws + at;
  };
  p.plan = (int2*)take((size_t)c.B * 8);
  p.ml = (float2*)take(parts * H * 8);
  p.o = (float*)take(parts * H * DP * 4);
  p.score = (float*)take(accumulate ? (size_t)c.B * p.units * p.heads * ((c.cap + most - 1) / most * most) * 4 : 0);
  if (space) *space = p;
  return n;
}

template <typename T, int DP, bool PAD, bool SEL>
void launch_flat(const CacheArgs& c, const PagedArgs& a, const PagedSpace& w, unsigned grid, hipStream_t s) {
  auto with = [&](auto acc, auto r) {
    constexpr bool ACC = decltype(acc)::value;
    constexpr int R = decltype(r)::value;
    if (c.page.d % FLAT_KT == 0)
      paged4_flat<T, DP, PAD, ACC, SEL, R, true><<<grid, 256, 0, s>>>(c, a, w);
    else
      paged4_flat<T, DP, PAD, ACC, SEL, R, false><<<grid, 256, 0, s>>>(c, a, w);
  };
  auto by_group = [&](auto acc) {  // (more query heads than 16 make tiles of 16)
    if (a.group <= 4) with(acc, std::integral_constant<int, 4>{});
    else if (a.group <= 8) with(acc, std::integral_constant<int, 2>{});
    else with(acc, std::integral_constant<int, 1>{});
  };
  if constexpr (!SEL) {
    if (a.accumulate) return by_group(std::true_type{});
  }
  by_group(std::false_type{});
}

template <typename T, bool FOUR> int paged_tile(const PagedArgs& a) {
  return FOUR && a.flat ? FLAT_KT : tile_tokens<T, FOUR>();
}

template <typename T, int DP, bool PAD, bool FOUR, bool SEL>
hipError_t launch_paged(const CacheArgs& c, const PagedArgs& a, const PagedSpace& ws,
                        hipStream_t s) {
  PagedSpace w = ws;
  if (hipError_t e = in_launches(((int64_t)ws.units * ws.ranges + 3) / 4, 256, [&](int first, unsigned grid) {
        w.block0 = first;
        if constexpr (FOUR) {
          if (a.flat) {
            launch_flat<T, DP, PAD, SEL>(c, a, w, grid, s);
            return;
          }
        }
        if constexpr (!SEL) {
          if (a.accumulate) {
            paged_attention<T, DP, PAD, true, FOUR, SEL><<<grid, 256, 0, s>>>(c, a, w);
            return;
          }
        }
        paged_attention<T, DP, PAD, false, FOUR, SEL><<<grid, 256, 0, s>>>(c, a, w);
      }))
    return e;
  // (workgroups past a sequence's tokens leave at once)
  const int chunks = a.accumulate ? std::max(1, std::min((c.cap + 1023) / 1024, 16384 / c.B)) : 1;
  const int weights = a.accumulate ? c.B * chunks : 0;
  // waves a row: enough for the parts of an average sequence in one go, and
  // two at least, since one sequence may have most of them
  const int parts = c.B <= PAGED_SPLIT ? ws.ranges / c.B + 1 : 1;
  const int wpr = parts <= 2 * JOIN_AHEAD ? 2 : parts <= 4 * JOIN_AHEAD ? 4 : 16;
  const int64_t rows = ((int64_t)c.B * a.H * wpr + 15) / 16;
  return in_launches(weights + rows, 1024, [&](int first, unsigned grid) {
    w.block0 = first;
    if constexpr (FOUR) {
      if (a.flat) {
        paged_join<T, DP, FLAT_KT, FOUR, SEL><<<grid, 1024, 0, s>>>(c, a, w, (int)rows, chunks, wpr);
        return;
      }
    }
    paged_join<T, DP, tile_tokens<T, FOUR>(), FOUR, SEL><<<grid, 1024, 0, s>>>(c, a, w, (int)rows, chunks, wpr);
  });
}

template <typename T, bool FOUR, bool SEL>
hipError_t launch_paged_by_width(const CacheArgs& c, const PagedArgs& a, const PagedSpace& ws, hipStream_t s) {
  if (c.dh == 64) return launch_paged<T, 64, false, FOUR, SEL>(c, a, ws, s);
  if (c.dh < 64) return launch_paged<T, 64, true, FOUR, SEL>(c, a, ws, s);
  if (c.dh == 128) return launch_paged<T, 128, false, FOUR, SEL>(c, a, ws, s);
  return launch_paged<T, 128, true, FOUR, SEL>(c, a, ws, s);
}
}  // namespace
}  // namespace fusion
