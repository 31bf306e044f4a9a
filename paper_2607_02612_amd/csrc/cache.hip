// Paged token caches: appending rows, attention of one new token per sequence
// with the accumulated attention weight of every cached token, and eviction
// by that weight.
#include "kernels.h"

#include <algorithm>
#include <type_traits>

namespace fusion {
namespace {

size_t round256(size_t v) { return (v + 255) & ~(size_t)255; }

// Page of a sequence's slot, or -1 where the table holds none.
__device__ __forceinline__ int page_of(const CacheArgs& c, int b, uint32_t pg) {
  const int p = c.table[(int64_t)b * c.max_pages + pg];
  return (unsigned)p < (unsigned)c.pages ? p : -1;
}
__device__ __forceinline__ int held(const CacheArgs& c, int b) {
  return max(0, min(c.len[b], c.cap));
}

// 16-byte pieces of the rows of a token's key heads (or value heads).
struct RowPieces {
  int per_head, all;
};
template <typename T>
__device__ __forceinline__ RowPieces row_pieces(const CacheArgs& c) {
  const int p = c.dh * (int)sizeof(T) / 16;
  return {p, p * c.Hkv};
}
// Address of a piece of a cached row.
template <typename T>
__device__ __forceinline__ uint4* piece(void* base, int64_t page_stride, int64_t row_stride,
                                        int64_t head_stride, int page, int place, int h, int d) {
  return (uint4*)((T*)base + page * page_stride + place * row_stride + h * head_stride) + d;
}

// Offsets of the samples of one launch as kernel arguments.
constexpr int APPEND_SEQS = 256;
struct AppendSeqs {
  int n, first;  // samples, the first one's index
  int cu[APPEND_SEQS + 1];
};
struct OneRowEach {};

// --------------------------------------------------------------- append --
// Row r of sample i goes to slot len + r - cu[i]: a copy, bound by its bytes.
// A wave copies whole rows in 16-byte pieces.  With few rows a sample, one
// workgroup takes a sample's rows and moves its lengths on; else the lengths
// move in a launch of their own, after all rows have read them.
constexpr int APPEND_FEW = 8;  // rows of a sample up to which one workgroup takes them

template <typename T>
__device__ __forceinline__ void append_row(const CacheArgs& c, const AppendArgs& a, int b, int r,
                                           int64_t slot, int pos, int lane, int step) {
  if (slot >= c.cap) return;
  if (lane == 0) {
    c.weight[(int64_t)b * c.cap + slot] = 0.f;
    c.pos[(int64_t)b * c.cap + slot] = pos;
  }
  const uint32_t pg = quot((uint32_t)slot, c.page);
  const int page = page_of(c, b, pg), place = (int)(slot - (int64_t)pg * c.page.d);
  if (page < 0) return;
  const RowPieces rp = row_pieces<T>(c);
  for (int t = lane; t < rp.all; t += step) {
    const int h = t / rp.per_head, d = t - h * rp.per_head;
    const uint4 k = ((const uint4*)((const T*)a.k + r * a.k_row + h * a.k_head))[d];
    const uint4 v = ((const uint4*)((const T*)a.v + r * a.v_row + h * a.v_head))[d];
    *piece<T>(c.k, c.k_page, c.k_row, c.k_head, page, place, h, d) = k;
    *piece<T>(c.v, c.v_page, c.v_row, c.v_head, page, place, h, d) = v;
  }
}

// One workgroup per sample (Seqs: AppendSeqs, or OneRowEach).
template <typename T, typename Seqs>
__global__ __launch_bounds__(256) void append_few(CacheArgs c, AppendArgs a, Seqs sq) {
  int b = blockIdx.x, r0 = b, n = 1;
  if constexpr (std::is_same<Seqs, AppendSeqs>::value) {
    b += sq.first;
    r0 = sq.cu[blockIdx.x];
    n = sq.cu[blockIdx.x + 1] - r0;
  }
  const int have = held(c, b), seen = c.seen[b];
  __syncthreads();  // all waves have the lengths
  if (threadIdx.x == 0 && n > 0) {
    const int fit = min(n, c.cap - have);
    c.len[b] = have + fit;
    c.seen[b] = seen + fit;
  }
  if (n == 1) {
    append_row<T>(c, a, b, r0, have, seen, threadIdx.x, 256);
  } else {
    for (int i = threadIdx.x >> 6; i < n; i += 4)
      append_row<T>(c, a, b, r0 + i, (int64_t)have + i, seen + i, threadIdx.x & 63, 64);
  }
}

template <typename T>
__global__ __launch_bounds__(256) void append_many(CacheArgs c, AppendArgs a, AppendSeqs sq) {
  const int r = sq.cu[0] + blockIdx.x * 4 + (threadIdx.x >> 6);
  if (r >= sq.cu[sq.n]) return;
  int lo = 0, hi = sq.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (sq.cu[mid] <= r) lo = mid; else hi = mid - 1;
  }
  const int b = sq.first + lo, nth = r - sq.cu[lo];
  append_row<T>(c, a, b, r, (int64_t)held(c, b) + nth, c.seen[b] + nth, threadIdx.x & 63, 64);
}

__global__ __launch_bounds__(256) void append_lengths(CacheArgs c, AppendSeqs sq) {
  const int t = blockIdx.x * 256 + threadIdx.x;
  if (t >= sq.n) return;
  const int b = sq.first + t, have = held(c, b), fit = min(sq.cu[t + 1] - sq.cu[t], c.cap - have);
  if (sq.cu[t + 1] == sq.cu[t]) return;
  c.len[b] = have + fit;
  c.seen[b] += fit;
}

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
// not arise.
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
constexpr int PAGED_WAVES = 2048;  // parts in all, about

struct PagedSpace {
  int2* plan;    // [B]: first part, number of parts
  float2* ml;    // [parts][H]: maximum (base 2), sum
  float* o;      // [parts][H][DP]
  float* score;  // [B][tiles][H][KT], base 2, by visible token
  int ranges;    // parts per unit
  int units, qtiles, tiles;
};

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
};
__device__ __forceinline__ Visible visible(const CacheArgs& c, const PagedArgs& a, int b) {
  Visible v;
  v.n = v.nv = held(c, b);
  const int seen = c.seen[b];
  v.head = v.gap = 0;
  v.by_pos = a.window < kNoWindow && seen != v.n;
  v.oldest = (int)max((int64_t)seen - a.window, (int64_t)INT32_MIN);
  if (a.window < kNoWindow && !v.by_pos && v.n - a.window > a.sinks) {
    v.head = a.sinks;
    v.nv = a.sinks + a.window;
    v.gap = v.n - v.nv;
  }
  return v;
}

template <typename T, int DP, bool PAD, bool ACC>
__global__ __launch_bounds__(256, 2) void paged_attention(CacheArgs c, PagedArgs a, PagedSpace ws) {
  constexpr bool BF = sizeof(T) == 2;
  constexpr int KT = BF ? 32 : 16, NSUB = KT / 16;
  constexpr int EPP = 16 / sizeof(T);       // values per 16-byte piece
  constexpr int NL = DP / EPP / 4;          // pieces per lane and token
  constexpr int ND = DP / 16;
  constexpr int VROW = BF ? DP * 2 : (DP + 4) * 4;  // bytes of a token's values in LDS
  __shared__ __attribute__((aligned(16))) char v_all[4 * KT * VROW];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int g = lane >> 4, cl = lane & 15;
  const int id = blockIdx.x * 4 + wave, unit = id % ws.units, range = id / ws.units;
  if (range >= ws.ranges) return;
  char* Vs = v_all + wave * KT * VROW;
  const int kh = unit / ws.qtiles, qt = unit % ws.qtiles;
  const int h0 = kh * a.group + qt * 16, nq = min(16, a.group - qt * 16);
  const int dh = c.dh;
  const float sc2 = a.scale * kLog2e;

  auto segment = [&](int b, int ta, int tb, int part) {
    Visible vis = visible(c, a, b);
    vis.nv = __builtin_amdgcn_readfirstlane(vis.nv);
    vis.head = __builtin_amdgcn_readfirstlane(vis.head);
    vis.gap = __builtin_amdgcn_readfirstlane(vis.gap);
    vis.oldest = __builtin_amdgcn_readfirstlane(vis.by_pos ? vis.oldest : INT32_MIN);
    // Q^T operand
    uint4 q[NL];
#pragma unroll
    for (int s = 0; s < NL; s++) {
      q[s] = make_uint4(0, 0, 0, 0);
      const int d = (4 * s + g) * EPP;
      if (cl < nq && (!PAD || d < dh))
        q[s] = *(const uint4*)((const T*)a.q + (int64_t)b * a.q_row + (int64_t)(h0 + cl) * a.q_head + d);
    }
    const int* table = c.table + (int64_t)b * c.max_pages;
    // (positions that decide nothing are read from the table's line)
    const int* pos = vis.oldest == INT32_MIN ? table : c.pos + (int64_t)b * c.cap;
    const bool by_pos = vis.oldest != INT32_MIN;
    // page, place and position of the lane's tokens of a tile
    struct Tokens {
      int page[NSUB], place[NSUB], at[NSUB];
    };
    auto look_up = [&](int t) {
      Tokens k;
#pragma unroll
      for (int u = 0; u < NSUB; u++) {
        const int x = vis.slot(min(t * KT + 16 * u + cl, vis.nv - 1));
        const uint32_t pg = quot((uint32_t)x, c.page);
        k.page[u] = table[pg];
        k.place[u] = x - (int)(pg * c.page.d);
        k.at[u] = pos[by_pos ? (uint32_t)x : pg];
      }
      return k;
    };
    // keys and values of the lane's tokens; hidden ones read the cache's first row
    uint4 kr[NSUB][NL], vr[NSUB][NL];
    uint32_t mask_next;  // visible tokens of the tile, one bit each
    bool see[NSUB];
    const T* kp[NSUB];
    const T* vp[NSUB];
    auto point = [&](int t, const Tokens& tk) {
      mask_next = 0;
#pragma unroll
      for (int u = 0; u < NSUB; u++) {
        see[u] = (t * KT + 16 * u + cl < vis.nv) & ((unsigned)tk.page[u] < (unsigned)c.pages) &
                 ((tk.at[u] >= vis.oldest) | (tk.at[u] < a.sinks));
        mask_next |= (uint32_t)(__ballot(see[u]) & 0xFFFF) << (16 * u);
        const int64_t p = see[u] ? tk.page[u] : 0, r = see[u] ? tk.place[u] : 0;
        kp[u] = (const T*)c.k + p * c.k_page + r * c.k_row + kh * c.k_head;
        vp[u] = (const T*)c.v + p * c.v_page + r * c.v_row + kh * c.v_head;
      }
    };
    auto load_kv = [&]() {
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
    // Scores of a tile to the workspace, `n` of the unit's heads (rows past
    // them are past the buffer's end and dropped).
    auto store_scores = [&](int t, const f32x4_t* S, int n) {
      const auto rows = __builtin_amdgcn_make_buffer_rsrc(
          ws.score + (((int64_t)b * ws.tiles + t) * a.H + h0) * KT, 0, n * KT * 4, 0x00027000);
#pragma unroll
      for (int u = 0; u < NSUB; u++)
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, S[u]), rows,
                                               (cl * KT + 16 * u + 4 * g) * 4, 0, 0);
    };
    // One tile in straight line, with its memory operations in a fixed order
    // (look-ups two tiles ahead, the next tile's keys, its values, this tile's
    // scores), so that each wait counts exactly the operations after the one
    // it needs: with a branch or another order every tile waited for its
    // stores too (2 x 131,072 tokens, 32 heads: XXX us).  LAST: no tile follows.
    auto tile = [&](int t, Tokens& ahead, auto last_c) {
      constexpr bool LAST = decltype(last_c)::value;
      const uint32_t mask = mask_next;
      f32x4_t S[NSUB];
#pragma unroll
      for (int u = 0; u < NSUB; u++) {
        S[u] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < NL; s++) {
          if constexpr (BF) {
            S[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, kr[u][s]),
                                                           __builtin_bit_cast(bf16x8_t, q[s]),
                                                           S[u], 0, 0, 0);
          } else {
            const f32x4_t kf = __builtin_bit_cast(f32x4_t, kr[u][s]);
            const f32x4_t qf = __builtin_bit_cast(f32x4_t, q[s]);
#pragma unroll
            for (int i = 0; i < 4; i++)
              S[u] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[i], qf[i], S[u], 0, 0, 0);
          }
        }
      }
#pragma unroll
      for (int u = 0; u < NSUB; u++)
#pragma unroll
        for (int s = 0; s < NL; s++) {
          const uint4 x = vr[u][s];
          const uint4 v = make_uint4(see[u] ? x.x : 0, see[u] ? x.y : 0, see[u] ? x.z : 0,
                                     see[u] ? x.w : 0);
          const int r = 16 * u + cl, p = 4 * s + g;
          if constexpr (BF)
            *(uint4*)(Vs + r * VROW + (((p >> 1) ^ (r & (DP / 16 - 1))) << 5) + ((p & 1) << 4)) = v;
          else
            *(uint4*)(Vs + r * VROW + p * 16) = v;
        }
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (!LAST) {
        point(t + 1, ahead);
        __builtin_amdgcn_sched_barrier(0);
        ahead = look_up(min(t + 2, tb - 1));
        __builtin_amdgcn_sched_barrier(0);
        load_kv();
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int u = 0; u < NSUB; u++)
#pragma unroll
        for (int j = 0; j < 4; j++)
          S[u][j] = mask >> (16 * u + 4 * g + j) & 1 ? S[u][j] * sc2 : -INFINITY;
      if constexpr (ACC) store_scores(t, S, nq);
      float mt = fmaxf(fmaxf(S[0][0], S[0][1]), fmaxf(S[0][2], S[0][3]));
      if (NSUB > 1)
        mt = fmaxf(mt, fmaxf(fmaxf(S[NSUB - 1][0], S[NSUB - 1][1]), fmaxf(S[NSUB - 1][2], S[NSUB - 1][3])));
      mt = max_xor32(max_xor16(mt));
      const bool grow = mt > m + 8.f;
      const float f = grow ? __builtin_amdgcn_exp2f(m - mt) : 1.f;
      m = grow ? mt : m;
      l *= f;
#pragma unroll
      for (int d = 0; d < ND; d++)
#pragma unroll
        for (int j = 0; j < 4; j++) O[d][j] *= f;
      const float mu = m == -INFINITY ? 0.f : m;
#pragma unroll
      for (int u = 0; u < NSUB; u++) {
#pragma unroll
        for (int j = 0; j < 4; j++) S[u][j] = __builtin_amdgcn_exp2f(S[u][j] - mu);
        l += (S[u][0] + S[u][1]) + (S[u][2] + S[u][3]);
      }
      if constexpr (BF) {
        // P as the sum of two bf16 numbers, 16 bits of precision: the second
        // product costs nothing beside the loads
        union { uint32_t u[4]; bf16x8_t v; } p, p2;
#pragma unroll
        for (int w = 0; w < 4; w++) {
          const float e0 = S[w / 2 * (NSUB - 1)][w % 2 * 2], e1 = S[w / 2 * (NSUB - 1)][w % 2 * 2 + 1];
          p.u[w] = pack_bf16x2(e0, e1);
          p2.u[w] = pack_bf16x2(e0 - __uint_as_float(p.u[w] << 16),
                                e1 - __uint_as_float(p.u[w] & 0xFFFF0000u));
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
                    Vs + r * VROW + ((d ^ (r & (DP / 16 - 1))) << 5) + ((cl & 3) << 3)));
          }
          O[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf.v, p.v, O[d], 0, 0, 0);
          O[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf.v, p2.v, O[d], 0, 0, 0);
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
    Tokens ahead = look_up(ta);
    point(ta, ahead);
    ahead = look_up(min(ta + 1, tb - 1));
    load_kv();
    if constexpr (ACC) {
      // (stores of nothing, so that the first tile finds as many as the others)
      const f32x4_t none[2] = {};
      store_scores(ta, none, 0);
    }
    for (int t = ta; t < tb - 1; t++) tile(t, ahead, std::false_type{});
    tile(tb - 1, ahead, std::true_type{});
    l = sum_xor32(sum_xor16(l));
    if (cl < nq) {
      const int64_t o = (int64_t)part * a.H + h0 + cl;
      if (g == 0) ws.ml[o] = make_float2(m, l);
#pragma unroll
      for (int d = 0; d < ND; d++) *(f32x4_t*)(ws.o + o * DP + 16 * d + 4 * g) = O[d];
    }
  };

  // the sequences whose tiles form the line: all, or the part's own
  const bool split = c.B <= PAGED_SPLIT;
  const int b0 = split ? 0 : range, b1 = split ? c.B : range + 1;
  auto tiles_of = [&](int b) { return b < b1 ? (visible(c, a, b).nv + KT - 1) / KT : 0; };
  int total = 0;
  for (int b = b0; b < b1; b += 64)
    total += __builtin_amdgcn_readfirstlane(wave_sum_i(tiles_of(b + lane)));
  const int per = max(1, split ? (total + ws.ranges - 1) / ws.ranges : total);
  const int first = split ? range * per : 0, last = min(first + per, total);
  const bool planner = unit == 0 && (range == 0 || !split);
  if (first >= total && !planner) return;
  int before = 0;  // tiles of the sequences before b
  for (int b = b0; b < b1 && (before < last || planner); b += 64) {
    const int t = tiles_of(b + lane);
    int p = t;  // inclusive, then exclusive sum over the lanes
    for (int o = 1; o < 64; o <<= 1) {
      const int v = __shfl_up(p, o, 64);
      if (lane >= o) p += v;
    }
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

// The parts of every sequence joined: the first workgroups write the output
// rows, four each (4 waves a row), the others add the weights of 1024 visible
// tokens of a sequence: 4 tokens a lane, a fourth of the heads a wave, summed
// over the waves in order.  Loads go out JOIN_AHEAD at a time, since a
// sequence of the chip alone has hundreds of parts (two of 131,072 tokens took
// 37 us with one row of parts after the other).
constexpr int JOIN_HEADS = 128;
constexpr int JOIN_AHEAD = 8;
template <typename T, int DP>
__global__ __launch_bounds__(1024) void paged_join(CacheArgs c, PagedArgs a, PagedSpace ws,
                                                   int rows, int chunks) {
  constexpr int KT = sizeof(T) == 2 ? 32 : 16;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  __shared__ __attribute__((aligned(16))) float part[16][256];
  __shared__ float2 s_ml[JOIN_HEADS];
  if (blockIdx.x < rows) {
    const int64_t row = (int64_t)blockIdx.x * 4 + (wave >> 2);
    const bool real = row < (int64_t)c.B * a.H;
    const int b = real ? (int)(row / a.H) : 0, h = real ? (int)(row % a.H) : 0, w4 = wave & 3;
    const int2 plan = ws.plan[b];
    float m = -INFINITY;
    for (int i = lane; i < plan.y; i += 64)
      m = fmaxf(m, ws.ml[(int64_t)(plan.x + i) * a.H + h].x);
    m = wave_max(m);
    const float mu = m == -INFINITY ? 0.f : m;
    float o0 = 0.f, o1 = 0.f, l = 0.f;
    for (int i = w4; i < plan.y; i += 4 * JOIN_AHEAD) {
      float2 ml[JOIN_AHEAD];
      float x0[JOIN_AHEAD], x1[JOIN_AHEAD];
#pragma unroll
      for (int u = 0; u < JOIN_AHEAD; u++) {
        const int64_t p = (int64_t)(plan.x + min(i + 4 * u, plan.y - 1)) * a.H + h;
        ml[u] = ws.ml[p];
        x0[u] = ws.o[p * DP + lane];
        x1[u] = DP > 64 ? ws.o[p * DP + 64 + lane] : 0.f;
      }
#pragma unroll
      for (int u = 0; u < JOIN_AHEAD; u++) {
        const float f = i + 4 * u < plan.y ? __builtin_amdgcn_exp2f(ml[u].x - mu) : 0.f;
        l = fmaf(ml[u].y, f, l);
        o0 = fmaf(x0[u], f, o0);
        o1 = fmaf(x1[u], f, o1);
      }
    }
    part[wave][lane] = o0;
    if (DP > 64) part[wave][64 + lane] = o1;
    if (lane == 0) s_ml[wave].y = l;
    __syncthreads();
    const int d = tid & 255, w = wave & ~3;  // a row's first wave
    l = (s_ml[w].y + s_ml[w + 1].y) + (s_ml[w + 2].y + s_ml[w + 3].y);
    if (real && d < c.dh) {
      const float o = (part[w][d] + part[w + 1][d]) + (part[w + 2][d] + part[w + 3][d]);
      ((T*)a.out)[row * c.dh + d] = St<T>::put(l == 0.f ? 0.f : o / l);
    }
    return;
  }
  const int64_t id = (int64_t)blockIdx.x - rows;
  const int b = (int)(id / chunks), first = (int)(id % chunks) * 1024;
  const Visible vis = visible(c, a, b);
  if (first >= vis.nv) return;
  const int2 plan = ws.plan[b];
  for (int hc = 0; hc < a.H; hc += JOIN_HEADS) {
    const int nh = min(JOIN_HEADS, a.H - hc);
    __syncthreads();
    // maximum and 1 / (sum H) of the heads, 32 lanes a head
    for (int h = tid >> 5; h < nh; h += 32) {
      float m = -INFINITY, l = 0.f;
      for (int i = tid & 31; i < plan.y; i += 32 * JOIN_AHEAD) {
        float2 ml[JOIN_AHEAD];
        float m2 = m;
#pragma unroll
        for (int u = 0; u < JOIN_AHEAD; u++) {
          ml[u] = ws.ml[(int64_t)(plan.x + min(i + 32 * u, plan.y - 1)) * a.H + hc + h];
          if (i + 32 * u >= plan.y) ml[u].x = -INFINITY;
        }
#pragma unroll
        for (int u = 0; u < JOIN_AHEAD; u++) m2 = fmaxf(m2, ml[u].x);
        if (m2 != -INFINITY) {
          l *= __builtin_amdgcn_exp2f(m - m2);
#pragma unroll
          for (int u = 0; u < JOIN_AHEAD; u++) l = fmaf(ml[u].y, __builtin_amdgcn_exp2f(ml[u].x - m2), l);
        }
        m = m2;
      }
      for (int o = 16; o; o >>= 1) {
        const float mo = __shfl_xor(m, o, 32), lo = __shfl_xor(l, o, 32), m2 = fmaxf(m, mo);
        if (m2 != -INFINITY)
          l = l * __builtin_amdgcn_exp2f(m - m2) + lo * __builtin_amdgcn_exp2f(mo - m2);
        m = m2;
      }
      if ((tid & 31) == 0)
        s_ml[h] = make_float2(m == -INFINITY ? 0.f : m, l == 0.f ? 0.f : 1.f / (l * (float)a.H));
    }
    __syncthreads();
    for (int x0 = first; x0 < vis.nv; x0 += chunks * 1024) {
      const int x = x0 + (wave & 3) * 256 + lane * 4, h0 = wave >> 2;
      f32x4_t w = {0.f, 0.f, 0.f, 0.f};
      if (x < vis.nv) {
        const float* sp = ws.score + (((int64_t)b * ws.tiles + x / KT) * a.H + hc) * KT + x % KT;
        for (int h = h0; h < nh; h += 4 * JOIN_AHEAD) {
          f32x4_t s[JOIN_AHEAD];
#pragma unroll
          for (int u = 0; u < JOIN_AHEAD; u++) s[u] = *(const f32x4_t*)(sp + min(h + 4 * u, nh - 1) * KT);
#pragma unroll
          for (int u = 0; u < JOIN_AHEAD; u++) {
            const float2 ml = s_ml[min(h + 4 * u, nh - 1)];
            const float r = h + 4 * u < nh ? ml.y : 0.f;
#pragma unroll
            for (int j = 0; j < 4; j++) w[j] = fmaf(__builtin_amdgcn_exp2f(s[u][j] - ml.x), r, w[j]);
          }
        }
      }
      *(f32x4_t*)&part[wave][lane * 4] = w;
      __syncthreads();
      const int xt = x0 + tid;
      if (xt < vis.nv) {
        const int t = tid >> 8, i = tid & 255;
        c.weight[(int64_t)b * c.cap + vis.slot(xt)] +=
            (part[t][i] + part[4 + t][i]) + (part[8 + t][i] + part[12 + t][i]);
      }
      __syncthreads();
    }
  }
}

// -------------------------------------------------------------- evict --
// Order of the tokens as unsigned integers: protected tokens above all, then
// by weight (-0 equals 0), NaN below everything.
__device__ __forceinline__ uint32_t keep_key(float w, bool safe) {
  if (safe) return 0xFFFFFFFFu;
  if (w != w) return 0u;
  const uint32_t u = __float_as_uint(w + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

struct EvictSpace {
  int* moves;   // [B]
  int2* move;   // [B][room]: (free slot, kept slot beyond the budget)
  int room;     // most moves of a sequence
};

template <typename T>
__device__ __forceinline__ void move_row(const CacheArgs& c, int b, int2 m, int lane, int step) {
  const uint32_t pd = quot(m.x, c.page), ps = quot(m.y, c.page);
  const int to = page_of(c, b, pd), from = page_of(c, b, ps);
  if (to < 0 || from < 0) return;
  const int rd = m.x - (int)(pd * c.page.d), rs = m.y - (int)(ps * c.page.d);
  const RowPieces rp = row_pieces<T>(c);
  for (int t = lane; t < rp.all; t += step) {
    const int h = t / rp.per_head, d = t - h * rp.per_head;
    const uint4 k = *piece<T>(c.k, c.k_page, c.k_row, c.k_head, from, rs, h, d);
    const uint4 v = *piece<T>(c.v, c.v_page, c.v_row, c.v_head, from, rs, h, d);
    *piece<T>(c.k, c.k_page, c.k_row, c.k_head, to, rd, h, d) = k;
    *piece<T>(c.v, c.v_page, c.v_row, c.v_head, to, rd, h, d) = v;
  }
}

// The choice, one workgroup of NT threads per sequence.  The budget-th largest
// key is found from the top by digits of 12, 10 and 10 bits: counts of the
// keys that share the digits found so far in bins, a sum over the bins from
// the highest, the bin where it reaches the rank.  (The first digit holds the
// sign, the exponent and three bits of the weight, so that weights of similar
// size meet in few bins: the counts are LDS atomics, and lanes that hit one
// address wait for each other.)  Each thread holds E neighbouring slots' keys
// in registers, of longer sequences one chunk of NT E slots after the other,
// read again in every round.  Then one pass in slot order lists the free
// slots below the budget and hands them to the kept ones beyond it.  Bound by
// the rounds' latency (barriers, bins); 64 sequences of 4,097 slots are read
// in 0.5 us.
constexpr int EVICT_BINS = 4096;
constexpr int EVICT_FEW = 32;  // moves that the choosing workgroup makes itself
template <typename T, int NT, int E>
__global__ __launch_bounds__(NT) void evict_select(CacheArgs c, EvictArgs a, EvictSpace ws) {
  constexpr int NW = NT / 64;
  const int b = blockIdx.x, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int n = held(c, b), seen = c.seen[b];
  float* weight = c.weight + (int64_t)b * c.cap;
  int* pos = c.pos + (int64_t)b * c.cap;
  int* src = a.src + (int64_t)b * a.budget;
  for (int x = tid; x < a.budget; x += NT) src[x] = x < n ? x : -1;
  if (n <= a.budget) {
    if (tid == 0) {
      ws.moves[b] = 0;
      c.len[b] = n;
    }
    return;
  }
  __shared__ int bins[EVICT_BINS];
  __shared__ int s_found[2], s_wave[2][NW];
  // exclusive sum over the workgroup's threads (two values at once)
  auto scan = [&](int u, int v, int* before_u, int* before_v, int* total_u, int* total_v) {
    int iu = u, iv = v;
    for (int o = 1; o < 64; o <<= 1) {
      const int tu = __shfl_up(iu, o, 64), tv = __shfl_up(iv, o, 64);
      if (lane >= o) {
        iu += tu;
        iv += tv;
      }
    }
    __syncthreads();
    if (lane == 63) {
      s_wave[0][wave] = iu;
      s_wave[1][wave] = iv;
    }
    __syncthreads();
    int bu = 0, bv = 0, au = 0, av = 0;
    for (int w = 0; w < NW; w++) {
      const int tu = s_wave[0][w], tv = s_wave[1][w];
      if (w < wave) {
        bu += tu;
        bv += tv;
      }
      au += tu;
      av += tv;
    }
    *before_u = bu + iu - u;
    *before_v = bv + iv - v;
    *total_u = au;
    *total_v = av;
  };
  uint32_t key[E];
  const int chunks = (n + NT * E - 1) / (NT * E);
  auto load = [&](int ch) {
#pragma unroll
    for (int e = 0; e < E; e++) {
      const int x = min((ch * NT + tid) * E + e, n - 1), p = pos[x];
      key[e] = keep_key(weight[x], p < a.sinks || seen - p <= a.recent);
    }
  };
  load(0);
  uint32_t prefix = 0;
  int want = a.budget;  // rank of the key searched, among those with the prefix
  constexpr int SHIFT[3] = {20, 10, 0};
#pragma unroll
  for (int round = 0; round < 3; round++) {
    const int shift = SHIFT[round], nb = round ? 1024 : 4096;
    const int per = nb / NT;  // bins per thread
    for (int i = tid; i < nb; i += NT) bins[i] = 0;
    __syncthreads();
    for (int ch = 0; ch < chunks; ch++) {
      if (chunks > 1 && (ch || round)) load(ch);
#pragma unroll
      for (int e = 0; e < E; e++)
        if ((ch * NT + tid) * E + e < n &&
            (round == 0 || key[e] >> (shift + 10) == prefix >> (shift + 10)))
          atomicAdd(&bins[key[e] >> shift & (nb - 1)], 1);
    }
    __syncthreads();
    // thread t sums bins nb - 1 - t per .. down
    int mine = 0;
    for (int i = 0; i < per; i++) mine += bins[nb - 1 - tid * per - i];
    int above, unused0, unused1, unused2;
    scan(mine, 0, &above, &unused0, &unused1, &unused2);
    if (above < want && above + mine >= want) {
      int i = nb - 1 - tid * per, left = want - above;
      for (; left > bins[i]; i--) left -= bins[i];
      s_found[0] = i;
      s_found[1] = left;
    }
    __syncthreads();
    prefix |= (uint32_t)s_found[0] << shift;
    want = s_found[1];
    __syncthreads();
  }
  // keys above `prefix` stay, and the first `want` equal to it
  int ties = 0, holes = 0, late = 0;
  int2* mv = ws.move + (int64_t)b * ws.room;
  for (int ch = 0; ch < chunks; ch++) {
    if (chunks > 1) load(ch);
    const int x0 = (ch * NT + tid) * E;
    int tie = 0;
#pragma unroll
    for (int e = 0; e < E; e++) tie += x0 + e < n && key[e] == prefix;
    int rank, unused, more, unused2;
    scan(tie, 0, &rank, &unused, &more, &unused2);
    rank += ties;
    ties += more;
    uint64_t free = 0, over = 0;  // the thread's free slots, kept slots beyond the budget
    static_assert(E <= 64, "one bit per slot");
#pragma unroll
    for (int e = 0; e < E; e++) {
      if (x0 + e >= n) continue;
      const bool eq = key[e] == prefix, keep = key[e] > prefix || (eq && rank < want);
      rank += eq;
      if (x0 + e < a.budget && !keep) free |= 1ull << e;
      if (x0 + e >= a.budget && keep) over |= 1ull << e;
    }
    int hi, li, nh, nl;
    scan(__popcll(free), __popcll(over), &hi, &li, &nh, &nl);
    for (hi += holes; free; free &= free - 1) mv[hi++].x = x0 + __builtin_ctzll(free);
    for (li += late; over; over &= over - 1) mv[li++].y = x0 + __builtin_ctzll(over);
    holes += nh;
    late += nl;
  }
  __syncthreads();
  for (int i = tid; i < holes; i += NT) {
    const int2 m = mv[i];
    weight[m.x] = weight[m.y];
    pos[m.x] = pos[m.y];
    src[m.x] = m.y;
  }
  if (ws.room <= EVICT_FEW)
    for (int i = wave; i < holes; i += NW) move_row<T>(c, b, mv[i], lane, 64);
  if (tid == 0) {
    ws.moves[b] = holes;
    c.len[b] = a.budget;
  }
}

// One wave per move.
template <typename T>
__global__ __launch_bounds__(256) void evict_move(CacheArgs c, EvictSpace ws) {
  const int b = blockIdx.x, n = ws.moves[b];
  for (int i = blockIdx.y * 4 + (threadIdx.x >> 6); i < n; i += gridDim.y * 4)
    move_row<T>(c, b, ws.move[(int64_t)b * ws.room + i], threadIdx.x & 63, 64);
}

}  // namespace

template <typename T>
hipError_t launch_cache_append(const CacheArgs& c, const AppendArgs& a, const int32_t* cu_host,
                               hipStream_t s) {
  if (!cu_host) {
    append_few<T><<<c.B, 256, 0, s>>>(c, a, OneRowEach{});
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
    if (rows == 0) continue;
    if (most <= APPEND_FEW) {
      append_few<T><<<sq.n, 256, 0, s>>>(c, a, sq);
    } else {
      append_many<T><<<(rows + 3) / 4, 256, 0, s>>>(c, a, sq);
      append_lengths<<<(sq.n + 255) / 256, 256, 0, s>>>(c, sq);
    }
    if (hipError_t e = hipGetLastError()) return e;
  }
  return hipSuccess;
}
template hipError_t launch_cache_append<float>(const CacheArgs&, const AppendArgs&,
                                               const int32_t*, hipStream_t);
template hipError_t launch_cache_append<bf16_t>(const CacheArgs&, const AppendArgs&,
                                                const int32_t*, hipStream_t);

namespace {
// Layout of the workspace; `space` null: its size alone.
size_t paged_space(const CacheArgs& c, int KT, int H, int accumulate, char* ws,
                   PagedSpace* space) {
  PagedSpace p;
  const int group = H / c.Hkv, DP = c.dh <= 64 ? 64 : 128;
  p.qtiles = (group + 15) / 16;
  p.units = c.Hkv * p.qtiles;
  const bool split = c.B <= PAGED_SPLIT;
  p.ranges = split ? std::max(1, PAGED_WAVES / p.units) : c.B;
  p.tiles = (c.cap + KT - 1) / KT;
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
  p.score = (float*)take(accumulate ? (size_t)c.B * p.tiles * H * KT * 4 : 0);
  if (space) *space = p;
  return n;
}

template <typename T, int DP, bool PAD>
hipError_t launch_paged(const CacheArgs& c, const PagedArgs& a, const PagedSpace& ws,
                        hipStream_t s) {
  const unsigned grid = (unsigned)(((int64_t)ws.units * ws.ranges + 3) / 4);
  if (a.accumulate)
    paged_attention<T, DP, PAD, true><<<grid, 256, 0, s>>>(c, a, ws);
  else
    paged_attention<T, DP, PAD, false><<<grid, 256, 0, s>>>(c, a, ws);
  if (hipError_t e = hipGetLastError()) return e;
  // (workgroups past a sequence's tokens leave at once)
  const int rows = (int)(((int64_t)c.B * a.H + 3) / 4);
  const int chunks = a.accumulate ? std::max(1, std::min((c.cap + 1023) / 1024, 16384 / c.B)) : 0;
  paged_join<T, DP><<<(unsigned)(rows + (int64_t)c.B * chunks), 1024, 0, s>>>(c, a, ws, rows, chunks);
  return hipGetLastError();
}
constexpr int tile_tokens(size_t size) { return size == 2 ? 32 : 16; }
}  // namespace

size_t paged_workspace_bytes(const CacheArgs& c, size_t elem, int H, int accumulate) {
  return paged_space(c, tile_tokens(elem), H, accumulate, nullptr, nullptr);
}

template <typename T>
hipError_t launch_paged_attention(const CacheArgs& c, const PagedArgs& a, hipStream_t s) {
  PagedSpace ws;
  paged_space(c, tile_tokens(sizeof(T)), a.H, a.accumulate, (char*)a.ws, &ws);
  if (c.dh == 64) return launch_paged<T, 64, false>(c, a, ws, s);
  if (c.dh < 64) return launch_paged<T, 64, true>(c, a, ws, s);
  if (c.dh == 128) return launch_paged<T, 128, false>(c, a, ws, s);
  return launch_paged<T, 128, true>(c, a, ws, s);
}
template hipError_t launch_paged_attention<float>(const CacheArgs&, const PagedArgs&, hipStream_t);
template hipError_t launch_paged_attention<bf16_t>(const CacheArgs&, const PagedArgs&, hipStream_t);

static int evict_room(const CacheArgs& c, int budget) {
  return std::max(0, std::min(budget, c.cap - budget));
}
size_t evict_workspace_bytes(const CacheArgs& c, int budget) {
  return round256((size_t)c.B * 4) + (size_t)c.B * evict_room(c, budget) * 8;
}

template <typename T>
hipError_t launch_cache_evict(const CacheArgs& c, const EvictArgs& a, hipStream_t s) {
  const EvictSpace ws{(int*)a.ws, (int2*)((char*)a.ws + round256((size_t)c.B * 4)),
                      evict_room(c, a.budget)};
  if (c.cap <= 1024)
    evict_select<T, 256, 4><<<c.B, 256, 0, s>>>(c, a, ws);
  else if (c.cap <= 4096)
    evict_select<T, 1024, 4><<<c.B, 1024, 0, s>>>(c, a, ws);
  else if (c.cap <= 8192)
    evict_select<T, 1024, 8><<<c.B, 1024, 0, s>>>(c, a, ws);
  else
    evict_select<T, 1024, 16><<<c.B, 1024, 0, s>>>(c, a, ws);
  if (hipError_t e = hipGetLastError()) return e;
  if (ws.room > EVICT_FEW) {
    const int y = std::min((ws.room + 3) / 4, std::max(1, 4096 / c.B));
    evict_move<T><<<dim3(c.B, y), 256, 0, s>>>(c, ws);
  }
  return hipGetLastError();
}
template hipError_t launch_cache_evict<float>(const CacheArgs&, const EvictArgs&, hipStream_t);
template hipError_t launch_cache_evict<bf16_t>(const CacheArgs&, const EvictArgs&, hipStream_t);

}  // namespace fusion
