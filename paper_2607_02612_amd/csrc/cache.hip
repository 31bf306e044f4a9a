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
constexpr int APPEND_BLOCKS = 1 << 22;  // workgroups of a launch (2^32 threads are too many for one)

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
  const int end = sq.cu[sq.n];
  for (int r = sq.cu[0] + blockIdx.x * 4 + (threadIdx.x >> 6); r < end; r += gridDim.x * 4) {
    int lo = 0, hi = sq.n - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (sq.cu[mid] <= r) lo = mid; else hi = mid - 1;
    }
    const int b = sq.first + lo, nth = r - sq.cu[lo];
    append_row<T>(c, a, b, r, (int64_t)held(c, b) + nth, c.seen[b] + nth, threadIdx.x & 63, 64);
  }
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
// not arise.  Of a visible token it does: where a weight underflows, and where
// the second of the two bf16 numbers that stand for it is 0 or negative; the
// join mends it.
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

constexpr int LIST = 512;  // tokens of a part that are gathered at a time

struct PagedSpace {
  int2* plan;    // [B]: first part, number of parts
  float2* ml;    // [parts][H]: maximum (base 2), sum
  float* o;      // [parts][H][DP]
  float* score;  // [B][units][tiles][heads][KT], base 2, by visible token
  int ranges;    // parts per unit
  int units, qtiles, tiles, heads;  // (heads of a unit, at most 16)
  int block0;    // number of the launch's first workgroup
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
  __device__ __forceinline__ bool by_position(const int* pos, int x, int sinks) const {
    return !by_pos || pos[x] >= oldest || pos[x] < sinks;
  }
};
__device__ __forceinline__ Visible visible(const CacheArgs& c, const PagedArgs& a, int b) {
  Visible v;
  v.n = v.nv = held(c, b);
  const int seen = c.seen[b];
  v.head = v.gap = 0;
  v.by_pos = a.window > 0 && seen != v.n;
  v.oldest = (int)max((int64_t)seen - a.window, (int64_t)INT32_MIN);
  if (a.window > 0 && !v.by_pos && v.n - a.window > a.sinks) {
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
  // LDS that a wave's values leave free: scores held back, or a list of tokens
  // (allocated in units of 1280 bytes, 160 KB a CU, for the workgroups that run at once)
  constexpr int SHARE = 160 * 1024 / (DP <= 64 ? 3 : 2) / 1280 * 1280 / 4;
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
    Visible vis = visible(c, a, b);
    vis.nv = __builtin_amdgcn_readfirstlane(vis.nv);
    vis.head = __builtin_amdgcn_readfirstlane(vis.head);
    vis.gap = __builtin_amdgcn_readfirstlane(vis.gap);
    vis.oldest = __builtin_amdgcn_readfirstlane(vis.oldest);
    const bool by_pos = __builtin_amdgcn_readfirstlane(vis.by_pos);
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
    uint4 kr[NSUB][NL], vr[NSUB][NL];
    uint32_t mask_next;  // visible tokens of the tile, one bit each
    bool see[NSUB];
    const T* kp[NSUB];
    const T* vp[NSUB];
    auto point = [&](int t, const Tokens& tk) {
      mask_next = 0;
#pragma unroll
      for (int u = 0; u < NSUB; u++) {
        see[u] = (t * KT + 16 * u + cl < limit) & ((unsigned)tk.page[u] < (unsigned)c.pages);
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
#pragma unroll
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
            *(uint4*)(Vs + v_at(r, p >> 1) + ((p & 1) << 4 ^ (r >> 3 & 1) << 4)) = v;
          else
            *(uint4*)(Vs + r * VROW + p * 16) = v;
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
                    Vs + v_at(r, d) + ((cl & 3) << 3 ^ (r >> 3 & 1) << 4)));
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

// The parts of every sequence joined: the first workgroups add the weights of
// 1024 visible tokens of a sequence each (4 tokens a lane, a fourth of the
// heads a wave, summed over the waves in order), the others write the output
// rows, `wpr` waves a row.  Bound by a chain of dependent loads, so they go out
// JOIN_AHEAD at a time, the scores before the statistics that they wait for:
// one stream alone has hundreds of parts (two of 131,072 tokens took 37 us with
// one part after the other, 23 with the statistics first).
//
// Where parts of a row are not finite its waves look through the visible values:
// the output of a dimension with infinite or NaN ones is their sum, since weights
// are positive.
constexpr int JOIN_HEADS = 128;
constexpr int JOIN_AHEAD = 4;  // (8 leave registers for one workgroup a CU: 17.5 us instead of 13.2)
// (maximum, sum) of two parts
__device__ __forceinline__ float2 join_ml(float2 a, float2 b) {
  const float m = fmaxf(a.x, b.x), mu = m == -INFINITY ? 0.f : m;
  return make_float2(m, a.y * __builtin_amdgcn_exp2f(a.x - mu) + b.y * __builtin_amdgcn_exp2f(b.x - mu));
}

template <typename T, int DP>
__global__ __launch_bounds__(1024, 8) void paged_join(CacheArgs c, PagedArgs a, PagedSpace ws,
                                                   int weights, int chunks, int wpr) {
  constexpr int KT = sizeof(T) == 2 ? 32 : 16;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  __shared__ __attribute__((aligned(16))) float part[16][256];
  __shared__ float2 s_ml[JOIN_HEADS];
  __shared__ __attribute__((aligned(16))) char s_odd[16];
  const int block = blockIdx.x + ws.block0;
  if (block >= weights) {
    const int64_t row = ((int64_t)block - weights) * (16 / wpr) + wave / wpr;
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
    if (__builtin_amdgcn_readfirstlane(odds.x | odds.y | odds.z | odds.w)) {
      __syncthreads();
      float e0 = 0.f, e1 = 0.f;
      if (real) {
        const Visible vis = visible(c, a, b);
        const int d1 = 64 + lane;
        for (int i = wave % wpr; i < vis.nv; i += wpr * 2) {
#pragma unroll
          for (int u = 0; u < 2; u++) {
            const int x = vis.slot(min(i + wpr * u, vis.nv - 1));  // (twice the last one: the same sum)
            const uint32_t pg = quot((uint32_t)x, c.page);
            const int page = page_of(c, b, pg);
            const bool see = (page >= 0) & vis.by_position(c.pos + (int64_t)b * c.cap, x, a.sinks);
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
  const int b = block / chunks, first = block % chunks * 1024;
  const Visible vis = visible(c, a, b);
  if (first >= vis.nv) return;
  const int2 plan = ws.plan[b];
  const int h0 = wave >> 2;  // the wave's heads: h0, h0 + 4, ..
  // scores of 4 tokens from x on under JOIN_AHEAD of the wave's heads from h on
  auto load_scores = [&](int x, int h, f32x4_t* s) {
    const float* sp = ws.score + (int64_t)b * ws.units * ws.tiles * ws.heads * KT +
                      (int64_t)(min(x, vis.nv - 1) / KT) * ws.heads * KT + x % KT;
#pragma unroll
    for (int u = 0; u < JOIN_AHEAD; u++) {
      const int hu = min(h + 4 * u, a.H - 1), kh = hu / a.group, r = hu - kh * a.group;
      s[u] = *(const f32x4_t*)(sp + ((int64_t)(kh * ws.qtiles + r / 16) * ws.tiles * ws.heads + r % 16) * KT);
    }
  };
  for (int hc = 0; hc < a.H; hc += JOIN_HEADS) {
    const int nh = min(JOIN_HEADS, a.H - hc);
    f32x4_t s[JOIN_AHEAD];
    load_scores(first + (wave & 3) * 256 + lane * 4, hc + h0, s);
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
        c.weight[(int64_t)b * c.cap + vis.slot(xt)] +=
            (part[t][i] + part[4 + t][i]) + (part[8 + t][i] + part[12 + t][i]);
      }
      __syncthreads();
    }
  }
}

// -------------------------------------------------------------- evict --
// Order of the tokens as unsigned integers: protected tokens above all, then
// by weight (-0 equals 0), NaN below everything, and tokens that are `lost` too.
__device__ __forceinline__ uint32_t keep_key(float w, bool safe, bool lost) {
  if (lost) return 0u;
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

// The choice, one workgroup of NT threads per sequence.  The budget-th largest
// key is found from the top by digits of 12, 10 and 10 bits: counts of the
// keys that share the digits found so far in bins, a sum over the bins from
// the highest, the bin where it reaches the rank; the search ends where the
// rank takes all of a bin.  (The first digit holds the sign, the exponent and
// three bits of the weight, so that weights of similar size meet in few bins:
// the counts are LDS atomics, and lanes that hit one address wait for each
// other.)  Threads hold E slots' keys in registers, NT apart; longer sequences
// go through them in chunks that are read again in every round.  A token past
// the budget whose slot has no page is lost: it was never stored, and moved into
// a page it would stand for the keys that lie there.  (The budget's own slots
// are as many as may stay and rank above it, so it never does.)  Then ranks in
// slot order (ballots, and one sum over the waves' counts) list the free slots
// below the budget and hand them to the kept ones beyond it.  Bound by the
// latency of loads, atomics and barriers: 64 sequences of 4,097 slots are read
// in 0.5 us and take 9.8 (15.3 with all digits searched, slots blocked over the
// threads and shuffles through LDS).
constexpr int EVICT_FEW = 32;  // moves that the choosing workgroup makes itself
template <typename T, int NT, int E>
__global__ __launch_bounds__(NT) void evict_select(CacheArgs c, EvictArgs a, EvictSpace ws) {
  constexpr int NW = NT / 64, CHUNK = NT * E;
  const int b = blockIdx.x, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int n = held(c, b);
  const int newest = (int)max((int64_t)c.seen[b] - a.recent, (int64_t)INT32_MIN);
  float* weight = c.weight + (int64_t)b * c.cap;
  int* pos = c.pos + (int64_t)b * c.cap;
  int* src = a.src + (int64_t)b * a.budget;
  if (n <= a.budget) {
    for (int x = tid; x < a.budget; x += NT) src[x] = x < n ? x : -1;
    if (tid == 0) {
      ws.moves[b] = 0;
      c.len[b] = n;
    }
    return;
  }
  uint32_t key[E];
  const int chunks = (n + CHUNK - 1) / CHUNK;
  auto load = [&](int ch) {
    float w[E];
    int p[E], page[E];
#pragma unroll
    for (int e = 0; e < E; e++) {
      const int x = min(ch * CHUNK + e * NT + tid, n - 1);
      w[e] = weight[x];
      p[e] = pos[x];
      page[e] = 0;
      if (x >= a.budget) page[e] = page_of(c, b, quot((uint32_t)x, c.page));
    }
#pragma unroll
    for (int e = 0; e < E; e++)
      key[e] = keep_key(w[e], p[e] < a.sinks || p[e] >= newest, page[e] < 0);
  };
  load(0);
  __shared__ __attribute__((aligned(16))) int bins[4096 + 1024 + 1024];
  __shared__ int s_found[3][2], s_wave[NW], s_count[E * NW + 1];
  for (int i = tid; i < 4096 + 2048; i += NT) bins[i] = 0;
  for (int x = tid; x < a.budget; x += NT) src[x] = x;
  uint32_t least = 0;    // keys above it stay
  int want = a.budget;   // and the first `want` of those equal to it
  constexpr int SHIFT[3] = {20, 10, 0};
  __syncthreads();
#pragma unroll
  for (int round = 0; round < 3; round++) {
    const int shift = SHIFT[round], nb = round ? 1024 : 4096;
    int* bin = bins + (round == 0 ? 0 : round == 1 ? 4096 : 4096 + 1024);
    for (int ch = 0; ch < chunks; ch++) {
      if (chunks > 1 && (ch || round)) load(ch);
#pragma unroll
      for (int e = 0; e < E; e++)
        if (ch * CHUNK + e * NT + tid < n && (round == 0 || key[e] >> (shift + 10) == least >> (shift + 10)))
          atomicAdd(&bin[key[e] >> shift & (nb - 1)], 1);
    }
    __syncthreads();
    // thread t sums the bins nb - per (t + 1) .. + per - 1
    const int per = nb / NT;
    int mine = 0;
    for (int i = 1; i <= per; i++) mine += bin[nb - tid * per - i];
    const int upto = wave_scan(mine);
    if (lane == 63) s_wave[wave] = upto;
    __syncthreads();
    int above = upto - mine;
    for (int w = 0; w < wave; w++) above += s_wave[w];
    if (above < want && above + mine >= want) {
      int i = nb - tid * per - 1, left = want - above;
      for (; left > bin[i]; i--) left -= bin[i];
      s_found[round][0] = i;
      s_found[round][1] = left == bin[i] ? 0 : left;
    }
    __syncthreads();
    least |= (uint32_t)s_found[round][0] << shift;
    want = s_found[round][1];
    if (want == 0) break;  // the whole bin stays
  }
  if (want == 0) least--;  // (the whole bin stays; not the lowest, since n > budget)
  // exclusive sums, in slot order, of the chunk's counts by e and wave
  auto sum_counts = [&]() {
    __syncthreads();
    if (wave == 0) {
      int before = 0;
      for (int i = 0; i < E * NW; i += 64) {
        const int v = i + lane < E * NW ? s_count[i + lane] : 0, upto = wave_scan(v);
        if (i + lane < E * NW) s_count[i + lane] = before + upto - v;
        before += __builtin_amdgcn_readlane(upto, 63);
      }
      if (lane == 0) s_count[E * NW] = before;
    }
    __syncthreads();
  };
  const uint64_t below = (1ull << lane) - 1;
  int ties = 0, holes = 0, late = 0;
  int2* mv = ws.move + (int64_t)b * ws.room;
  for (int ch = 0; ch < chunks; ch++) {
    if (chunks > 1) load(ch);
    const int x0 = ch * CHUNK + tid;
    uint32_t keep = 0;  // one bit per e
    static_assert(E <= 32 && CHUNK < 32768, "bits of a thread, two counts in a word");
    if (want > 0) {
      __syncthreads();
#pragma unroll
      for (int e = 0; e < E; e++) {
        const uint64_t eq = __ballot(x0 + e * NT < n && key[e] == least);
        if (lane == 0) s_count[e * NW + wave] = __popcll(eq);
      }
      sum_counts();
#pragma unroll
      for (int e = 0; e < E; e++) {
        const bool eq = x0 + e * NT < n && key[e] == least;
        const uint64_t m = __ballot(eq);
        const int rank = ties + s_count[e * NW + wave] + (int)__popcll(m & below);
        if (eq && rank < want) keep |= 1u << e;
      }
      ties += s_count[E * NW];
    }
#pragma unroll
    for (int e = 0; e < E; e++) keep |= (uint32_t)(key[e] > least) << e;
    __syncthreads();
    auto flags = [&](int e, uint64_t* hole, uint64_t* over) {
      const int x = x0 + e * NT;
      const bool k = keep >> e & 1;
      *hole = __ballot(x < n && x < a.budget && !k);
      *over = __ballot(x < n && x >= a.budget && k);
    };
#pragma unroll
    for (int e = 0; e < E; e++) {
      uint64_t hole, over;
      flags(e, &hole, &over);
      if (lane == 0) s_count[e * NW + wave] = (int)__popcll(hole) | (int)__popcll(over) << 16;
    }
    sum_counts();
#pragma unroll
    for (int e = 0; e < E; e++) {
      uint64_t hole, over;
      flags(e, &hole, &over);
      const int at = s_count[e * NW + wave];
      if (hole >> lane & 1) mv[holes + (at & 0xFFFF) + (int)__popcll(hole & below)].x = x0 + e * NT;
      if (over >> lane & 1) mv[late + (at >> 16) + (int)__popcll(over & below)].y = x0 + e * NT;
    }
    holes += s_count[E * NW] & 0xFFFF;
    late += s_count[E * NW] >> 16;
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
      append_many<T><<<std::min((rows + 3) / 4, APPEND_BLOCKS), 256, 0, s>>>(c, a, sq);
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
  p.ranges = split ? std::max(1, (DP == 64 ? PAGED_WAVES_64 : PAGED_WAVES) / p.units) : c.B;
  p.tiles = (c.cap + KT - 1) / KT;
  p.heads = std::min(group, 16);
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
  p.score = (float*)take(accumulate ? (size_t)c.B * p.units * p.tiles * p.heads * KT * 4 : 0);
  if (space) *space = p;
  return n;
}

template <typename T, int DP, bool PAD>
hipError_t launch_paged(const CacheArgs& c, const PagedArgs& a, const PagedSpace& ws,
                        hipStream_t s) {
  PagedSpace w = ws;
  if (hipError_t e = in_launches(((int64_t)ws.units * ws.ranges + 3) / 4, 256, [&](int first, unsigned grid) {
        w.block0 = first;
        if (a.accumulate)
          paged_attention<T, DP, PAD, true><<<grid, 256, 0, s>>>(c, a, w);
        else
          paged_attention<T, DP, PAD, false><<<grid, 256, 0, s>>>(c, a, w);
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
    paged_join<T, DP><<<grid, 1024, 0, s>>>(c, a, w, weights, chunks, wpr);
  });
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
