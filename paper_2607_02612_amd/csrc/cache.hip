// Paged token caches: appending rows, attention of one new token per sequence
// with the accumulated attention weight of every cached token, and eviction
// by that weight.
#include "kernels.h"

#include <algorithm>

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

// Offsets of a batch as kernel arguments.
constexpr int APPEND_SEQS = 896;
struct AppendSeqs {
  int n, first;  // samples of this launch, the first one's index
  int cu[APPEND_SEQS + 1];
};

// --------------------------------------------------------------- append --
// One workgroup per new row; row r of sample i goes to slot len + r - cu[i].
template <typename T>
__global__ __launch_bounds__(256) void append_kernel(CacheArgs c, AppendArgs a, AppendSeqs sq) {
  int b, r, nth;
  if (sq.n == 0) {  // one row per sample
    b = r = blockIdx.x;
    nth = 0;
  } else {
    r = sq.cu[0] + blockIdx.x;
    int lo = 0, hi = sq.n - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (sq.cu[mid] <= r) lo = mid; else hi = mid - 1;
    }
    b = sq.first + lo;
    nth = r - sq.cu[lo];
  }
  const int64_t slot = (int64_t)held(c, b) + nth;
  if (slot >= c.cap) return;
  if (threadIdx.x == 0) {
    c.weight[(int64_t)b * c.cap + slot] = 0.f;
    c.pos[(int64_t)b * c.cap + slot] = c.seen[b] + nth;
  }
  const uint32_t pg = quot((uint32_t)slot, c.page);
  const int p = page_of(c, b, pg);
  if (p < 0) return;
  const int64_t in_page = slot - (int64_t)pg * c.page.d;
  T* kd = (T*)c.k + p * c.k_page + in_page * c.k_row;
  T* vd = (T*)c.v + p * c.v_page + in_page * c.v_row;
  const T* ks = (const T*)a.k + r * a.k_row;
  const T* vs = (const T*)a.v + r * a.v_row;
  for (int t = threadIdx.x; t < c.Hkv * c.dh; t += 256) {
    const int h = t / c.dh, d = t - h * c.dh;
    kd[h * c.k_head + d] = ks[h * a.k_head + d];
    vd[h * c.v_head + d] = vs[h * a.v_head + d];
  }
}

__global__ __launch_bounds__(256) void append_lengths(CacheArgs c, AppendSeqs sq) {
  const int t = blockIdx.x * 256 + threadIdx.x;
  if (t >= (sq.n ? sq.n : c.B)) return;
  const int b = sq.n ? sq.first + t : t, n = sq.n ? sq.cu[t + 1] - sq.cu[t] : 1;
  const int have = held(c, b), fit = min(n, c.cap - have);
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
// weight that every token drew.  P is rounded to bf16 before it multiplies V
// (the matrix operand's type), nothing else is until the output.
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr int PAGED_SPLIT = 1024;  // sequences up to which the work is split over their lengths
constexpr int PAGED_WAVES = 2048;  // parts in all, about

struct PagedSpace {
  int2* plan;    // [B]: first part, number of parts
  float2* ml;    // [parts][H]: maximum (base 2), sum
  float* o;      // [parts][H][DP]
  float* score;  // [B][H][capv], base 2, by visible token
  int ranges;    // parts per unit
  int units, qtiles, capv;
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

template <typename T, int DP, bool PAD, bool SPLIT>
__global__ __launch_bounds__(256) void paged_attention(CacheArgs c, PagedArgs a, PagedSpace ws) {
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
    const Visible vis = visible(c, a, b);
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
    const int* pos = c.pos + (int64_t)b * c.cap;
    // page, place and visibility of the lane's tokens of a tile
    int page[NSUB], place[NSUB], at[NSUB];
    auto look_up = [&](int t) {
#pragma unroll
      for (int u = 0; u < NSUB; u++) {
        const int x = vis.slot(min(t * KT + 16 * u + cl, vis.nv - 1));
        const uint32_t pg = quot((uint32_t)x, c.page);
        page[u] = table[pg];
        place[u] = x - (int)(pg * c.page.d);
        at[u] = vis.by_pos ? pos[x] : 0;
      }
    };
    uint4 kr[NSUB][NL], vr[NSUB][NL];
    uint32_t mask = 0, mask_next;  // visible tokens of the tile, one bit each
    bool see[NSUB];
    auto load_kv = [&](int t) {
      mask_next = 0;
#pragma unroll
      for (int u = 0; u < NSUB; u++) {
        see[u] = t * KT + 16 * u + cl < vis.nv && (unsigned)page[u] < (unsigned)c.pages &&
                 (!vis.by_pos || at[u] >= vis.oldest || at[u] < a.sinks);
        mask_next |= (uint32_t)(__ballot(see[u]) & 0xFFFF) << (16 * u);
      }
      if (mask_next == 0) return;
#pragma unroll
      for (int u = 0; u < NSUB; u++) {
        const int64_t p = see[u] ? page[u] : 0, r = see[u] ? place[u] : 0;
        const T* k = (const T*)c.k + p * c.k_page + r * c.k_row + kh * c.k_head;
        const T* v = (const T*)c.v + p * c.v_page + r * c.v_row + kh * c.v_head;
#pragma unroll
        for (int s = 0; s < NL; s++) {
          const int d = (4 * s + g) * EPP;
          kr[u][s] = vr[u][s] = make_uint4(0, 0, 0, 0);
          if (!PAD || d < dh) {
            kr[u][s] = *(const uint4*)(k + d);
            vr[u][s] = *(const uint4*)(v + d);
          }
        }
      }
    };
    float m = -INFINITY, l = 0.f;
    f32x4_t O[ND];
#pragma unroll
    for (int d = 0; d < ND; d++) O[d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    look_up(ta);
    load_kv(ta);
    if (ta + 1 < tb) look_up(ta + 1);
    for (int t = ta; t < tb; t++) {
      mask = mask_next;
      f32x4_t S[NSUB];
#pragma unroll
      for (int u = 0; u < NSUB; u++) S[u] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      if (mask) {
#pragma unroll
        for (int u = 0; u < NSUB; u++) {
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
#pragma unroll
          for (int s = 0; s < NL; s++) {
            const uint4 v = see[u] ? vr[u][s] : make_uint4(0, 0, 0, 0);
            const int r = 16 * u + cl, p = 4 * s + g;
            if constexpr (BF)
              *(uint4*)(Vs + r * VROW + (((p >> 1) ^ (r & (DP / 16 - 1))) << 5) + ((p & 1) << 4)) = v;
            else
              *(uint4*)(Vs + r * VROW + p * 16) = v;
          }
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      if (t + 1 < tb) load_kv(t + 1);
      if (t + 2 < tb) look_up(t + 2);
      __builtin_amdgcn_sched_barrier(0);
      if (mask == 0 && !a.accumulate) continue;
#pragma unroll
      for (int u = 0; u < NSUB; u++)
#pragma unroll
        for (int j = 0; j < 4; j++)
          S[u][j] = mask >> (16 * u + 4 * g + j) & 1 ? S[u][j] * sc2 : -INFINITY;
      if (a.accumulate && cl < nq) {
        float* sp = ws.score + ((int64_t)b * a.H + h0 + cl) * ws.capv + t * KT + 4 * g;
#pragma unroll
        for (int u = 0; u < NSUB; u++) *(f32x4_t*)(sp + 16 * u) = S[u];
      }
      if (mask == 0) continue;
      float mt = fmaxf(fmaxf(S[0][0], S[0][1]), fmaxf(S[0][2], S[0][3]));
      if (NSUB > 1)
        mt = fmaxf(mt, fmaxf(fmaxf(S[NSUB - 1][0], S[NSUB - 1][1]), fmaxf(S[NSUB - 1][2], S[NSUB - 1][3])));
      mt = max_xor32(max_xor16(mt));
      const bool grow = mt > m + 8.f;
      if (__any(grow)) {
        const float f = grow ? __builtin_amdgcn_exp2f(m - mt) : 1.f;
        if (grow) m = mt;
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
        union { uint32_t u[4]; bf16x8_t v; } p;
        p.u[0] = pack_bf16x2(S[0][0], S[0][1]);
        p.u[1] = pack_bf16x2(S[0][2], S[0][3]);
        p.u[2] = pack_bf16x2(S[NSUB - 1][0], S[NSUB - 1][1]);
        p.u[3] = pack_bf16x2(S[NSUB - 1][2], S[NSUB - 1][3]);
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
        }
      } else {
#pragma unroll
        for (int j = 0; j < 4; j++)
#pragma unroll
          for (int d = 0; d < ND; d++)
            O[d] = __builtin_amdgcn_mfma_f32_16x16x4f32(
                *(const float*)(Vs + (4 * g + j) * VROW + (16 * d + cl) * 4), S[0][j], O[d], 0, 0, 0);
      }
    }
    l = sum_xor32(sum_xor16(l));
    if (cl < nq) {
      const int64_t o = (int64_t)part * a.H + h0 + cl;
      if (g == 0) ws.ml[o] = make_float2(m, l);
#pragma unroll
      for (int d = 0; d < ND; d++) *(f32x4_t*)(ws.o + o * DP + 16 * d + 4 * g) = O[d];
    }
  };

  auto tiles_of = [&](int b) {
    if (b >= c.B) return 0;
    return (visible(c, a, b).nv + KT - 1) / KT;
  };
  if constexpr (!SPLIT) {
    const int t = __builtin_amdgcn_readfirstlane(tiles_of(range));
    if (unit == 0 && lane == 0) ws.plan[range] = make_int2(range, t > 0);
    if (t > 0) segment(range, 0, t, range);
    return;
  }
  int total = 0;
  for (int b = 0; b < c.B; b += 64) total += wave_sum_i(tiles_of(b + lane));
  const int per = max(1, (total + ws.ranges - 1) / ws.ranges);
  const int first = range * per, last = min(first + per, total);
  const bool planner = unit == 0 && range == 0;
  if (first >= total && !planner) return;
  int before = 0;  // tiles of the sequences before b
  for (int b = 0; b < c.B && (before < last || planner); b += 64) {
    const int t = tiles_of(b + lane);
    int p = t;  // inclusive, then exclusive sum over the lanes
    for (int o = 1; o < 64; o <<= 1) {
      const int v = __shfl_up(p, o, 64);
      if (lane >= o) p += v;
    }
    const int sum = __shfl(p, 63, 64);
    p += before - t;
    before += sum;
    if (planner && b + lane < c.B)
      ws.plan[b + lane] = make_int2(p / per + b + lane, t > 0 ? (p + t - 1) / per - p / per + 1 : 0);
    for (uint64_t mine = __ballot(t > 0 && p < last && p + t > first); mine; mine &= mine - 1) {
      const int i = __builtin_ctzll(mine);
      const int tp = __builtin_amdgcn_readlane(p, i), tn = __builtin_amdgcn_readlane(t, i);
      segment(b + i, max(first - tp, 0), min(last - tp, tn), range + b + i);
    }
  }
}

// The parts of every sequence joined: workgroups 0 .. B H - 1 write an output
// row each, the others add the weights of 1024 visible tokens of a sequence.
constexpr int JOIN_HEADS = 128;
template <typename T>
__global__ __launch_bounds__(256) void paged_join(CacheArgs c, PagedArgs a, PagedSpace ws, int DP,
                                                  int chunks) {
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  __shared__ float part[4][128];
  __shared__ float2 s_ml[JOIN_HEADS];
  if ((int64_t)blockIdx.x < (int64_t)c.B * a.H) {
    const int b = blockIdx.x / a.H, h = blockIdx.x % a.H;
    const int2 plan = ws.plan[b];
    float m = -INFINITY;
    for (int i = lane; i < plan.y; i += 64)
      m = fmaxf(m, ws.ml[(int64_t)(plan.x + i) * a.H + h].x);
    m = wave_max(m);
    const float mu = m == -INFINITY ? 0.f : m;
    float o0 = 0.f, o1 = 0.f, l = 0.f;
    for (int i = wave; i < plan.y; i += 4) {
      const int64_t p = (int64_t)(plan.x + i) * a.H + h;
      const float2 ml = ws.ml[p];
      const float f = __builtin_amdgcn_exp2f(ml.x - mu);
      l += ml.y * f;
      if (ml.x == -INFINITY) continue;
      if (lane < DP) o0 = fmaf(ws.o[p * DP + lane], f, o0);
      if (64 + lane < DP) o1 = fmaf(ws.o[p * DP + 64 + lane], f, o1);
    }
    part[wave][lane] = o0;
    part[wave][64 + lane] = o1;
    if (lane == 0) s_ml[wave].y = l;
    __syncthreads();
    l = (s_ml[0].y + s_ml[1].y) + (s_ml[2].y + s_ml[3].y);
    if (tid < c.dh) {
      const float o = (part[0][tid] + part[1][tid]) + (part[2][tid] + part[3][tid]);
      ((T*)a.out)[((int64_t)b * a.H + h) * c.dh + tid] = St<T>::put(l == 0.f ? 0.f : o / l);
    }
    return;
  }
  const int64_t id = blockIdx.x - (int64_t)c.B * a.H;
  const int b = (int)(id / chunks), first = (int)(id % chunks) * 1024;
  const Visible vis = visible(c, a, b);
  const int2 plan = ws.plan[b];
  for (int x0 = first; x0 < vis.nv; x0 += chunks * 1024) {
    const int x = x0 + tid * 4;
    f32x4_t w = {0.f, 0.f, 0.f, 0.f};
    for (int hc = 0; hc < a.H; hc += JOIN_HEADS) {
      const int nh = min(JOIN_HEADS, a.H - hc);
      __syncthreads();
      // maximum and 1 / (sum H) of the heads, 16 lanes a head
      for (int h = tid >> 4; h < nh; h += 16) {
        float m = -INFINITY, l = 0.f;
        for (int i = tid & 15; i < plan.y; i += 16) {
          const float2 ml = ws.ml[(int64_t)(plan.x + i) * a.H + hc + h];
          const float m2 = fmaxf(m, ml.x);
          if (m2 != -INFINITY)
            l = l * __builtin_amdgcn_exp2f(m - m2) + ml.y * __builtin_amdgcn_exp2f(ml.x - m2);
          m = m2;
        }
        for (int o = 8; o; o >>= 1) {
          const float mo = __shfl_xor(m, o, 16), lo = __shfl_xor(l, o, 16), m2 = fmaxf(m, mo);
          if (m2 != -INFINITY)
            l = l * __builtin_amdgcn_exp2f(m - m2) + lo * __builtin_amdgcn_exp2f(mo - m2);
          m = m2;
        }
        if ((tid & 15) == 0)
          s_ml[h] = make_float2(m == -INFINITY ? 0.f : m, l == 0.f ? 0.f : 1.f / (l * (float)a.H));
      }
      __syncthreads();
      if (x < vis.nv) {
        const float* sp = ws.score + ((int64_t)b * a.H + hc) * ws.capv + x;
        for (int h = 0; h < nh; h++) {
          const f32x4_t s = *(const f32x4_t*)(sp + (int64_t)h * ws.capv);
          const float2 ml = s_ml[h];
#pragma unroll
          for (int j = 0; j < 4; j++) w[j] = fmaf(__builtin_amdgcn_exp2f(s[j] - ml.x), ml.y, w[j]);
        }
      }
    }
#pragma unroll
    for (int j = 0; j < 4; j++)
      if (x + j < vis.nv) c.weight[(int64_t)b * c.cap + vis.slot(x + j)] += w[j];
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

// One workgroup of 1024 per sequence: the budget-th largest key by four
// rounds of 256 bins, then one pass in slot order that lists free slots below
// the budget and hands them to the kept ones beyond it.
__global__ __launch_bounds__(1024) void evict_select(CacheArgs c, EvictArgs a, EvictSpace ws) {
  const int b = blockIdx.x, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int n = held(c, b), seen = c.seen[b];
  float* weight = c.weight + (int64_t)b * c.cap;
  int* pos = c.pos + (int64_t)b * c.cap;
  int* src = a.src + (int64_t)b * a.budget;
  for (int x = tid; x < a.budget; x += 1024) src[x] = x < n ? x : -1;
  if (n <= a.budget) {
    if (tid == 0) {
      ws.moves[b] = 0;
      c.len[b] = n;
    }
    return;
  }
  auto key_of = [&](int x) {
    const int p = pos[x];
    return keep_key(weight[x], p < a.sinks || seen - p <= a.recent);
  };
  __shared__ int bins[256];
  __shared__ int s_digit, s_want, s_w[16];
  uint32_t prefix = 0;
  int want = a.budget;  // rank of the key searched, among those with the prefix
  for (int shift = 24; shift >= 0; shift -= 8) {
    if (tid < 256) bins[tid] = 0;
    __syncthreads();
    for (int x = tid; x < n; x += 1024) {
      const uint32_t k = key_of(x);
      if (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8)))
        atomicAdd(&bins[(k >> shift) & 255], 1);
    }
    __syncthreads();
    if (tid == 0) {
      int left = want, d = 255;
      for (; d > 0 && left > bins[d]; d--) left -= bins[d];
      s_digit = d;
      s_want = left;
    }
    __syncthreads();
    prefix |= (uint32_t)s_digit << shift;
    want = s_want;
    __syncthreads();
  }
  // keys above `prefix` stay, and the first `want` equal to it
  auto scan = [&](bool v, int& total) {  // count of set flags before this thread's
    const uint64_t m = __ballot(v);
    __syncthreads();
    if (lane == 0) s_w[wave] = __popcll(m);
    __syncthreads();
    int before = 0;
    total = 0;
    for (int w = 0; w < 16; w++) {
      if (w < wave) before += s_w[w];
      total += s_w[w];
    }
    return before + (int)__popcll(m & ((1ull << lane) - 1));
  };
  int ties = 0, holes = 0, late = 0;
  int2* mv = ws.move + (int64_t)b * ws.room;
  for (int x0 = 0; x0 < n; x0 += 1024) {
    const int x = x0 + tid;
    const uint32_t k = x < n ? key_of(x) : 0u;
    const bool tie = x < n && k == prefix;
    int total;
    const int rank = ties + scan(tie, total);
    ties += total;
    const bool keep = x < n && (k > prefix || (tie && rank < want));
    const bool hole = x < n && x < a.budget && !keep, over = keep && x >= a.budget;
    const int hi = holes + scan(hole, total);
    holes += total;
    if (hole) mv[hi].x = x;
    const int li = late + scan(over, total);
    late += total;
    if (over) mv[li].y = x;
  }
  __syncthreads();
  for (int i = tid; i < holes; i += 1024) {
    const int2 m = mv[i];
    weight[m.x] = weight[m.y];
    pos[m.x] = pos[m.y];
    src[m.x] = m.y;
  }
  if (tid == 0) {
    ws.moves[b] = holes;
    c.len[b] = a.budget;
  }
}

template <typename T>
__global__ __launch_bounds__(256) void evict_move(CacheArgs c, EvictSpace ws) {
  const int b = blockIdx.x, n = ws.moves[b];
  for (int i = blockIdx.y; i < n; i += gridDim.y) {
    const int2 m = ws.move[(int64_t)b * ws.room + i];
    const uint32_t pd = quot(m.x, c.page), ps = quot(m.y, c.page);
    const int pgd = page_of(c, b, pd), pgs = page_of(c, b, ps);
    if (pgd < 0 || pgs < 0) continue;
    const int64_t rd = m.x - (int64_t)pd * c.page.d, rs = m.y - (int64_t)ps * c.page.d;
    T* k = (T*)c.k;
    T* v = (T*)c.v;
    for (int t = threadIdx.x; t < c.Hkv * c.dh; t += 256) {
      const int h = t / c.dh, d = t - h * c.dh;
      k[pgd * c.k_page + rd * c.k_row + h * c.k_head + d] =
          k[pgs * c.k_page + rs * c.k_row + h * c.k_head + d];
      v[pgd * c.v_page + rd * c.v_row + h * c.v_head + d] =
          v[pgs * c.v_page + rs * c.v_row + h * c.v_head + d];
    }
  }
}

}  // namespace

template <typename T>
hipError_t launch_cache_append(const CacheArgs& c, const AppendArgs& a, const int32_t* cu_host,
                               hipStream_t s) {
  AppendSeqs sq;
  if (!cu_host) {
    sq.n = 0;
    append_kernel<T><<<c.B, 256, 0, s>>>(c, a, sq);
    append_lengths<<<(c.B + 255) / 256, 256, 0, s>>>(c, sq);
    return hipGetLastError();
  }
  for (int f = 0; f < c.B; f += APPEND_SEQS) {
    sq.first = f;
    sq.n = std::min(c.B - f, APPEND_SEQS);
    std::copy(cu_host + f, cu_host + f + sq.n + 1, sq.cu);
    const int rows = sq.cu[sq.n] - sq.cu[0];
    if (rows == 0) continue;
    append_kernel<T><<<rows, 256, 0, s>>>(c, a, sq);
    append_lengths<<<(sq.n + 255) / 256, 256, 0, s>>>(c, sq);
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
size_t paged_space(const CacheArgs& c, int H, int accumulate, char* ws, PagedSpace* space) {
  PagedSpace p;
  const int group = H / c.Hkv, DP = c.dh <= 64 ? 64 : 128;
  p.qtiles = (group + 15) / 16;
  p.units = c.Hkv * p.qtiles;
  const bool split = c.B <= PAGED_SPLIT;
  p.ranges = split ? std::max(1, PAGED_WAVES / p.units) : c.B;
  p.capv = (c.cap + 31) / 32 * 32;
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
  p.score = (float*)take(accumulate ? (size_t)c.B * H * p.capv * 4 : 0);
  if (space) *space = p;
  return n;
}

template <typename T, int DP, bool PAD>
hipError_t launch_paged(const CacheArgs& c, const PagedArgs& a, const PagedSpace& ws,
                        hipStream_t s) {
  const unsigned grid = (unsigned)(((int64_t)ws.units * ws.ranges + 3) / 4);
  if (c.B <= PAGED_SPLIT)
    paged_attention<T, DP, PAD, true><<<grid, 256, 0, s>>>(c, a, ws);
  else
    paged_attention<T, DP, PAD, false><<<grid, 256, 0, s>>>(c, a, ws);
  if (hipError_t e = hipGetLastError()) return e;
  // (workgroups past a sequence's tokens leave at once)
  const int chunks = a.accumulate ? std::max(1, std::min((c.cap + 1023) / 1024, 16384 / c.B)) : 0;
  const unsigned join = (unsigned)((int64_t)c.B * a.H + (int64_t)c.B * chunks);
  paged_join<T><<<join, 256, 0, s>>>(c, a, ws, DP, chunks);
  return hipGetLastError();
}
}  // namespace

size_t paged_workspace_bytes(const CacheArgs& c, int H, int accumulate) {
  return paged_space(c, H, accumulate, nullptr, nullptr);
}

template <typename T>
hipError_t launch_paged_attention(const CacheArgs& c, const PagedArgs& a, hipStream_t s) {
  PagedSpace ws;
  paged_space(c, a.H, a.accumulate, (char*)a.ws, &ws);
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
  evict_select<<<c.B, 1024, 0, s>>>(c, a, ws);
  if (ws.room > 0) {
    const int x = std::min(ws.room, std::max(1, 4096 / c.B));
    evict_move<T><<<dim3(c.B, x), 256, 0, s>>>(c, ws);
  }
  return hipGetLastError();
}
template hipError_t launch_cache_evict<float>(const CacheArgs&, const EvictArgs&, hipStream_t);
template hipError_t launch_cache_evict<bf16_t>(const CacheArgs&, const EvictArgs&, hipStream_t);

}  // namespace fusion
