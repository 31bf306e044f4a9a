// Paged token caches: appending rows, attention of one new token per sequence
// with the accumulated attention weight of every cached token, and eviction
// by that weight.
#include "paged.h"

#include <algorithm>
#include <type_traits>

namespace fusion {
namespace {

// 16-byte pieces of the rows of a token's key heads (or value heads); in 4 bits
// (T uint8_t) a piece is a block of 32 values with one scale.
struct RowPieces {
  int per_head, all;
};
template <typename T>
__device__ __forceinline__ RowPieces row_pieces(const CacheArgs& c) {
  const int p = sizeof(T) == 1 ? c.dh / 32 : c.dh * (int)sizeof(T) / 16;
  return {p, p * c.Hkv};
}
// Address of a piece of a cached row.
template <typename T>
__device__ __forceinline__ uint4* piece(void* base, int64_t page_stride, int64_t row_stride,
                                        int64_t head_stride, int page, int place, int h, int d) {
  return (uint4*)((T*)base + page * page_stride + place * row_stride + h * head_stride) + d;
}

// --------------------------------------------------------------- append --
// Row r of sample i goes to slot len + r - cu[i]: a copy, bound by its bytes.
// A wave copies whole rows in 16-byte pieces.  With few rows a sample, one
// workgroup takes a sample's rows and moves its lengths on; else the lengths
// move in a launch of their own, after all rows have read them.

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
    if constexpr (sizeof(T) == 1) {
      c.ks[to * c.ks_page + rd * c.ks_row + h * c.ks_head + d] =
          c.ks[from * c.ks_page + rs * c.ks_row + h * c.ks_head + d];
      c.vs[to * c.vs_page + rd * c.vs_row + h * c.vs_head + d] =
          c.vs[from * c.vs_page + rs * c.vs_row + h * c.vs_head + d];
    }
  }
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

template <typename T>
size_t paged_workspace_bytes(const CacheArgs& c, int H, int accumulate) {
  return paged_space<T, false>(c, H, accumulate, nullptr, nullptr, tile_tokens<T, false>());
}

template <typename T>
hipError_t launch_paged_attention(const CacheArgs& c, const PagedArgs& a, hipStream_t s) {
  PagedSpace ws;
  paged_space<T, false>(c, a.H, a.accumulate, (char*)a.ws, &ws, tile_tokens<T, false>());
  return launch_paged_by_width<T, false, false>(c, a, ws, s);
}
template size_t paged_workspace_bytes<float>(const CacheArgs&, int, int);
template size_t paged_workspace_bytes<bf16_t>(const CacheArgs&, int, int);
template hipError_t launch_paged_attention<float>(const CacheArgs&, const PagedArgs&, hipStream_t);
template hipError_t launch_paged_attention<bf16_t>(const CacheArgs&, const PagedArgs&, hipStream_t);

static int evict_room(const CacheArgs& c, int budget) {
  return std::max(0, std::min(budget, c.cap - budget));
}
size_t evict_workspace_bytes(const CacheArgs& c, int budget) {
  return round256((size_t)c.B * 4) + (size_t)c.B * evict_room(c, budget) * 8;
}

namespace {
template <typename T>
hipError_t launch_evict(const CacheArgs& c, const EvictArgs& a, hipStream_t s) {
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
}  // namespace

template <typename T>
hipError_t launch_cache_evict(const CacheArgs& c, const EvictArgs& a, hipStream_t s) {
  return c.ks ? launch_evict<uint8_t>(c, a, s) : launch_evict<T>(c, a, s);
}
template hipError_t launch_cache_evict<float>(const CacheArgs&, const EvictArgs&, hipStream_t);
template hipError_t launch_cache_evict<bf16_t>(const CacheArgs&, const EvictArgs&, hipStream_t);

}  // namespace fusion
