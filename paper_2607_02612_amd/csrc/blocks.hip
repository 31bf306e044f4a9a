// Attention over the pages of a token cache that a cheap score chooses for each
// key head.
//
// With lo_d and hi_d the least and the greatest value of dim d over a page's
// keys, no product q.k with a key of the page passes
//   sum_d max(q_d lo_d, q_d hi_d) = sum_d q_d (q_d >= 0 ? hi_d : lo_d),
// and the largest of these bounds over the query heads of a key head is the
// page's score.  The `blocks` pages with the highest scores are attended, the
// sequence's `first` and `recent` ones among them whatever their scores; of equal
// scores the lower page's counts as the higher.  Scores are summed in 64 bits
// and rounded to 32, so that the choice does not go by the order of a sum
// (products of bf16 numbers are exact, and so are nearly all their sums).
#include "paged.h"

namespace fusion {
namespace {

constexpr unsigned STRIDE_BLOCKS = 1 << 22;  // workgroups of a launch, which stride over the rest

// Eight values of a cached row: dims d .. d + 7 of the row's head (T: the type of
// the bounds).
template <typename T, bool FOUR>
__device__ __forceinline__ void held8(const CacheArgs& c, int page, int place, int h, int d, float* x) {
  if constexpr (FOUR) {
    const uint32_t codes = *(const uint32_t*)((const uint8_t*)c.k + page * c.k_page + place * c.k_row +
                                              h * c.k_head + d / 2);
    const uint32_t s = c.ks[page * c.ks_page + place * c.ks_row + h * c.ks_head + d / 32];
    const uint4 v = four_word(codes, __uint_as_float(s << 23));
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; i++) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  } else {
    load8((const T*)c.k + page * c.k_page + place * c.k_row + h * c.k_head + d, x);
  }
}

// ------------------------------------------------------------------ bounds --
// A workgroup takes 16 pieces of eight dims of a page (of the pages that hold a
// sequence's newest slots), 16 lanes side by side and 16 tokens at a time; the
// parts meet over the lanes and then in LDS.  Least and greatest are exact in
// any order; NaN has no part in them.  Bound by latency: the newest page of 64
// sequences (64 bf16 tokens, 8 heads of 128) takes 5.1 us, so a page's pieces are spread
// over workgroups.
template <typename T, bool FOUR>
__global__ __launch_bounds__(256) void page_bounds(CacheArgs c, BoundsArgs a, FastDiv pieces, int touched,
                                                   int chunks) {
  __shared__ float s_lo[3][16][9], s_hi[3][16][9];
  const int tid = threadIdx.x, ps = (int)c.page.d, all = c.Hkv * (int)pieces.d;
  const int wave = tid >> 6, mine = tid & 15, set = tid >> 4;
  // (no division of 64 bits: it takes longer than the work of a page)
  auto bounds = [&](int b, int t, int chunk) {
    const int n = held(c, b);
    const int from = a.newest ? (int)quot((uint32_t)max(0, n - a.newest), c.page) : 0;
    const int64_t pg = (int64_t)from + t;
    if (pg * ps >= n) return;
    const int page = page_of(c, b, (uint32_t)pg), rows = (int)min((int64_t)ps, n - pg * ps);
    if (page < 0) return;
    const int p = chunk * 16 + mine, h = (int)quot((uint32_t)p, pieces);
    const int d = (p - h * (int)pieces.d) * 8;
    float lo[8], hi[8];
#pragma unroll
    for (int i = 0; i < 8; i++) {
      lo[i] = INFINITY;
      hi[i] = -INFINITY;
    }
    if (p < all) {
      for (int r = set; r < rows; r += 64) {
        float x[4][8];
#pragma unroll
        for (int u = 0; u < 4; u++) held8<T, FOUR>(c, page, min(r + 16 * u, rows - 1), h, d, x[u]);
#pragma unroll
        for (int u = 0; u < 4; u++)
#pragma unroll
          for (int i = 0; i < 8; i++) {
            lo[i] = fminf(lo[i], x[u][i]);
            hi[i] = fmaxf(hi[i], x[u][i]);
          }
      }
    }
#pragma unroll
    for (int i = 0; i < 8; i++) {
      lo[i] = -max_xor32(max_xor16(-lo[i]));
      hi[i] = max_xor32(max_xor16(hi[i]));
    }
    if (wave > 0 && (tid & 63) < 16) {
#pragma unroll
      for (int i = 0; i < 8; i++) {
        s_lo[wave - 1][mine][i] = lo[i];
        s_hi[wave - 1][mine][i] = hi[i];
      }
    }
    __syncthreads();
    if (tid < 16 && p < all) {
#pragma unroll
      for (int w = 0; w < 3; w++)
#pragma unroll
        for (int i = 0; i < 8; i++) {
          lo[i] = fminf(lo[i], s_lo[w][mine][i]);
          hi[i] = fmaxf(hi[i], s_hi[w][mine][i]);
        }
      const int64_t at = ((int64_t)page * c.Hkv + h) * c.dh + d;
      store8((T*)a.lo + at, lo);
      store8((T*)a.hi + at, hi);
    }
    __syncthreads();
  };
  for (int b = blockIdx.z; b < c.B; b += gridDim.z)
    for (int t = blockIdx.y; t < touched; t += gridDim.y)
      for (int chunk = blockIdx.x; chunk < chunks; chunk += gridDim.x) bounds(b, t, chunk);
}

// ------------------------------------------------------------------ scores --
// Order of the pages as unsigned integers: those always chosen above all, then
// pages whose score is NaN (an infinite key beside a zero: no bound), then by
// score, and pages that are not there below everything.
constexpr uint32_t KEY_ALWAYS = 0xFFFFFFFFu, KEY_NAN = 0xFFFFFFFEu;
__device__ __forceinline__ uint32_t score_key(float score) {
  if (score != score) return KEY_NAN;
  const uint32_t u = __float_as_uint(score + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Value of lane ^ O within 16 lanes.
template <int O>
__device__ __forceinline__ double lane_xor(double v) {
  const uint64_t u = __double_as_longlong(v);
  const uint32_t lo = (uint32_t)lane_xor_i<O>((int)(uint32_t)u), hi = (uint32_t)lane_xor_i<O>((int)(u >> 32));
  return __longlong_as_double((uint64_t)hi << 32 | lo);
}

// Bounds of a page for the 16 lanes that take it, eight dims each (past the head:
// the last eight again).
struct PageDims {
  float lo[8], hi[8];
  bool there;
};
template <typename T>
__device__ __forceinline__ PageDims page_dims(const CacheArgs& c, const BlockArgs& a, int b, int kh, int p,
                                              int lane) {
  const int d = (lane & 15) * 8, page = page_of(c, b, p);
  const int64_t at = ((int64_t)max(page, 0) * c.Hkv + kh) * c.dh + min(d, c.dh - 8);
  PageDims x;
  x.there = page >= 0;
  load8((const T*)a.lo + at, x.lo);
  load8((const T*)a.hi + at, x.hi);
  return x;
}

// Largest key of the page's scores.  Four heads at a time, each of which ends in
// the lanes whose number's last two bits are its own.  The loads go out together,
// before any is used (a head without one more: the last head again).
template <typename T> struct Dims8 {
  uint4 u[sizeof(T) / 2];
};
template <typename T>
__device__ __forceinline__ void load_heads(const CacheArgs& c, const BlockArgs& a, int b, int kh, int h0,
                                           int lane, Dims8<T>* q) {
  const int d = min((lane & 15) * 8, c.dh - 8);
  const T* qp = (const T*)a.p.q + (int64_t)b * a.p.q_row + (int64_t)kh * a.p.group * a.p.q_head + d;
#pragma unroll
  for (int h = 0; h < 4; h++) {
    const uint4* from = (const uint4*)(qp + min(h0 + h, a.p.group - 1) * a.p.q_head);
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; i++) q[h].u[i] = from[i];
  }
}
template <typename T>
__device__ __forceinline__ uint32_t page_key(const CacheArgs& c, const BlockArgs& a, int b, int kh,
                                             const PageDims& x, int lane, Dims8<T>* q) {
  uint32_t key = 0;
  for (int h0 = 0; h0 < a.p.group; h0 += 4) {
    if (h0) load_heads<T>(c, a, b, kh, h0, lane, q);
    double s[4];
#pragma unroll
    for (int h = 0; h < 4; h++) {
      float f[8];
      load8((const T*)&q[h], f);
      s[h] = 0.0;
      if (h0 + h >= a.p.group) continue;
#pragma unroll
      for (int j = 0; j < 8; j++) s[h] = fma((double)f[j], (double)(f[j] >= 0.f ? x.hi[j] : x.lo[j]), s[h]);
      s[h] = (lane & 15) * 8 < c.dh ? s[h] : 0.0;  // (a lane past the head has the last one's dims again)
    }
    const bool one = lane & 1, two = lane & 2;
    // heads 0, 1 to the even lanes, 2, 3 to the odd ones; then the first or the second of them
    const double u = (one ? s[2] : s[0]) + lane_xor<1>(one ? s[0] : s[2]);
    const double v = (one ? s[3] : s[1]) + lane_xor<1>(one ? s[1] : s[3]);
    double w = (two ? v : u) + lane_xor<2>(two ? u : v);
    w += lane_xor<4>(w);
    w += lane_xor<8>(w);
    if (h0 + (one ? 2 : 0) + (two ? 1 : 0) < a.p.group) key = max(key, score_key((float)w));
  }
  key = max(key, (uint32_t)lane_xor_i<1>((int)key));
  key = max(key, (uint32_t)lane_xor_i<2>((int)key));
  return x.there ? key : 0u;
}
// The key of a page that may always be chosen.
__device__ __forceinline__ uint32_t final_key(uint32_t key, int p, int pages, const BlockArgs& a) {
  return p < a.first || p >= pages - a.recent ? KEY_ALWAYS : key;
}

__device__ __forceinline__ int page_count(const CacheArgs& c, int n) {
  return (int)quot((uint32_t)n + c.page.d - 1, c.page);
}
// Sequences of no more pages than are chosen.
__device__ __forceinline__ void choose_all(const CacheArgs& c, int b, int pages, int blocks, int* chosen,
                                           int* at, int tid, int step) {
  for (int i = tid; i < blocks; i += step) {
    chosen[i] = i < pages ? i : -1;
    at[i] = i < pages ? page_of(c, b, i) : -1;
  }
}

// The keys, by workgroups of SCORE_PAGES pages.  A chain of loads (length, page,
// bounds) hidden by many small workgroups: 4,096 of them, half past the ends of their
// sequences, take 12.5 us for 17 MB of bounds (64 sequences of up to 128 pages, 32
// heads over 8), 9.6 for two sequences of 2,048; 10.2 and 8.5 with sums in 32 bits.  The
// key heads run fastest over the workgroups, since they are neighbours in memory
// (slowest: 14.7), then the sequences: with their chunks fastest (13.4) the XCDs whose
// chunks lie past most ends would have no work.
constexpr int SCORE_PAGES = 16;
template <typename T>
__global__ __launch_bounds__(256) void block_scores(CacheArgs c, BlockArgs a, uint32_t* keys, FastDiv batch,
                                                    uint32_t units) {
  const int lane = threadIdx.x & 63, kh = blockIdx.x;
  for (uint32_t unit = blockIdx.y; unit < units; unit += gridDim.y) {
    const uint32_t chunk = quot(unit, batch);
    const int b = (int)(unit - chunk * batch.d);
    const int pages = page_count(c, held(c, b));
    const int p = (int)chunk * SCORE_PAGES + (threadIdx.x >> 4);
    if (pages <= a.p.blocks || p - (lane >> 4) >= pages) continue;
    const int64_t bk = (int64_t)b * c.Hkv + kh;
    Dims8<T> q[4];
    load_heads<T>(c, a, b, kh, 0, lane, q);
    const PageDims x = page_dims<T>(c, a, b, kh, min(p, c.max_pages - 1), lane);
    const uint32_t key = page_key<T>(c, a, b, kh, x, lane, q);
    if ((lane & 15) == 0 && p < pages) keys[bk * c.max_pages + p] = final_key(key, p, pages, a);
  }
}

// The choice among few pages, a wave per sequence and key head: the blocks-th
// largest key is found bit by bit, with counts of ballots and no barrier (512
// choices among up to 128 pages: 5.3 us, by block_choose 10.9; 48 among up to 417
// with 8 keys a lane: 10.3, by block_choose 6.4).
constexpr int FEW_E = 4, FEW_PAGES = 64 * FEW_E;
__global__ __launch_bounds__(256) void block_choose_few(CacheArgs c, BlockArgs a, const uint32_t* keys,
                                                        int* sel) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, blocks = a.p.blocks, kh = blockIdx.y;
  for (int b = blockIdx.x * 4 + wave; b < c.B; b += gridDim.x * 4) {
    const int64_t bk = (int64_t)b * c.Hkv + kh;
    const int pages = __builtin_amdgcn_readfirstlane(page_count(c, held(c, b)));
    int* chosen = a.chosen + bk * blocks;
    int* at = sel + bk * blocks;
    if (pages <= blocks) {
      choose_all(c, b, pages, blocks, chosen, at, lane, 64);
      continue;
    }
    uint32_t key[FEW_E];
    int page[FEW_E];
#pragma unroll
    for (int e = 0; e < FEW_E; e++) {
      const int p = 64 * e + lane;
      key[e] = p < pages ? keys[bk * c.max_pages + p] : 0u;
      page[e] = p < pages ? page_of(c, b, p) : -1;
    }
    auto count = [&](uint32_t from) {  // keys from `from` on, from > 0 (so none past the last page)
      int n = 0;
#pragma unroll
      for (int e = 0; e < FEW_E; e++)
        if (64 * e < pages) n += (int)__popcll(__ballot(key[e] >= from));
      return n;
    };
    uint32_t least = 0;
    int n = pages;
    for (int bit = 31; bit >= 0 && n != blocks; bit--) {
      const uint32_t to = least | 1u << bit;
      const int m = count(to);
      if (m >= blocks) {
        least = to;
        n = m;
      }
    }
    // keys above `least`, and of those equal to it the first
    const int want = n == blocks ? n : blocks - count(least + 1);  // (n > blocks: not all keys are the largest)
    const uint64_t below = (1ull << lane) - 1;
    int done = 0, ties = 0;
#pragma unroll
    for (int e = 0; e < FEW_E; e++) {
      const int p = 64 * e + lane;
      const uint64_t same = __ballot(p < pages && key[e] == least);
      const bool take = p < pages && (key[e] > least ||
                                      (key[e] == least && ties + (int)__popcll(same & below) < want));
      const uint64_t taken = __ballot(take);
      if (take) {
        const int i = done + (int)__popcll(taken & below);
        chosen[i] = p;
        at[i] = page[e];
      }
      done += (int)__popcll(taken);
      ties += (int)__popcll(same);
    }
  }
}

// One workgroup per sequence and key head: the blocks-th largest key from the
// top by digits of 12, 10 and 10 bits (counts in LDS), then the chosen pages in
// order; bound by its barriers, 9.6 us for 16 choices among up to 2,048 pages.  The
// threads hold CHOOSE_PAGES keys, 1024 apart; more are read again in every round.
constexpr int CHOOSE_E = 4, CHOOSE_PAGES = 1024 * CHOOSE_E;
__global__ __launch_bounds__(1024) void block_choose(CacheArgs c, BlockArgs a, const uint32_t* keys, int* sel) {
  __shared__ int bins[4096 + 2048], s_found[2], s_wave[16], s_count[16][2];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int blocks = a.p.blocks;
  for (int b = blockIdx.x; b < c.B; b += gridDim.x) {
    const int kh = blockIdx.y;
    const int64_t bk = (int64_t)b * c.Hkv + kh;
    const int pages = page_count(c, held(c, b));
    int* chosen = a.chosen + bk * blocks;
    int* at = sel + bk * blocks;
    if (pages <= blocks) {
      choose_all(c, b, pages, blocks, chosen, at, tid, 1024);
      continue;
    }
    const uint32_t* kp = keys + bk * c.max_pages;
    uint32_t key[CHOOSE_E];
    int page[CHOOSE_E];
    const int chunks = (pages + CHOOSE_PAGES - 1) / CHOOSE_PAGES;
    auto load = [&](int ch) {
#pragma unroll
      for (int e = 0; e < CHOOSE_E; e++) {
        const int p = min(ch * CHOOSE_PAGES + e * 1024 + tid, pages - 1);
        key[e] = kp[p];
        page[e] = page_of(c, b, p);
      }
    };
    load(0);
    __syncthreads();
    for (int i = tid; i < 4096 + 2048; i += 1024) bins[i] = 0;
    __syncthreads();
    uint32_t least = 0;  // keys above it are chosen
    int want = blocks;   // and the first `want` of those equal to it
    for (int round = 0; round < 3; round++) {
      const int shift = round == 0 ? 20 : round == 1 ? 10 : 0, nb = round ? 1024 : 4096;
      int* bin = bins + (round == 0 ? 0 : 4096 + 1024 * (round - 1));
      for (int ch = 0; ch < chunks; ch++) {
        if (chunks > 1 && (ch || round)) load(ch);
#pragma unroll
        for (int e = 0; e < CHOOSE_E; e++)
          if (ch * CHOOSE_PAGES + e * 1024 + tid < pages &&
              (round == 0 || key[e] >> (shift + 10) == least >> (shift + 10)))
            atomicAdd(&bin[key[e] >> shift & (nb - 1)], 1);
      }
      __syncthreads();
      // thread t sums the bins nb - per (t + 1) .. + per - 1
      const int per = nb / 1024;
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
        s_found[0] = i;
        s_found[1] = left == bin[i] ? 0 : left;
      }
      __syncthreads();
      least |= (uint32_t)s_found[0] << shift;
      want = s_found[1];
      if (want == 0) break;  // the whole bin is chosen
    }
    if (want == 0) least--;  // (not the lowest bin, since there are more pages than blocks)
    int done = 0, ties = 0;
    const uint64_t below = (1ull << lane) - 1;
    for (int ch = 0; ch < chunks; ch++) {
      if (chunks > 1) load(ch);
#pragma unroll
      for (int e = 0; e < CHOOSE_E; e++) {
        const int p = ch * CHOOSE_PAGES + e * 1024 + tid;
        if (ch * CHOOSE_PAGES + e * 1024 >= pages) break;
        const uint64_t more = __ballot(p < pages && key[e] > least);
        const uint64_t same = __ballot(p < pages && key[e] == least);
        __syncthreads();
        if (lane == 0) {
          s_count[wave][0] = (int)__popcll(more);
          s_count[wave][1] = (int)__popcll(same);
        }
        __syncthreads();
        int m = done, t = ties;
        for (int w = 0; w < 16; w++) {
          const int cm = s_count[w][0], ct = s_count[w][1];
          m += w < wave ? cm : 0;
          t += w < wave ? ct : 0;
          done += cm;
          ties += ct;
        }
        m += (int)__popcll(more & below);
        t += (int)__popcll(same & below);
        // (of the equal ones before p the first `want` were taken)
        if (more >> lane & 1 || ((same >> lane & 1) && t < want)) {
          const int i = m + min(t, want);
          chosen[i] = p;
          at[i] = page[e];
        }
      }
    }
    __syncthreads();
  }
}

template <typename T, bool FOUR>
size_t block_space(const CacheArgs& c, int H, int blocks, char* ws, PagedSpace* space, uint32_t** keys,
                   int KT) {
  size_t n = paged_space<T, FOUR>(c, H, 0, ws, space, KT);
  if (space) {
    *keys = (uint32_t*)(ws + n);
    space->sel = (const int*)(ws + n + round256((size_t)c.B * c.Hkv * c.max_pages * 4));
  }
  return n + round256((size_t)c.B * c.Hkv * c.max_pages * 4) + round256((size_t)c.B * c.Hkv * blocks * 4);
}

template <typename T, bool FOUR>
hipError_t launch_blocks(const CacheArgs& c, const BlockArgs& a, hipStream_t s) {
  PagedSpace ws;
  uint32_t* keys;
  block_space<T, FOUR>(c, a.p.H, a.p.blocks, (char*)a.p.ws, &ws, &keys, paged_tile<T, FOUR>(a.p));
  if (c.max_pages > a.p.blocks) {
    // (a batch has at most 2^34 slots, so units fit 2^31)
    const uint32_t units = (uint32_t)c.B * (uint32_t)((c.max_pages + SCORE_PAGES - 1) / SCORE_PAGES);
    block_scores<T><<<dim3(c.Hkv, std::min(units, std::min(65535u, STRIDE_BLOCKS / c.Hkv))), 256, 0, s>>>(
        c, a, keys, fast_div(c.B), units);
    if (hipError_t e = hipGetLastError()) return e;
  }
  const unsigned most = std::max(1u, (STRIDE_BLOCKS >> 2) / c.Hkv);
  if (c.max_pages <= FEW_PAGES)
    block_choose_few<<<dim3(std::min((c.B + 3) / 4u, most), c.Hkv), 256, 0, s>>>(c, a, keys, (int*)ws.sel);
  else
    block_choose<<<dim3(std::min<unsigned>(c.B, most), c.Hkv), 1024, 0, s>>>(c, a, keys, (int*)ws.sel);
  if (hipError_t e = hipGetLastError()) return e;
  return launch_paged_by_width<T, FOUR, true>(c, a.p, ws, s);
}
}  // namespace

template <typename T>
hipError_t launch_page_bounds(const CacheArgs& c, const BoundsArgs& a, hipStream_t s) {
  const FastDiv pieces = fast_div((uint32_t)c.dh / 8);
  const int ps = (int)c.page.d, chunks = (c.Hkv * (int)pieces.d + 15) / 16;
  int64_t touched = c.max_pages;
  if (a.newest) touched = std::min<int64_t>(touched, ((int64_t)a.newest - 2 + ps) / ps + 1);
  const unsigned x = std::min(chunks, 256), z = std::min(c.B, 1024);
  const dim3 grid(x, (unsigned)std::min<int64_t>(touched, std::min(65535u, STRIDE_BLOCKS / (x * z))), z);
  if (c.ks)
    page_bounds<T, true><<<grid, 256, 0, s>>>(c, a, pieces, (int)touched, chunks);
  else
    page_bounds<T, false><<<grid, 256, 0, s>>>(c, a, pieces, (int)touched, chunks);
  return hipGetLastError();
}
template hipError_t launch_page_bounds<float>(const CacheArgs&, const BoundsArgs&, hipStream_t);
template hipError_t launch_page_bounds<bf16_t>(const CacheArgs&, const BoundsArgs&, hipStream_t);

template <typename T>
size_t block_workspace_bytes(const CacheArgs& c, int H, int blocks) {
  return c.ks ? block_space<T, true>(c, H, blocks, nullptr, nullptr, nullptr, FLAT_KT)
              : block_space<T, false>(c, H, blocks, nullptr, nullptr, nullptr, tile_tokens<T, false>());
}
template <typename T>
hipError_t launch_block_attention(const CacheArgs& c, const BlockArgs& a, hipStream_t s) {
  return c.ks ? launch_blocks<T, true>(c, a, s) : launch_blocks<T, false>(c, a, s);
}
template size_t block_workspace_bytes<float>(const CacheArgs&, int, int);
template size_t block_workspace_bytes<bf16_t>(const CacheArgs&, int, int);
template hipError_t launch_block_attention<float>(const CacheArgs&, const BlockArgs&, hipStream_t);
template hipError_t launch_block_attention<bf16_t>(const CacheArgs&, const BlockArgs&, hipStream_t);

}  // namespace fusion
