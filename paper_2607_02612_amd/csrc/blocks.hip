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

constexpr int STRIDE_BLOCKS = 1 << 22;  // workgroups of a launch, which stride over the rest

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
// One workgroup per page of a sequence, of those that hold its newest slots: the
// threads take eight dims of a head and every n-th token each, and the parts meet
// in LDS.  Least and greatest are exact in any order; NaN has no part in them.
template <typename T, bool FOUR>
__global__ __launch_bounds__(256) void page_bounds(CacheArgs c, BoundsArgs a, FastDiv pieces, int touched) {
  __shared__ float s_lo[256][9], s_hi[256][9];
  const int tid = threadIdx.x, ps = (int)c.page.d, all = c.Hkv * (int)pieces.d;
  const int wide = min(all, 256), sets = 256 / wide;  // threads over the dims, and over the tokens
  const int mine = tid % wide, set = tid / wide;
  for (int64_t unit = blockIdx.x; unit < (int64_t)c.B * touched; unit += gridDim.x) {
    const int b = (int)(unit / touched), n = held(c, b);
    const int from = a.newest ? max(0, n - a.newest) / ps : 0;
    const int64_t pg = (int64_t)from + unit % touched;
    if (pg * ps >= n) continue;
    const int page = page_of(c, b, (uint32_t)pg), rows = (int)min((int64_t)ps, n - pg * ps);
    if (page < 0) continue;
    for (int p0 = 0; p0 < all; p0 += wide) {
      const int p = p0 + mine, h = (int)quot((uint32_t)p, pieces), d = (p - h * (int)pieces.d) * 8;
      float lo[8], hi[8];
#pragma unroll
      for (int i = 0; i < 8; i++) {
        lo[i] = INFINITY;
        hi[i] = -INFINITY;
      }
      if (p < all && set < sets) {
        for (int r = set; r < rows; r += 4 * sets) {
          float x[4][8];
#pragma unroll
          for (int u = 0; u < 4; u++) held8<T, FOUR>(c, page, min(r + u * sets, rows - 1), h, d, x[u]);
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
        s_lo[tid][i] = lo[i];
        s_hi[tid][i] = hi[i];
      }
      __syncthreads();
      if (p < all && set == 0) {
        for (int w = 1; w < sets; w++)
#pragma unroll
          for (int i = 0; i < 8; i++) {
            lo[i] = fminf(lo[i], s_lo[w * wide + tid][i]);
            hi[i] = fmaxf(hi[i], s_hi[w * wide + tid][i]);
          }
        const int64_t at = ((int64_t)page * c.Hkv + h) * c.dh + d;
        store8((T*)a.lo + at, lo);
        store8((T*)a.hi + at, hi);
      }
      __syncthreads();
    }
  }
}

// ------------------------------------------------------------------ scores --
// Value of lane ^ O within 16 lanes.
template <int O>
__device__ __forceinline__ double lane_xor_d(double v) {
  const uint64_t u = __double_as_longlong(v);
  const uint32_t lo = (uint32_t)lane_xor_i<O>((int)(uint32_t)u), hi = (uint32_t)lane_xor_i<O>((int)(u >> 32));
  return __longlong_as_double((uint64_t)hi << 32 | lo);
}

constexpr int SCORE_PAGES = 64;  // pages of a workgroup
constexpr int SCORE_HEADS = 32;  // query heads that it holds at a time

// 16 lanes take a page, eight dims each, and four pages one after the other.
template <typename T>
__global__ __launch_bounds__(256) void block_scores(CacheArgs c, BlockArgs a, float* score, int chunks) {
  __shared__ __attribute__((aligned(16))) float qs[SCORE_HEADS * 128];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int d = (lane & 15) * 8;
  for (int64_t unit = blockIdx.x; unit < (int64_t)c.B * c.Hkv * chunks; unit += gridDim.x) {
    const int chunk = (int)(unit % chunks), bk = (int)(unit / chunks), b = bk / c.Hkv, kh = bk % c.Hkv;
    const int n = held(c, b), pages = (int)quot((uint32_t)n + c.page.d - 1, c.page);
    const int p0 = chunk * SCORE_PAGES + wave * 16 + (lane >> 4);
    if (pages <= a.p.blocks || chunk * SCORE_PAGES >= pages) continue;  // (all are chosen, or none is here)
    float lo[4][8], hi[4][8], most[4];
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const int p = min(p0 + 4 * i, pages - 1), page = max(0, page_of(c, b, p));
      const int64_t at = ((int64_t)page * c.Hkv + kh) * c.dh + d;
      most[i] = -INFINITY;
#pragma unroll
      for (int j = 0; j < 8; j++) lo[i][j] = hi[i][j] = 0.f;
      if (d < c.dh) {
        load8((const T*)a.lo + at, lo[i]);
        load8((const T*)a.hi + at, hi[i]);
      }
    }
    for (int h0 = 0; h0 < a.p.group; h0 += SCORE_HEADS) {
      const int heads = min(SCORE_HEADS, a.p.group - h0);
      __syncthreads();
      for (int i = tid; i < heads * 16; i += 256) {
        const int h = i >> 4, e = (i & 15) * 8;
        float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (e < c.dh)
          load8((const T*)a.p.q + (int64_t)b * a.p.q_row +
                    (int64_t)(kh * a.p.group + h0 + h) * a.p.q_head + e, x);
        *(float4*)&qs[h * 128 + e] = make_float4(x[0], x[1], x[2], x[3]);
        *(float4*)&qs[h * 128 + e + 4] = make_float4(x[4], x[5], x[6], x[7]);
      }
      __syncthreads();
      for (int h = 0; h < heads; h++) {
        float q[8];
        *(float4*)q = *(const float4*)&qs[h * 128 + d];
        *(float4*)(q + 4) = *(const float4*)&qs[h * 128 + d + 4];
#pragma unroll
        for (int i = 0; i < 4; i++) {
          double s = 0.0;
#pragma unroll
          for (int j = 0; j < 8; j++) s = fma((double)q[j], (double)(q[j] >= 0.f ? hi[i][j] : lo[i][j]), s);
          s += lane_xor_d<1>(s);
          s += lane_xor_d<2>(s);
          s += lane_xor_d<4>(s);
          s += lane_xor_d<8>(s);
          const float f = (float)s;
          most[i] = f > most[i] || f != f ? f : most[i];
        }
      }
    }
    if ((lane & 15) == 0) {
#pragma unroll
      for (int i = 0; i < 4; i++)
        if (p0 + 4 * i < pages) score[(int64_t)bk * c.max_pages + p0 + 4 * i] = most[i];
    }
  }
}

// ------------------------------------------------------------------ choice --
// Order of the pages as unsigned integers: those always chosen above all, then
// pages whose score is NaN (an infinite key beside a zero: no bound), then by
// score, and pages that are not there below everything.
__device__ __forceinline__ uint32_t page_key(float score, bool always, bool there) {
  if (always) return 0xFFFFFFFFu;
  if (!there) return 0u;
  if (score != score) return 0xFFFFFFFEu;
  const uint32_t u = __float_as_uint(score + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// One workgroup per sequence and key head: the blocks-th largest key from the
// top by digits of 12, 10 and 10 bits (counts in LDS), then the chosen pages in
// order.
__global__ __launch_bounds__(256) void block_choose(CacheArgs c, BlockArgs a, const float* score, int* sel) {
  __shared__ int bins[4096], s_found[2], s_wave[4], s_count[4][2];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int blocks = a.p.blocks;
  for (int64_t bk = blockIdx.x; bk < (int64_t)c.B * c.Hkv; bk += gridDim.x) {
    const int b = (int)(bk / c.Hkv), n = held(c, b);
    const int pages = (int)quot((uint32_t)n + c.page.d - 1, c.page);
    int* chosen = a.chosen + bk * blocks;
    int* at = sel + bk * blocks;
    if (pages <= blocks) {
      for (int i = tid; i < blocks; i += 256) {
        chosen[i] = i < pages ? i : -1;
        at[i] = i < pages ? page_of(c, b, i) : -1;
      }
      continue;
    }
    const float* sc = score + bk * c.max_pages;
    auto key_of = [&](int p) {
      return page_key(sc[p], p < a.first || p >= pages - a.recent, page_of(c, b, p) >= 0);
    };
    uint32_t least = 0;  // keys above it are chosen
    int want = blocks;   // and the first `want` of those equal to it
    for (int round = 0; round < 3; round++) {
      const int shift = round == 0 ? 20 : round == 1 ? 10 : 0, nb = round ? 1024 : 4096;
      __syncthreads();
      for (int i = tid; i < nb; i += 256) bins[i] = 0;
      __syncthreads();
      for (int p = tid; p < pages; p += 256) {
        const uint32_t k = key_of(p);
        if (round == 0 || k >> (shift + 10) == least >> (shift + 10)) atomicAdd(&bins[k >> shift & (nb - 1)], 1);
      }
      __syncthreads();
      // thread t sums the bins nb - per (t + 1) .. + per - 1
      const int per = nb / 256;
      int mine = 0;
      for (int i = 1; i <= per; i++) mine += bins[nb - tid * per - i];
      const int upto = wave_scan(mine);
      if (lane == 63) s_wave[wave] = upto;
      __syncthreads();
      int above = upto - mine;
      for (int w = 0; w < wave; w++) above += s_wave[w];
      if (above < want && above + mine >= want) {
        int i = nb - tid * per - 1, left = want - above;
        for (; left > bins[i]; i--) left -= bins[i];
        s_found[0] = i;
        s_found[1] = left == bins[i] ? 0 : left;
      }
      __syncthreads();
      least |= (uint32_t)s_found[0] << shift;
      want = s_found[1];
      if (want == 0) break;  // the whole bin is chosen
    }
    if (want == 0) least--;  // (not the lowest bin, since there are more pages than blocks)
    int done = 0, ties = 0;
    const uint64_t below = (1ull << lane) - 1;
    for (int p0 = 0; p0 < pages; p0 += 256) {
      const int p = p0 + tid;
      const uint32_t k = p < pages ? key_of(p) : 0u;
      const uint64_t more = __ballot(p < pages && k > least), same = __ballot(p < pages && k == least);
      __syncthreads();
      if (lane == 0) {
        s_count[wave][0] = (int)__popcll(more);
        s_count[wave][1] = (int)__popcll(same);
      }
      __syncthreads();
      int m = done, t = ties, all_m = 0, all_t = 0;
      for (int w = 0; w < 4; w++) {
        if (w < wave) {
          m += s_count[w][0];
          t += s_count[w][1];
        }
        all_m += s_count[w][0];
        all_t += s_count[w][1];
      }
      m += (int)__popcll(more & below);
      t += (int)__popcll(same & below);
      // (of the equal ones before p the first `want` were taken)
      const bool take = more >> lane & 1 || ((same >> lane & 1) && t < want);
      if (take) {
        const int i = m + min(t, want);
        chosen[i] = p;
        at[i] = page_of(c, b, p);
      }
      done += all_m;
      ties += all_t;
    }
  }
}

template <typename T, bool FOUR>
size_t block_space(const CacheArgs& c, int H, int blocks, char* ws, PagedSpace* space, float** score) {
  size_t n = paged_space<T, FOUR>(c, H, 0, ws, space);
  if (space) {
    *score = (float*)(ws + n);
    space->sel = (const int*)(ws + n + round256((size_t)c.B * c.Hkv * c.max_pages * 4));
  }
  return n + round256((size_t)c.B * c.Hkv * c.max_pages * 4) + round256((size_t)c.B * c.Hkv * blocks * 4);
}

template <typename T, bool FOUR>
hipError_t launch_blocks(const CacheArgs& c, const BlockArgs& a, hipStream_t s) {
  PagedSpace ws;
  float* score;
  block_space<T, FOUR>(c, a.p.H, a.p.blocks, (char*)a.p.ws, &ws, &score);
  const int chunks = (c.max_pages + SCORE_PAGES - 1) / SCORE_PAGES;
  const int64_t heads = (int64_t)c.B * c.Hkv;
  if (c.max_pages > a.p.blocks) {
    block_scores<T><<<(unsigned)std::min<int64_t>(heads * chunks, STRIDE_BLOCKS), 256, 0, s>>>(c, a, score, chunks);
    if (hipError_t e = hipGetLastError()) return e;
  }
  block_choose<<<(unsigned)std::min<int64_t>(heads, STRIDE_BLOCKS), 256, 0, s>>>(c, a, score, (int*)ws.sel);
  if (hipError_t e = hipGetLastError()) return e;
  return launch_paged_by_width<T, FOUR, true>(c, a.p, ws, s);
}
}  // namespace

template <typename T>
hipError_t launch_page_bounds(const CacheArgs& c, const BoundsArgs& a, hipStream_t s) {
  const FastDiv pieces = fast_div((uint32_t)c.dh / 8);
  const int ps = (int)c.page.d;
  int64_t touched = c.max_pages;
  if (a.newest) touched = std::min<int64_t>(touched, (a.newest - 1) / ps + 2);
  const unsigned grid = (unsigned)std::min<int64_t>(c.B * touched, STRIDE_BLOCKS);
  if (c.ks)
    page_bounds<T, true><<<grid, 256, 0, s>>>(c, a, pieces, (int)touched);
  else
    page_bounds<T, false><<<grid, 256, 0, s>>>(c, a, pieces, (int)touched);
  return hipGetLastError();
}
template hipError_t launch_page_bounds<float>(const CacheArgs&, const BoundsArgs&, hipStream_t);
template hipError_t launch_page_bounds<bf16_t>(const CacheArgs&, const BoundsArgs&, hipStream_t);

template <typename T>
size_t block_workspace_bytes(const CacheArgs& c, int H, int blocks) {
  return c.ks ? block_space<T, true>(c, H, blocks, nullptr, nullptr, nullptr)
              : block_space<T, false>(c, H, blocks, nullptr, nullptr, nullptr);
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
