// Paged token caches: appending rows, attention of one new token per sequence
// with the accumulated attention weight of every cached token, and eviction
// by that weight.
#include "kernels.h"

#include <algorithm>

namespace fusion {
namespace {

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
// One workgroup per (query head, sequence), one key per lane; the scores and
// the softmax statistics of each head go to the workspace.
struct PagedSpace {
  float* score;  // [B][H][cap]
  float2* ml;    // [B][H]: maximum, sum
};
size_t round256(size_t v) { return (v + 255) & ~(size_t)255; }

template <typename T>
__global__ __launch_bounds__(256) void paged_attention_valu(CacheArgs c, PagedArgs a,
                                                            PagedSpace ws) {
  const int h = blockIdx.y, b = blockIdx.x, kh = h / a.group, dh = c.dh;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int n = held(c, b), last = c.seen[b] - 1;
  __shared__ float qs[128], part[4][128], pm[4], pl[4];
  if (threadIdx.x < dh)
    qs[threadIdx.x] = St<T>::get(((const T*)a.q)[b * a.q_row + h * a.q_head + threadIdx.x]) * a.scale;
  __syncthreads();
  float m = -INFINITY, l = 0.f, o0 = 0.f, o1 = 0.f;
  for (int x0 = wave * 64; x0 < n; x0 += 256) {
    const int x = x0 + lane;
    bool see = x < n;
    if (see) {
      const int pos = c.pos[(int64_t)b * c.cap + x];
      see = last - pos < a.window || pos < a.sinks;
    }
    int64_t ko = 0, vo = 0;
    if (see) {
      const uint32_t pg = quot((uint32_t)x, c.page);
      const int p = page_of(c, b, pg);
      const int64_t in_page = x - (int64_t)pg * c.page.d;
      see = p >= 0;
      ko = p * c.k_page + in_page * c.k_row + kh * c.k_head;
      vo = p * c.v_page + in_page * c.v_row + kh * c.v_head;
    }
    float s = -INFINITY;
    if (see) {
      s = 0.f;
      for (int d = 0; d < dh; d++) s = fmaf(qs[d], St<T>::get(((const T*)c.k)[ko + d]), s);
    }
    if (a.accumulate && x < n) ws.score[((int64_t)b * a.H + h) * c.cap + x] = s;
    const uint64_t seen = __ballot(see);
    if (!seen) continue;
    const float m2 = fmaxf(m, wave_max(s));
    const float e = see ? expf(s - m2) : 0.f, f = m == -INFINITY ? 0.f : expf(m - m2);
    l = l * f + wave_sum(e);
    o0 *= f;
    o1 *= f;
    m = m2;
    for (uint64_t left = seen; left; left &= left - 1) {
      const int t = __builtin_ctzll(left);
      const float p = __shfl(e, t, 64);
      const T* v = (const T*)c.v + __shfl(vo, t, 64);
      if (lane < dh) o0 = fmaf(p, St<T>::get(v[lane]), o0);
      if (64 + lane < dh) o1 = fmaf(p, St<T>::get(v[64 + lane]), o1);
    }
  }
  part[wave][lane] = o0;
  part[wave][64 + lane] = o1;
  if (lane == 0) {
    pm[wave] = m;
    pl[wave] = l;
  }
  __syncthreads();
  m = fmaxf(fmaxf(pm[0], pm[1]), fmaxf(pm[2], pm[3]));
  float o = 0.f;
  l = 0.f;
  for (int w = 0; w < 4; w++) {
    const float f = pm[w] == -INFINITY ? 0.f : expf(pm[w] - m);
    l += pl[w] * f;
    if (threadIdx.x < dh) o += part[w][threadIdx.x] * f;
  }
  if (threadIdx.x < dh)
    ((T*)a.out)[((int64_t)b * a.H + h) * dh + threadIdx.x] = St<T>::put(l == 0.f ? 0.f : o / l);
  if (threadIdx.x == 0) ws.ml[(int64_t)b * a.H + h] = make_float2(m, l);
}

__global__ __launch_bounds__(256) void paged_weight_kernel(CacheArgs c, PagedArgs a,
                                                           PagedSpace ws) {
  const int b = blockIdx.x, n = held(c, b);
  for (int x = blockIdx.y * 256 + threadIdx.x; x < n; x += gridDim.y * 256) {
    float w = 0.f;
    for (int h = 0; h < a.H; h++) {
      const float2 ml = ws.ml[(int64_t)b * a.H + h];
      const float s = ws.score[((int64_t)b * a.H + h) * c.cap + x];
      if (s != -INFINITY) w += expf(s - ml.x) / ml.y;
    }
    c.weight[(int64_t)b * c.cap + x] += w / (float)a.H;
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

size_t paged_workspace_bytes(const CacheArgs& c, int H, int accumulate) {
  return round256((size_t)c.B * H * 8) + (accumulate ? (size_t)c.B * H * c.cap * 4 : 0);
}

template <typename T>
hipError_t launch_paged_attention(const CacheArgs& c, const PagedArgs& a, hipStream_t s) {
  const PagedSpace ws{(float*)((char*)a.ws + round256((size_t)c.B * a.H * 8)), (float2*)a.ws};
  paged_attention_valu<T><<<dim3(c.B, a.H), 256, 0, s>>>(c, a, ws);
  if (a.accumulate) 
    paged_weight_kernel<<<dim3(c.B, std::min((c.cap + 255) / 256, 1024)), 256, 0, s>>>(c, a, ws);
  return hipGetLastError();
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
