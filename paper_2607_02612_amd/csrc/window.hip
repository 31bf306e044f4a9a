// Attention over packed ragged rows under a sliding window with a few first
// rows that stay visible:
//   o_i = sum_{j in S_i} E_ij v_j / sum_{j in S_i} E_ij,
//   E_ij = exp(q_i k_j / sqrt(dh) + ln size_j - m_i),  m_i = max over S_i,
// S_i the rows of the sample that row i sees.
#include "kernels.h"

#include <algorithm>

namespace fusion {
namespace {

// Samples of one launch: their offsets and the first row tile of each, as
// kernel arguments (at most 4 KiB with the hidden ones).
constexpr int WIN_SEQS = 448;
struct WindowSeqs {
  int n;
  int cu[WIN_SEQS + 1];
  int tile[WIN_SEQS + 1];
};

// One wave per query row and head, one key per lane.
constexpr int WIN_ROWS = 4;  // rows per workgroup
template <typename T>
__global__ __launch_bounds__(256) void window_attention_valu(WindowArgs a, WindowSeqs sq) {
  const int tile = blockIdx.x, h = blockIdx.y;
  int lo = 0, hi = sq.n - 1;  // the last sample whose first tile is not after this one
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (sq.tile[mid] <= tile) lo = mid; else hi = mid - 1;
  }
  const int base = sq.cu[lo], n = sq.cu[lo + 1] - base;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int i = (tile - sq.tile[lo]) * WIN_ROWS + wave;
  if (i >= n) return;
  const int dh = a.dh, kh = h / a.group;
  __shared__ float qs[WIN_ROWS][128];
  const T* q = (const T*)a.q + (base + i) * a.q_row + h * a.q_head;
  for (int d = lane; d < dh; d += 64) qs[wave][d] = St<T>::get(q[d]) * a.scale;
  const T* kg = (const T*)a.k + base * a.k_row + kh * a.k_head;
  const T* vg = (const T*)a.v + base * a.v_row + kh * a.v_head;
  float m = -INFINITY, l = 0.f, o0 = 0.f, o1 = 0.f;
  for (int j0 = 0; j0 < n; j0 += 64) {
    const int j = j0 + lane;
    float s = -INFINITY;
    bool see = j < n && (i - j < a.window && j - i < a.window || j < a.sinks);
    if (a.causal && j > i) see = false;
    float lnsize = 0.f;
    if (see && a.size) {
      const float sz = a.size[base + j];
      see = sz > 0.f;
      lnsize = logf(sz);
    }
    if (see) {
      float dot = 0.f;
      for (int d = 0; d < dh; d++) dot = fmaf(qs[wave][d], St<T>::get(kg[j * a.k_row + d]), dot);
      s = dot + lnsize;
    }
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
      const T* v = vg + (j0 + t) * a.v_row;
      if (lane < dh) o0 = fmaf(p, St<T>::get(v[lane]), o0);
      if (64 + lane < dh) o1 = fmaf(p, St<T>::get(v[64 + lane]), o1);
    }
  }
  T* out = (T*)a.out + ((int64_t)(base + i) * a.H + h) * dh;
  const float r = l == 0.f ? 0.f : 1.f / l;
  if (lane < dh) out[lane] = St<T>::put(o0 * r);
  if (64 + lane < dh) out[64 + lane] = St<T>::put(o1 * r);
}

}  // namespace

template <typename T>
hipError_t launch_window_attention(const WindowArgs& a, const int32_t* cu_host, int batch,
                                   hipStream_t s) {
  for (int f = 0; f < batch; f += WIN_SEQS) {
    WindowSeqs sq;
    sq.n = std::min(batch - f, WIN_SEQS);
    int tiles = 0;
    for (int i = 0; i <= sq.n; i++) {
      sq.cu[i] = cu_host[f + i];
      sq.tile[i] = tiles;
      if (i < sq.n) tiles += (cu_host[f + i + 1] - cu_host[f + i] + WIN_ROWS - 1) / WIN_ROWS;
    }
    if (tiles == 0) continue;
    window_attention_valu<T><<<dim3(tiles, a.H), 256, 0, s>>>(a, sq);
    if (hipError_t e = hipGetLastError()) return e;
  }
  return hipSuccess;
}
template hipError_t launch_window_attention<float>(const WindowArgs&, const int32_t*, int,
                                                   hipStream_t);
template hipError_t launch_window_attention<bf16_t>(const WindowArgs&, const int32_t*, int,
                                                    hipStream_t);

}  // namespace fusion
