// Attention of one new token per sequence over a paged cache in 4 bits.
#include "paged.h"

namespace fusion {

template <typename T>
size_t paged4_workspace_bytes(const CacheArgs& c, int H, int accumulate) {
  return paged_space<T, true>(c, H, accumulate, nullptr, nullptr, FLAT_KT);
}

template <typename T>
hipError_t launch_paged4_attention(const CacheArgs& c, const PagedArgs& a, hipStream_t s) {
  PagedSpace ws;
  paged_space<T, true>(c, a.H, a.accumulate, (char*)a.ws, &ws, paged_tile<T, true>(a));
  return launch_paged_by_width<T, true, false>(c, a, ws, s);
}
template size_t paged4_workspace_bytes<float>(const CacheArgs&, int, int);
template size_t paged4_workspace_bytes<bf16_t>(const CacheArgs&, int, int);
template hipError_t launch_paged4_attention<float>(const CacheArgs&, const PagedArgs&, hipStream_t);
template hipError_t launch_paged4_attention<bf16_t>(const CacheArgs&, const PagedArgs&, hipStream_t);

}  // namespace fusion
