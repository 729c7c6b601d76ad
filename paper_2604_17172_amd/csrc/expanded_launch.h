// expanded_launch.h -- the launches of one width of keys; each expanded_<width>.hip includes it with
// EXPANDED_NOPE, so that the widths compile side by side.
#include "expanded.h"
#include "expanded_host.h"

namespace uzip_kv {

template <int T, int DR, int DV, int R, int RG, int SPLIT, bool DIRECT>
static uzip_status launch(const ExpandedCall &c) {
  typedef Expanded<EXPANDED_NOPE, DR, DV, R, RG, SPLIT> L;
  const auto kernel = expanded_kernel<T, EXPANDED_NOPE, DR, DV, R, RG, SPLIT, DIRECT>;
  // blocks: full ones, and a last one for each request and for the rows of none
  const uint64_t blocks = std::min<uint64_t>(c.a.n_rows, (uint64_t)c.a.n_rows / L::kRows + c.a.n_reqs + 1);
  if (hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(typename L::Lds)) != hipSuccess)
    return UZIP_EHIP;
  kernel<<<(uint32_t)(blocks * c.a.heads), L::kThreads, sizeof(typename L::Lds), c.stream>>>(c.a);
  return hipGetLastError() == hipSuccess ? UZIP_OK : UZIP_EHIP;
}
template <int T, int DR, int DV>
static uzip_status launch(const ExpandedCall &c) {
  if (!c.direct) return launch<T, DR, DV, 1, 1, 4, false>(c);
  return c.rows == 32 ? launch<T, DR, DV, 1, 1, 4, true>(c) : c.rows == 64 ? launch<T, DR, DV, 2, 1, 4, true>(c)
                                                                         : launch<T, DR, DV, 2, 2, expanded_by_eight(EXPANDED_NOPE, DR, DV) ? 4 : 2, true>(c);
}
template <int T>
static uzip_status launch(const ExpandedCall &c) {
  if (c.rot == 32) return c.value == 64 ? launch<T, 32, 64>(c) : launch<T, 32, 128>(c);
  return c.value == 64 ? launch<T, 64, 64>(c) : launch<T, 64, 128>(c);
}

template <>
uzip_status launch_expanded<EXPANDED_NOPE>(const ExpandedCall &c) {
  return c.type == UZIP_BF16 ? launch<UZIP_BF16>(c) : launch<UZIP_FP16>(c);
}

}  // namespace uzip_kv
