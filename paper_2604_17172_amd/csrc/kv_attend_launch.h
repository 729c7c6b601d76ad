// kv_attend_launch.h -- the launches of one head_dim; each kv_attend_<dim>.hip
// includes it with KV_DIM, so that the sizes compile side by side.
#include <algorithm>

#include "kv_attend.h"
#include "kv_host.h"

namespace uzip_kv {

template <int T, int CODE>
static void launch_few(const AttendCall &c, uint32_t blocks) {
  const AttendArgs &a = c.a;
  const uint64_t items = (uint64_t)a.c.heads * (((uint64_t)a.n_rows * a.group) / (16 * blocks) + a.n_reqs + 1);
  const uint32_t grid = (uint32_t)(items + a.target);
  const int64_t least = 1, most = INT64_MAX;
  if (blocks == 1) attend_few_kernel<T, CODE, KV_DIM, 1><<<grid, 256, 0, c.stream>>>(a, least, most);
  else if (blocks == 2) attend_few_kernel<T, CODE, KV_DIM, 2><<<grid, 256, 0, c.stream>>>(a, least, most);
  else if constexpr (KV_DIM <= 128) attend_few_kernel<T, CODE, KV_DIM, 4><<<grid, 256, 0, c.stream>>>(a, least, most);
  join_kernel<T, KV_DIM><<<(uint32_t)std::min<uint64_t>(items, a.target), 256, 0, c.stream>>>(a, 16 * blocks, least, most);
}

template <>
uzip_status launch_attend<KV_DIM>(const AttendCall &c) {
  const uint32_t blocks = few_blocks(KV_DIM, (uint64_t)c.max_new * c.a.group);
  const bool e5 = c.code == UZIP_E5M2;
  switch (c.type) {
    case UZIP_BF16: e5 ? launch_few<UZIP_BF16, UZIP_E5M2>(c, blocks) : launch_few<UZIP_BF16, UZIP_E4M3FN>(c, blocks); break;
    case UZIP_FP16: e5 ? launch_few<UZIP_FP16, UZIP_E5M2>(c, blocks) : launch_few<UZIP_FP16, UZIP_E4M3FN>(c, blocks); break;
    default: e5 ? launch_few<UZIP_FP32, UZIP_E5M2>(c, blocks) : launch_few<UZIP_FP32, UZIP_E4M3FN>(c, blocks); break;
  }
  return hipGetLastError() == hipSuccess ? UZIP_OK : UZIP_EHIP;
}

}  // namespace uzip_kv
