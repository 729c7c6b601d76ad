// kv_attend_launch.h -- the launches of one head_dim; each kv_attend_<dim>.hip
// includes it with KV_DIM, so that the sizes compile side by side.
#include <algorithm>

#include "kv_attend.h"
#include "kv_host.h"

namespace uzip_kv {

// Work for one kernel: lists of `least` to `most` rows in blocks of `rows`.
struct Share {
  uint32_t rows, grid, joins;  // workgroups: pieces, and blocks that can be split
  int64_t least, most;
};

static Share share_of(const AttendArgs &a, uint32_t rows, int64_t least, int64_t most) {
  // blocks: full ones and a last one for each list, or what lists of `most` can have
  const uint64_t lists = a.n_reqs + 1, all = (uint64_t)a.n_rows * a.group;
  const uint64_t each = most < (int64_t)all ? ((uint64_t)most + rows - 1) / rows : UINT64_MAX / lists;
  const uint64_t blocks = a.c.heads * std::min(all / rows + lists, lists * each);
  return {rows, (uint32_t)(blocks + a.target), (uint32_t)std::min<uint64_t>(blocks, a.target), least, most};
}

template <int T, int CODE>
static void launch_few(const AttendCall &c, uint32_t blocks, int64_t most) {
  const AttendArgs &a = c.a;
  const Share s = share_of(a, 16 * blocks, 1, most);
  if (blocks == 1) attend_few_kernel<T, CODE, KV_DIM, 1><<<s.grid, 256, 0, c.stream>>>(a, s.least, s.most);
  else if (blocks == 2) attend_few_kernel<T, CODE, KV_DIM, 2><<<s.grid, 256, 0, c.stream>>>(a, s.least, s.most);
  else if constexpr (KV_DIM <= 128) attend_few_kernel<T, CODE, KV_DIM, 4><<<s.grid, 256, 0, c.stream>>>(a, s.least, s.most);
  join_kernel<T, KV_DIM><<<dim3(s.joins, (s.rows + kJoinRows - 1) / kJoinRows), 64 * kJoinRows, 0, c.stream>>>(a, s.rows, false, s.least, s.most);
}

template <int T, int CODE>
static void launch(const AttendCall &c) {
  const AttendArgs &a = c.a;
  const uint64_t list = (uint64_t)c.max_new * a.group;
  if constexpr (T != UZIP_FP32) {
    if (many_rows(c.type, list)) {
      const Share s = share_of(a, 128, kManyFrom + 1, INT64_MAX);
      attend_many_kernel<T, CODE, KV_DIM><<<s.grid, 256, 0, c.stream>>>(a, s.least, s.most);
      join_kernel<T, KV_DIM><<<dim3(s.joins, (s.rows + kJoinRows - 1) / kJoinRows), 64 * kJoinRows, 0, c.stream>>>(a, s.rows, true, s.least, s.most);
      launch_few<T, CODE>(c, few_blocks(KV_DIM, a.group), kManyFrom);  // sized for the requests of one token
      return;
    }
  }
  launch_few<T, CODE>(c, few_blocks(KV_DIM, list), INT64_MAX);
}

template <>
uzip_status launch_attend<KV_DIM>(const AttendCall &c) {
  const bool e5 = c.code == UZIP_E5M2;
  switch (c.type) {
    case UZIP_BF16: e5 ? launch<UZIP_BF16, UZIP_E5M2>(c) : launch<UZIP_BF16, UZIP_E4M3FN>(c); break;
    case UZIP_FP16: e5 ? launch<UZIP_FP16, UZIP_E5M2>(c) : launch<UZIP_FP16, UZIP_E4M3FN>(c); break;
    default: e5 ? launch<UZIP_FP32, UZIP_E5M2>(c) : launch<UZIP_FP32, UZIP_E4M3FN>(c); break;
  }
  return hipGetLastError() == hipSuccess ? UZIP_OK : UZIP_EHIP;
}

}  // namespace uzip_kv
