// kv_attend_launch.h -- the launches of one head_dim; each kv_attend_<dim>.hip
// includes it with KV_DIM, so that the sizes compile side by side.
#include <algorithm>

#include "kv_attend.h"
#include "kv_host.h"

namespace uzip_kv {

// At most how many blocks the lists have, how many of them are split, and how many
// pieces there are.
static uint32_t blocks_bound(const AttendArgs &a, const Lists &l) {
  // full blocks and a last one for each list, or what lists of l.most rows can have
  const uint64_t lists = a.n_reqs + 1, all = (uint64_t)a.n_rows * a.group;
  const uint64_t each = l.most < all ? ((uint64_t)l.most + l.rows - 1) / l.rows : UINT32_MAX;
  return (uint32_t)(a.c.heads * std::min(all / l.rows + lists, lists * each));
}

static uint32_t most_split(const AttendArgs &a, const Lists &l) {
  return std::min(blocks_bound(a, l), (l.many ? l.per_unit : kFewPieces) * a.units);
}
static uint32_t most_pieces(const AttendArgs &a, const Lists &l) {
  return blocks_bound(a, l) + (l.many ? l.per_unit : kFewPieces) * a.units;
}

// No block has more than kMinSteps steps, so none is split.
static bool never_split(const AttendArgs &a) {
  return (uint64_t)a.max_pages * a.c.page <= (uint64_t)kMinSteps * kStep;
}

template <int T>
static void join(const AttendCall &c, const Lists &many, bool with_many, const Lists &few) {
  if (never_split(c.a)) return;
  const uint32_t n_many = with_many ? most_split(c.a, many) : 0, n_few = most_split(c.a, few);
  const uint32_t grid = n_many * (many.rows / kJoinRows) + n_few * (few.rows / kJoinRows);
  join_kernel<T, KV_DIM><<<grid, 256, 0, c.stream>>>(c.a, many, n_many, few);
}

template <int T, int CODE>
static void launch(const AttendCall &c) {
  const AttendArgs &a = c.a;
  const Layout at = layout(c.type, KV_DIM, a.c.heads, a.group, a.n_reqs, c.max_new);
  const Lists few{1, at.many ? many_from(KV_DIM) : UINT32_MAX, 16 * at.few, at.few == 1 ? 4u : 5u,
                  at.many ? 2 * many_pieces(KV_DIM) * a.units * kManyRows : 0, false, 0};
  const uint32_t n_few = most_pieces(a, few);
  if constexpr (T != UZIP_FP32) {
    if (at.many) {
      const Lists many{many_from(KV_DIM) + 1, UINT32_MAX, kManyRows, 7, 0, true, many_pieces(KV_DIM)};
      const uint32_t n_many = most_pieces(a, many);
      all_rows_kernel<T, CODE, KV_DIM><<<n_many + n_few, 256, 0, c.stream>>>(a, many, n_many, few);
      join<T>(c, many, true, few);
      return;
    }
  }
  if constexpr (has_two(T, KV_DIM)) {
    if (at.few == 2) few_rows_kernel<T, CODE, KV_DIM, 2><<<n_few, 256, 0, c.stream>>>(a, few);
  }
  if (at.few == 1) few_rows_kernel<T, CODE, KV_DIM, 1><<<n_few, 256, 0, c.stream>>>(a, few);
  join<T>(c, few, false, few);
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
