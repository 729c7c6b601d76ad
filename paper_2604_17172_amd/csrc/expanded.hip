// expanded.hip -- entry point of attention in the expanded form.
#include <cmath>

#include "expanded_host.h"

using namespace uzip_kv;

extern "C" {

uzip_status uzip_latent_attend_expanded(uzip_dtype dtype, const void *d_q, int64_t q_row, int64_t q_head, uint32_t n_rows,
                                        uint32_t n_heads, const void *d_k, int64_t k_row, int64_t k_head,
                                        const void *d_rot, int64_t rot_row, const void *d_v, int64_t v_row,
                                        int64_t v_head, uint32_t n_keys, uint32_t nope, uint32_t rot, uint32_t value,
                                        const int32_t *d_q_start, const int32_t *d_k_start, uint32_t n_reqs,
                                        uint32_t max_new, float scale, void *d_out, int64_t out_row, int64_t out_head,
                                        float *d_lse, hipStream_t stream) {
  if ((dtype != UZIP_BF16 && dtype != UZIP_FP16) || (nope != 64 && nope != 128) || (rot != 32 && rot != 64) || (value != 64 && value != 128) ||
      n_heads == 0 || n_heads > 1024 || n_rows > UZIP_KV_MAX_ROWS || n_keys > UZIP_KV_MAX_ROWS || n_reqs > UZIP_KV_MAX_REQUESTS ||
      (uint64_t)n_rows * n_heads > UZIP_KV_MAX_ROW_HEADS || !(scale - scale == 0))
    return UZIP_EINVAL;
  if (!aligned(d_q_start, 4) || !aligned(d_k_start, 4) || !aligned(d_lse, 4)) return UZIP_EINVAL;
  if (n_rows == 0) return UZIP_OK;
  if (!valid_rows(d_q, q_row, q_head, 2) || !valid_rows(d_out, out_row, out_head, 2) || !d_q_start || (n_reqs && !d_k_start)) return UZIP_EINVAL;
  if (n_keys && (!valid_rows(d_k, k_row, k_head, 2) || !valid_rows(d_rot, rot_row, 0, 2) || !valid_rows(d_v, v_row, v_head, 2))) return UZIP_EINVAL;
  if (const uzip_status s = device(nullptr); s != UZIP_OK) return s;
  ExpandedCall c{};
  c.a = {d_q, d_k, d_rot, d_v, d_out, d_lse, q_row, q_head, k_row, k_head, rot_row, v_row, v_head, out_row, out_head, d_q_start, d_k_start,
         n_rows, n_keys, n_heads, n_reqs, scale == 0 ? 1.0f : std::fabs(scale) * 1.4426950408889634f, scale < 0, scale == 0, false, false};
  auto at_multiples = [&](const void *p, int64_t row, int64_t head, int64_t of) { return aligned(p, of) && row * 2 % of == 0 && head * 2 % of == 0; };
  auto near = [&](int64_t row) { return row >= 0 && row < 1 << 23; };  // a row's bytes within 24 bits
  c.direct = at_multiples(d_k, k_row, k_head, 16) && at_multiples(d_rot, rot_row, 0, 16) && at_multiples(d_v, v_row, v_head, 16) && near(k_row) &&
               near(rot_row) && near(v_row);
  c.a.q_vec = at_multiples(d_q, q_row, q_head, 16);
  c.a.out_vec = at_multiples(d_out, out_row, out_head, 8);
  c.type = dtype;
  c.rot = rot;
  c.value = value;
  // Rows of a workgroup.  Four waves take 128 rows (two by two, each pair half of the tokens; or eight waves, a quarter each), or
  // 64 or 32 rows (each wave a quarter of the tokens): fewer where that leaves compute units idle.  In bf16, 128 + 64 and 128 channels, us with
  // 128, 64, 32 rows: 1024 tokens of 8 heads 29, 21, 16; 2048 of 16 heads 49, 44, 63; 4 x 1024 of 16 heads 54, 66, 94;
  // 8 x 512 of 8 heads 24, 33, 42; 32 x 64 behind 1000 of 16 heads 77, 74, 103; 64 x 30 behind 1000 of 8 heads 71, 70, 67.
  auto blocks = [&](uint32_t rows) { return ((uint64_t)n_rows / rows + n_reqs + 1) * n_heads; };
  c.rows = max_new <= 32 || blocks(32) <= 320 ? 32 : max_new <= 64 || blocks(64) <= (expanded_by_eight(nope, rot, value) ? 512 : 560) ? 64 : 128;
  c.stream = stream;
  return nope == 64 ? launch_expanded<64>(c) : launch_expanded<128>(c);
}

}  // extern "C"
