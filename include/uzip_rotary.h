/*
 * uzip_rotary.h -- rotary positions on MI355X (gfx950): of queries and keys, of
 * keys on their way into the paged 8-bit cache, and the places that they go by.
 *
 * A row at position p turns pair i of its head's rotary part by p * freq[i] radians:
 *   a' = m (a cos - b sin)   b' = m (a sin + b cos)
 * The conventions are those of uzip_kv.h.  Angles are taken in 64 bits, whatever the
 * position; turned values are products in 32 bits, rounded once.
 */
#ifndef UZIP_ROTARY_H
#define UZIP_ROTARY_H

#include "uzip_kv.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
  const int32_t *positions; /* [n_rows], may be negative */
  const float *freq;        /* [rot / 2] radians a position */
  uint32_t rot;             /* channels of the rotary part, even, 2 to 1024 */
  uint32_t first;           /* the channel where it begins */
  uint32_t interleaved;     /* 0: pairs (i, i + rot / 2); 1: pairs (2 i, 2 i + 1) */
  uint32_t inverse;         /* 1: the angle's sign changed, which is also the gradient */
  double magnitude;         /* m, on the rotary part alone; finite in 32 bits */
} uzip_turn;

/* The place of each row in its request, from what uzip_kv_plan leaves: row j of request i
 * is at d_lens[i] - (d_q_start[i + 1] - d_q_start[i]) + j.  -1 for rows of no request and
 * for rows of a request that took no part.
 * Errors: EINVAL, EHIP, EUNSUPPORTED. */
uzip_status uzip_kv_positions(const int32_t *d_lens, const int32_t *d_q_start, uint32_t n_reqs, uint32_t n_rows,
                              int32_t *d_positions, hipStream_t stream);

/* out[row][head] = x[row][head] turned; channels outside the rotary part are copied.
 * head_dim is any number up to 1024 with first + rot <= head_dim, n_heads up to 65535, n_rows *
 * n_heads up to UZIP_KV_MAX_ROW_HEADS.  d_out with d_x's
 * strides may be d_x; otherwise no value of the one lies on a value of the other.
 * Errors: EINVAL, EHIP, EUNSUPPORTED. */
uzip_status uzip_rotate(uzip_dtype dtype, const void *d_x, int64_t x_row, int64_t x_head, uint32_t n_rows,
                        uint32_t n_heads, uint32_t head_dim, const uzip_turn *turn, void *d_out, int64_t out_row,
                        int64_t out_head, hipStream_t stream);

/* uzip_kv_store with the keys turned first (in 32 bits: their codes are the only rounding),
 * and uzip_rotate of the step's queries (n_q_heads may be 0) in the same launch.
 * turn->inverse is 0.  Errors: EINVAL, EHIP, EUNSUPPORTED. */
uzip_status uzip_kv_rotate_store(const uzip_kv_cache *cache, uzip_dtype dtype, const void *d_k, int64_t k_row,
                                 int64_t k_head, const void *d_v, int64_t v_row, int64_t v_head, uint32_t n_rows,
                                 const int64_t *d_slots, const int32_t *d_runs, const int32_t *d_counts,
                                 uint32_t max_runs, const uzip_turn *turn, const void *d_q, int64_t q_row,
                                 int64_t q_head, uint32_t n_q_heads, void *d_q_out, int64_t out_row,
                                 int64_t out_head, hipStream_t stream);

#ifdef __cplusplus
}
#endif
#endif
