/*
 * uzip_kv.h -- paged 8-bit key/value cache on MI355X (gfx950): pages from
 * request lengths, the write of new tokens, and attention over the pages.
 *
 * The codec of uzip.h moves a request's cache from the GPU that read the
 * prompt to the one that answers (arXiv 2604.17172, section 5.3: transfer
 * between prefill and decode instances).  These calls are what both sides do
 * with it: the cache is held as FP8 codes, so its pages are coded as pairs
 * (UZIP_E4M3FN, UZIP_E5M2) without another conversion.
 *
 * Cache layout (P = page_tokens, D = head_dim, H = n_heads):
 *   k      u8 [n_pages][H][P][D]   codes of the keys
 *   v      u8 [n_pages][H][D][P]   codes of the values, a page transposed: a
 *                                  lane of the attention kernel takes its
 *                                  tokens of one channel in one load
 *   k_exp  u8 [n_pages][H]         exponent bytes: a key is code * 2^(e - 127)
 *   v_exp  u8 [n_pages][H]
 * One scale for each page and head, a power of two: a code's own exponent
 * makes finer scales useless, and scaling is then exact, so a value is
 * rounded once, where its code is made.
 *
 * Conventions, besides those of uzip.h (caller-owned device memory, no
 * allocation, work enqueued on the given stream, host-side errors returned
 * with nothing enqueued):
 *   - The cache arrays and the workspace are 16-byte aligned; every other
 *     array is aligned to its element.  Rows of q, k, v and out may lie at
 *     any element strides (slices of a fused projection); the D values of one
 *     head are contiguous.
 *   - head_dim is 64, 96, 128, 192 or 256; page_tokens 16, 32, 64, 128 or 256;
 *     n_pages * page_tokens < 2^31.
 *   - q, k, v and out are UZIP_BF16, UZIP_FP16 or UZIP_FP32; the cache's dtype is
 *     UZIP_E4M3FN or UZIP_E5M2 (here single codes, not pairs).
 *   - No call writes outside its outputs, whatever the lengths, pages, slots
 *     and runs on the device hold.  A page number outside [0, n_pages) is no
 *     page: nothing is stored to it and its tokens are not attended to.
 *   - A call keeps nothing for later calls; the results are the same bits
 *     whatever else runs on the GPU.  Calls that overlap in time need separate
 *     workspaces.
 */
#ifndef UZIP_KV_H
#define UZIP_KV_H

#include "uzip.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
  uint8_t *k;
  uint8_t *v;
  uint8_t *k_exp;
  uint8_t *v_exp;
  uint32_t n_pages;
  uint32_t n_heads;     /* heads of keys and values */
  uint32_t head_dim;
  uint32_t page_tokens;
  uzip_dtype dtype;     /* UZIP_E4M3FN or UZIP_E5M2 */
} uzip_kv_cache;

/* Requests of one plan, and rows of one call. */
#define UZIP_KV_MAX_REQUESTS 4096
#define UZIP_KV_MAX_ROWS (1u << 22)
#define UZIP_KV_MAX_ROW_HEADS (1u << 26) /* rows times query heads of one uzip_kv_attend */

/* Entries of d_runs: the most runs that n_rows new tokens of n_reqs requests
 * can make, at least 1.  Returns 0 for invalid arguments. */
uint32_t uzip_kv_max_runs(uint32_t n_rows, uint32_t n_reqs, uint32_t page_tokens);

/* One step's places.  Request i holds d_old[i] tokens in the pages that row i of
 * its block table names and takes d_new[i] more; its new rows lie one after
 * the other from row d_q_start[i] on, the requests in their order.
 *   d_free, n_free: pages to give out, taken from the front in the requests'
 *                order.
 *   n_rows:      rows that the step's arrays hold, >= the sum of d_new; rows
 *                past the sum belong to no request.
 *   d_table:     [n_reqs][max_pages]; entries ceil(old / P) up to
 *                ceil((old + new) / P) are written, no others.
 *   d_lens:      [n_reqs]     old + new
 *   d_q_start:   [n_reqs + 1] each request's first row, and the end of the last
 *   d_slots:     [n_rows]     page * P + place in the page; -1 for no place
 *   d_runs:      [max_runs][2] first row and rows of each run: the rows of one
 *                request that go to one page; entries past the count are
 *                not written
 *   d_counts:    [2]          pages taken from d_free; runs
 *   d_status:    device u32 (may be NULL): this call's UZIP_OK or error, whatever
 *                it held before, so each replay of a graph gives its own
 * A request whose pages are not to be had -- d_free at its end, or more than
 * max_pages of them (UZIP_ENOSPC) -- or whose lengths are negative or whose
 * rows do not fit n_rows (UZIP_EINVAL) takes no part: d_lens reads 0, its slots
 * -1, its table stays, and so it is with every later request that needs a page
 * once d_free is at its end.  If both errors occur the status is UZIP_ENOSPC.
 * The outputs are other arrays than d_old and d_new (EINVAL where d_lens is one of
 * them).  n_reqs <= UZIP_KV_MAX_REQUESTS.  Errors: EINVAL, EHIP, EUNSUPPORTED. */
uzip_status uzip_kv_plan(const int32_t *d_old, const int32_t *d_new, uint32_t n_reqs, const int32_t *d_free,
                         uint32_t n_free, uint32_t page_tokens, uint32_t n_rows, int32_t *d_table,
                         uint32_t max_pages, int32_t *d_lens, int32_t *d_q_start, int64_t *d_slots,
                         int32_t *d_runs, int32_t *d_counts, uint32_t *d_status, hipStream_t stream);

/* Store the new tokens' keys and values.  Row r's values of head h start at
 * d_k + r * k_row + h * k_head (elements; so for v).
 * For each run, head, and each of keys and values: e is the least exponent
 * byte in [27, 246] (e5m2: [27, 239]) with max |x| <= 448 (57344) * 2^(e - 127)
 * over the run's finite values, and not less than the page's own where the run
 * does not start the page; codes are x * 2^(127 - e) rounded to nearest even,
 * values past the largest code take that code.  Where e grew, the codes before the
 * run are rounded again; codes after it are left alone.  NaN gives the code
 * 0x7F with the value's sign; an infinity too in e4m3fn, which has none, and
 * the infinity in e5m2.
 *   d_slots, d_runs, d_counts: as uzip_kv_plan makes them; max_runs: entries of
 *                d_runs, whose number chooses the kernel.  Rows of a run have
 *                consecutive slots in one page, and no two runs of one call share
 *                a page.
 * Errors: EINVAL, EHIP, EUNSUPPORTED. */
uzip_status uzip_kv_store(const uzip_kv_cache *cache, uzip_dtype dtype, const void *d_k, int64_t k_row,
                          int64_t k_head, const void *d_v, int64_t v_row, int64_t v_head, uint32_t n_rows,
                          const int64_t *d_slots, const int32_t *d_runs, const int32_t *d_counts,
                          uint32_t max_runs, hipStream_t stream);

/* Workspace of uzip_kv_attend in bytes; 0 for invalid arguments. */
size_t uzip_kv_attend_workspace(uzip_dtype dtype, uint32_t n_rows, uint32_t n_q_heads, uint32_t n_heads,
                                uint32_t head_dim, uint32_t n_reqs, uint32_t max_new);

/* Attention of the new tokens over the pages, after they are stored.  Row j of
 * request i (j counted from its first row, n_i = d_q_start[i + 1] - d_q_start[i])
 * stands at place p = d_lens[i] - n_i + j and sees the places t with t <= p, t >=
 * 0 and, if window > 0, t > p - window:
 *   s_t = scale * sum_d q_d k_td     out_d = sum_t exp(s_t) v_td / sum_t exp(s_t)
 *   lse = log sum_t exp(s_t)
 * Query head a reads head a / (n_q_heads / n_heads) of the cache.  A row that sees
 * nothing (a request of length 0, a place before the first, a row past
 * d_q_start[n_reqs]) gives zeros and -infinity.  Products and sums are held in
 * 32 bits; probabilities enter the second product with at least 8 bits for
 * bf16, 16 for fp16 and 24 for fp32.
 * A value that is infinite or NaN is so for every row that sees it, however small its
 * weight.  Scores are scale * 2^(k_exp - 127) times the products of queries with codes,
 * and out is a sum of weights of at most 1 times values, over the sum of the weights:
 * where one of these passes the largest 32-bit number the results are not finite.
 *   max_new:     the most new tokens of a request.  It chooses kernels: a wrong
 *                value costs time, and the last bits may differ.
 *   d_table, max_pages, d_lens, d_q_start, n_reqs: as uzip_kv_plan leaves them; a
 *                length past max_pages * P counts as that.
 *   d_out:       row r, head a at d_out + r * out_row + a * out_head (elements).
 *   d_lse:       [n_rows][n_q_heads] (may be NULL).
 *   d_ws, ws_bytes: at least uzip_kv_attend_workspace.
 * n_q_heads is a multiple of n_heads <= 1024; n_rows * n_q_heads <=
 * UZIP_KV_MAX_ROW_HEADS; n_reqs <= UZIP_KV_MAX_REQUESTS.
 * Errors: EINVAL, ENOSPC, EHIP, EUNSUPPORTED. */
uzip_status uzip_kv_attend(const uzip_kv_cache *cache, uzip_dtype dtype, const void *d_q, int64_t q_row,
                           int64_t q_head, uint32_t n_rows, uint32_t n_q_heads, const int32_t *d_table,
                           uint32_t max_pages, const int32_t *d_lens, const int32_t *d_q_start, uint32_t n_reqs,
                           uint32_t max_new, float scale, uint32_t window, void *d_out, int64_t out_row,
                           int64_t out_head, float *d_lse, void *d_ws, size_t ws_bytes, hipStream_t stream);

#ifdef __cplusplus
}
#endif
#endif
