// kv_cache.hip -- pages, slots and runs from request lengths, and the write of
// new tokens into the 8-bit pages.
#include <algorithm>
#include <mutex>

#include "kv_device.h"
#include "kv_host.h"

namespace uzip_kv {

uzip_status device(int *cus) {
  constexpr int kMaxDevices = 64;
  struct Info {
    std::once_flag once;
    hipError_t err = hipSuccess;
    bool gfx950 = false;
    int cus = 0;
  };
  static Info info[kMaxDevices];
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) return UZIP_EHIP;
  Info &i = info[dev];
  std::call_once(i.once, [&]() {
    hipDeviceProp_t prop;
    i.err = hipGetDeviceProperties(&prop, dev);
    if (i.err != hipSuccess) return;
    i.gfx950 = strncmp(prop.gcnArchName, "gfx950", 6) == 0;
    i.cus = prop.multiProcessorCount;
  });
  if (i.err != hipSuccess) return UZIP_EHIP;
  if (cus) *cus = i.cus;
  return i.gfx950 ? UZIP_OK : UZIP_EUNSUPPORTED;
}

namespace {

// ------------------------------------------------------------------ plan
// Every workgroup takes the prefix sums over all requests for itself (three
// scans of at most 4096 lengths in LDS) and then writes its own rows, so one
// launch does it all and no workgroup waits for another.
constexpr int kPlanThreads = 256, kPlanRows = 1024;

struct PlanArgs {
  const int32_t *old_lens, *new_lens, *free_pages;
  int32_t *table, *lens, *q_start, *runs, *counts;
  int64_t *slots;
  int *status;
  uint32_t n_reqs, n_free, shift, n_rows, max_pages;
};

// Exclusive sum of v over the workgroup's threads; *total gets the sum of all.
__device__ int64_t block_scan(int64_t v, int64_t *part, int64_t *total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int64_t x = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t y = __shfl_up(x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();
  if (lane == 63) part[wave] = x;
  __syncthreads();
  int64_t before = 0, all = 0;
  for (int w = 0; w < kPlanThreads / 64; ++w) {
    if (w < wave) before += part[w];
    all += part[w];
  }
  *total = all;
  return before + x - v;
}

__global__ __launch_bounds__(kPlanThreads) void plan_kernel(PlanArgs a) {
  __shared__ int32_t first_row[UZIP_KV_MAX_REQUESTS + 1];
  __shared__ int32_t first_page[UZIP_KV_MAX_REQUESTS];  // -1: the request takes no part
  __shared__ int32_t first_run[UZIP_KV_MAX_REQUESTS];
  __shared__ int64_t part[kPlanThreads / 64];
  const uint32_t tid = threadIdx.x, n = a.n_reqs, P = 1u << a.shift;
  const uint32_t each = (n + kPlanThreads - 1) / kPlanThreads, lo = min(n, tid * each), hi = min(n, lo + each);
  int64_t total_rows, total_pages, total_runs;
  int error = 0;
  auto pages = [&](int64_t tokens) { return (tokens + P - 1) >> a.shift; };

  int64_t sum = 0;
  for (uint32_t i = lo; i < hi; ++i) sum += max(a.new_lens[i], 0);
  int64_t at = block_scan(sum, part, &total_rows);
  int64_t need = 0;
  for (uint32_t i = lo; i < hi; ++i) {
    const int64_t o = a.old_lens[i], w = a.new_lens[i];
    first_row[i] = (int32_t)min(at, (int64_t)a.n_rows);
    at += max(w, (int64_t)0);
    int32_t ok = 0;
    if (o < 0 || w < 0 || at > a.n_rows || o + w > INT32_MAX)
      error = min(error, (int)UZIP_EINVAL), ok = -1;
    else if (pages(o + w) > a.max_pages)
      error = min(error, (int)UZIP_ENOSPC), ok = -1;
    else
      need += pages(o + w) - pages(o);
    first_page[i] = ok;
  }
  if (tid == 0) first_row[n] = (int32_t)min(total_rows, (int64_t)a.n_rows);

  at = block_scan(need, part, &total_pages);
  int64_t taken = 0, runs = 0;
  for (uint32_t i = lo; i < hi; ++i) {
    if (first_page[i] < 0) continue;
    const int64_t o = a.old_lens[i], w = a.new_lens[i], take = pages(o + w) - pages(o);
    if (take > 0 && at + take > a.n_free) {
      error = min(error, (int)UZIP_ENOSPC);
      first_page[i] = -1;
    } else {
      first_page[i] = (int32_t)min(at, (int64_t)INT32_MAX);  // past the list only where no page is taken
      taken += take;
      if (w > 0) runs += ((o + w - 1) >> a.shift) - (o >> a.shift) + 1;
    }
    at += take;
  }

  at = block_scan(runs, part, &total_runs);
  for (uint32_t i = lo; i < hi; ++i) {
    if (first_page[i] < 0) continue;
    const int64_t o = a.old_lens[i], w = a.new_lens[i];
    first_run[i] = (int32_t)at;
    if (w > 0) at += ((o + w - 1) >> a.shift) - (o >> a.shift) + 1;
  }
  block_scan(taken, part, &total_pages);  // its barriers also end the writes of the tables above
  if (blockIdx.x == 0) {
    if (tid == 0) {
      a.counts[0] = (int32_t)total_pages;
      a.counts[1] = (int32_t)total_runs;
    }
    if (error && a.status) atomicMin(a.status, error);
  }

  for (uint32_t i = blockIdx.x * kPlanThreads + tid; i <= n; i += gridDim.x * kPlanThreads) {
    a.q_start[i] = first_row[i];
    if (i < n) a.lens[i] = first_page[i] < 0 ? 0 : a.old_lens[i] + a.new_lens[i];
  }
  const uint32_t end = min(a.n_rows, (blockIdx.x + 1) * (uint32_t)kPlanRows), used = (uint32_t)first_row[n];
  for (uint32_t r = blockIdx.x * kPlanRows + tid; r < end; r += kPlanThreads) {
    int64_t slot = -1;
    if (r < used) {
      uint32_t i = 0, top = n;  // the last request whose first row is not past r
      while (top - i > 1) {
        const uint32_t mid = (i + top) / 2;
        if ((uint32_t)first_row[mid] <= r) i = mid;
        else top = mid;
      }
      if (first_page[i] >= 0) {
        const uint32_t o = (uint32_t)a.old_lens[i], j = r - (uint32_t)first_row[i], pos = o + j;
        const uint32_t k = pos >> a.shift, off = pos & (P - 1), have = (uint32_t)pages(o);
        int32_t *entry = a.table + (size_t)i * a.max_pages + k;
        int32_t page;
        if (k < have) {
          page = *entry;
        } else {
          page = a.free_pages[(uint32_t)first_page[i] + (k - have)];
          if (off == 0) *entry = page;
        }
        slot = page < 0 ? -1 : ((int64_t)page << a.shift) + off;
        if (j == 0 || off == 0) {
          int32_t *run = a.runs + 2 * (size_t)(first_run[i] + (k - (o >> a.shift)));
          run[0] = (int32_t)r;
          run[1] = (int32_t)min(P - off, (uint32_t)a.new_lens[i] - j);
        }
      }
    }
    a.slots[r] = slot;
  }
}

// ------------------------------------------------------------------ store
struct StoreArgs {
  Cache c;
  const void *x[2];
  int64_t row[2], head[2];
  const int64_t *slots;
  const int32_t *runs, *counts;
  uint32_t n_rows;
};

constexpr int kStoreThreads = 256;

// One workgroup for a run, a head, and keys (z = 0) or values (z = 1): the
// largest finite magnitude, the page's exponent, the codes.
template <int T, int CODE>
__global__ __launch_bounds__(kStoreThreads) void store_kernel(StoreArgs a) {
  typedef typename Elem<T>::type Value;
  __shared__ float part[kStoreThreads / 64];
  if ((int32_t)blockIdx.x >= a.counts[1]) return;
  const uint32_t z = blockIdx.z, h = blockIdx.y, tid = threadIdx.x, D = a.c.dim, P = a.c.page;
  const int32_t row = a.runs[2 * (size_t)blockIdx.x];
  int32_t n = a.runs[2 * (size_t)blockIdx.x + 1];
  if (row < 0 || n <= 0 || (uint32_t)row >= a.n_rows) return;
  const int64_t slot = a.slots[row];
  if (slot < 0 || (uint64_t)slot >= (uint64_t)a.c.n_pages << a.c.page_shift) return;
  const uint32_t page = (uint32_t)(slot >> a.c.page_shift), off = (uint32_t)slot & (P - 1);
  n = min((uint32_t)n, min(P - off, a.n_rows - (uint32_t)row));
  const Value *x = (const Value *)a.x[z] + (int64_t)row * a.row[z] + (int64_t)h * a.head[z];
  const size_t ph = (size_t)page * a.c.heads + h;
  uint8_t *codes = (z ? a.c.v : a.c.k) + ph * P * D;
  uint8_t *exps = z ? a.c.v_exp : a.c.k_exp;
  auto place = [&](uint32_t t, uint32_t d) -> uint8_t & { return codes[z ? d * P + t : t * D + d]; };

  float amax = 0;
  for (uint32_t i = tid; i < (uint32_t)n * D; i += kStoreThreads) {
    const float f = fabsf((float)x[(int64_t)(i / D) * a.row[z] + i % D]);
    if (f < INFINITY) amax = fmaxf(amax, f);
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) amax = fmaxf(amax, __shfl_xor(amax, o));
  if ((tid & 63) == 0) part[tid >> 6] = amax;
  const int was = off ? exps[ph] : 0;
  __syncthreads();
  for (int w = 0; w < kStoreThreads / 64; ++w) amax = fmaxf(amax, part[w]);
  const int e = max(exponent_for<CODE>(amax), was);
  if (tid == 0 && e != was) exps[ph] = (uint8_t)e;
  const float inv = pow2(254 - e);
  for (uint32_t i = tid; i < (uint32_t)n * D; i += kStoreThreads)
    place(off + i / D, i % D) = (uint8_t)encode<CODE>((float)x[(int64_t)(i / D) * a.row[z] + i % D], inv);
  if (off && e > was) {
    const float down = pow2(max(127 + was - e, 0));
    for (uint32_t i = tid; i < off * D; i += kStoreThreads) {
      uint8_t &c = place(i / D, i % D);
      c = (uint8_t)recode<CODE>(c, down);
    }
  }
}

bool run_bound(uint32_t n_rows, uint32_t n_reqs, uint32_t page, uint64_t *bound) {
  if (!valid_page(page) || n_rows > UZIP_KV_MAX_ROWS || n_reqs > UZIP_KV_MAX_REQUESTS) return false;
  *bound = std::max<uint64_t>(1, std::min<uint64_t>(n_rows, (uint64_t)n_rows / page + 2ull * n_reqs));
  return true;
}

}  // namespace
}  // namespace uzip_kv

using namespace uzip_kv;

extern "C" {

uint32_t uzip_kv_max_runs(uint32_t n_rows, uint32_t n_reqs, uint32_t page_tokens) {
  uint64_t bound = 0;
  return run_bound(n_rows, n_reqs, page_tokens, &bound) ? (uint32_t)bound : 0;
}

uzip_status uzip_kv_plan(const int32_t *d_old, const int32_t *d_new, uint32_t n_reqs, const int32_t *d_free,
                         uint32_t n_free, uint32_t page_tokens, uint32_t n_rows, int32_t *d_table,
                         uint32_t max_pages, int32_t *d_lens, int32_t *d_q_start, int64_t *d_slots,
                         int32_t *d_runs, int32_t *d_counts, uint32_t *d_status, hipStream_t stream) {
  if (!valid_page(page_tokens) || n_reqs > UZIP_KV_MAX_REQUESTS || n_rows > UZIP_KV_MAX_ROWS ||
      n_free > INT32_MAX || max_pages > INT32_MAX)
    return UZIP_EINVAL;
  if (n_reqs && (!d_old || !d_new || !d_lens || (max_pages && !d_table))) return UZIP_EINVAL;
  if ((n_free && !d_free) || (n_rows && (!d_slots || !d_runs)) || !d_q_start || !d_counts) return UZIP_EINVAL;
  for (const void *p : {(const void *)d_old, (const void *)d_new, (const void *)d_free, (const void *)d_table,
                        (const void *)d_lens, (const void *)d_q_start, (const void *)d_runs, (const void *)d_counts,
                        (const void *)d_status})
    if (!aligned(p, 4)) return UZIP_EINVAL;
  if (!aligned(d_slots, 8)) return UZIP_EINVAL;
  if (const uzip_status s = device(nullptr); s != UZIP_OK) return s;
  PlanArgs a{d_old, d_new, d_free, d_table, d_lens, d_q_start, d_runs, d_counts, d_slots, (int *)d_status,
             n_reqs, n_free, (uint32_t)__builtin_ctz(page_tokens), n_rows, max_pages};
  const uint32_t grid = std::max(1u, (n_rows + kPlanRows - 1) / kPlanRows);
  plan_kernel<<<grid, kPlanThreads, 0, stream>>>(a);
  return hipGetLastError() == hipSuccess ? UZIP_OK : UZIP_EHIP;
}

uzip_status uzip_kv_store(const uzip_kv_cache *cache, uzip_dtype dtype, const void *d_k, int64_t k_row,
                          int64_t k_head, const void *d_v, int64_t v_row, int64_t v_head, uint32_t n_rows,
                          const int64_t *d_slots, const int32_t *d_runs, const int32_t *d_counts,
                          uint32_t max_runs, hipStream_t stream) {
  if (!valid_cache(cache) || !valid_type(dtype) || n_rows > UZIP_KV_MAX_ROWS || max_runs > UZIP_KV_MAX_ROWS)
    return UZIP_EINVAL;
  if (n_rows == 0 || max_runs == 0) return UZIP_OK;
  if (!valid_rows(d_k, k_row, k_head, type_bytes(dtype)) || !valid_rows(d_v, v_row, v_head, type_bytes(dtype)) ||
      !d_slots || !d_runs || !d_counts || !aligned(d_slots, 8) || !aligned(d_runs, 4) || !aligned(d_counts, 4))
    return UZIP_EINVAL;
  if (const uzip_status s = device(nullptr); s != UZIP_OK) return s;
  StoreArgs a{{cache->k, cache->v, cache->k_exp, cache->v_exp, cache->n_pages, cache->n_heads, cache->head_dim,
               cache->page_tokens, (uint32_t)__builtin_ctz(cache->page_tokens)},
              {d_k, d_v}, {k_row, v_row}, {k_head, v_head}, d_slots, d_runs, d_counts, n_rows};
  void (*fn)(StoreArgs) = nullptr;
  const bool e5 = cache->dtype == UZIP_E5M2;
  switch (dtype) {
    case UZIP_BF16: fn = e5 ? store_kernel<UZIP_BF16, UZIP_E5M2> : store_kernel<UZIP_BF16, UZIP_E4M3FN>; break;
    case UZIP_FP16: fn = e5 ? store_kernel<UZIP_FP16, UZIP_E5M2> : store_kernel<UZIP_FP16, UZIP_E4M3FN>; break;
    default: fn = e5 ? store_kernel<UZIP_FP32, UZIP_E5M2> : store_kernel<UZIP_FP32, UZIP_E4M3FN>; break;
  }
  fn<<<dim3(max_runs, cache->n_heads, 2), kStoreThreads, 0, stream>>>(a);
  return hipGetLastError() == hipSuccess ? UZIP_OK : UZIP_EHIP;
}

}  // extern "C"
