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
// Every workgroup takes the prefix sums over all requests for itself and then writes
// its own 256 rows, so one launch does it all and no workgroup waits for another.
// The work is the latency of a few dependent loads and scans: the sums of rows,
// pages and runs are taken in one pass, 256 requests at a time, as if no request ran
// out of rows or pages; only if one does are the three taken one after the other.
// 8 requests 3.2 us, 1024 with 65536 tokens 7.9 (three scans, 1024 rows a workgroup:
// 4.4 and 12.3).
constexpr int kPlanThreads = 256;

struct PlanArgs {
  const int32_t *old_lens, *new_lens, *free_pages;
  int32_t *table, *lens, *q_start, *runs, *counts;
  int64_t *slots;
  int *status;
  uint32_t n_reqs, n_free, shift, n_rows, max_pages;
};

// Sums that stop at a limit: a + b there is min(a + b, limit), which is associative
// and keeps sums of any lengths within 32 bits.
struct Sums {
  uint32_t rows, pages, runs;
};
__device__ __forceinline__ Sums add(const Sums &a, const Sums &b, const Sums &limit) {
  return {min(a.rows + b.rows, limit.rows), min(a.pages + b.pages, limit.pages), min(a.runs + b.runs, limit.runs)};
}

// Sums over the threads before this one, and over all (*total).
__device__ Sums block_scan(const Sums &v, const Sums &limit, Sums *part, Sums *total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  Sums x = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const Sums y = {__shfl_up(x.rows, o), __shfl_up(x.pages, o), __shfl_up(x.runs, o)};
    if (lane >= o) x = add(x, y, limit);
  }
  Sums before = {__shfl_up(x.rows, 1), __shfl_up(x.pages, 1), __shfl_up(x.runs, 1)};
  if (lane == 0) before = {0, 0, 0};
  __syncthreads();
  if (lane == 63) part[wave] = x;
  __syncthreads();
  Sums lower = {0, 0, 0}, all = {0, 0, 0};
#pragma unroll
  for (int w = 0; w < kPlanThreads / 64; ++w) {
    if (w < wave) lower = add(lower, part[w], limit);
    all = add(all, part[w], limit);
  }
  *total = all;
  return add(lower, before, limit);
}

__global__ __launch_bounds__(kPlanThreads) void plan_kernel(PlanArgs a) {
  extern __shared__ int32_t lds[];
  __shared__ Sums part[kPlanThreads / 64];
  __shared__ int trouble, worst;
  const uint32_t tid = threadIdx.x, n = a.n_reqs, P = 1u << a.shift;
  int32_t *first_row = lds, *first_page = lds + n + 1, *first_run = first_page + n;  // first_page -1: takes no part
  const Sums limit = {a.n_rows + 1, a.n_free + 1, a.n_rows + 1};
  auto pages = [&](int64_t tokens) { return (tokens + P - 1) >> a.shift; };
  // What request i needs; rows 0, -1 pages where its lengths or its table refuse it.
  struct Need {
    uint32_t rows;
    int64_t pages;
    uint32_t runs;
    int error;
  };
  auto need_of = [&](uint32_t i) {
    Need r{0, -1, 0, 0};
    if (i >= n) return r;
    const int64_t o = a.old_lens[i], w = a.new_lens[i];
    r.rows = (uint32_t)min(max(w, (int64_t)0), (int64_t)limit.rows);
    if (o < 0 || w < 0 || o + w > INT32_MAX) r.error = UZIP_EINVAL;
    else if (pages(o + w) > a.max_pages) r.error = UZIP_ENOSPC;
    else {
      r.pages = pages(o + w) - pages(o);
      r.runs = w > 0 ? (uint32_t)min(((o + w - 1) >> a.shift) - (o >> a.shift) + 1, (int64_t)limit.runs) : 0;
    }
    return r;
  };
  auto clamp_pages = [&](int64_t x) { return (uint32_t)min(max(x, (int64_t)0), (int64_t)limit.pages); };

  if (tid == 0) trouble = worst = 0;
  __syncthreads();
  Sums done = {0, 0, 0};
  int error = 0;
  bool short_of = false;
  Need next = need_of(tid);
  for (uint32_t base = 0; base < n; base += kPlanThreads) {
    const uint32_t i = base + tid;
    const Need r = next;
    next = need_of(i + kPlanThreads);
    Sums total;
    const Sums v = {r.rows, clamp_pages(r.pages), r.runs};
    const Sums at = add(done, block_scan(v, limit, part, &total), limit);
    done = add(done, total, limit);
    if (i < n) {
      first_row[i] = (int32_t)min(at.rows, a.n_rows);
      first_page[i] = r.error ? -1 : (int32_t)at.pages;
      first_run[i] = (int32_t)at.runs;
      error = min(error, r.error);
      short_of = short_of || at.rows + r.rows > a.n_rows || (r.pages > 0 && at.pages + v.pages > a.n_free);
    }
  }
  if (short_of) trouble = 1;
  __syncthreads();
  if (trouble) {  // a request runs out: rows first, then the pages of those whose rows fit, then the runs of those that have both
    uint32_t rows_done = 0;
    done = {0, 0, 0};
    for (uint32_t base = 0; base < n; base += kPlanThreads) {
      const uint32_t i = base + tid;
      const Need r = need_of(i);
      Sums total;
      const Sums at = block_scan({r.rows, 0, 0}, limit, part, &total);
      const uint32_t row = min(rows_done + at.rows, limit.rows);
      rows_done = min(rows_done + total.rows, limit.rows);
      const bool fits = row + r.rows <= a.n_rows;
      if (i < n && !fits) error = min(error, (int)UZIP_EINVAL);
      bool ok = fits && !r.error;
      const uint32_t take = ok ? clamp_pages(r.pages) : 0;
      const uint32_t page = min(done.pages + block_scan({0, take, 0}, limit, part, &total).pages, limit.pages);
      done.pages = min(done.pages + total.pages, limit.pages);
      if (ok && take > 0 && page + take > a.n_free) {
        ok = false;
        error = min(error, (int)UZIP_ENOSPC);
      }
      const uint32_t run = done.runs + block_scan({0, 0, ok ? r.runs : 0}, limit, part, &total).runs;
      done.runs += total.runs;
      if (i < n) {
        first_page[i] = ok ? (int32_t)page : -1;
        first_run[i] = (int32_t)run;
      }
    }
    done.rows = rows_done;
    // the pages given out: those before the first request that was refused for them
    __syncthreads();
    uint32_t given = 0;
    for (uint32_t i = tid; i < n; i += kPlanThreads)
      if (first_page[i] >= 0) {
        const Need r = need_of(i);
        if (r.pages > 0) given = max(given, (uint32_t)first_page[i] + (uint32_t)r.pages);
      }
#pragma unroll
    for (int o = 32; o; o >>= 1) given = max(given, __shfl_xor(given, o));
    __syncthreads();
    if ((tid & 63) == 0) part[tid >> 6].pages = given;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kPlanThreads / 64; ++w) given = max(given, part[w].pages);
    done.pages = given;
  }
  const uint32_t used = min(done.rows, a.n_rows);
  if (tid == 0) first_row[n] = (int32_t)used;
  if (blockIdx.x == 0) {
    if (tid == 0) {
      a.counts[0] = (int32_t)done.pages;
      a.counts[1] = (int32_t)done.runs;
    }
    if (error) atomicMin(&worst, error);
  }
  __syncthreads();
  if (blockIdx.x == 0 && tid == 0 && a.status) *a.status = worst;

  for (uint32_t i = blockIdx.x * kPlanThreads + tid; i <= n; i += gridDim.x * kPlanThreads) {
    a.q_start[i] = first_row[i];
    if (i < n) a.lens[i] = first_page[i] < 0 ? 0 : a.old_lens[i] + a.new_lens[i];
  }
  const uint32_t r = blockIdx.x * kPlanThreads + tid;
  if (r >= a.n_rows) return;
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

// ------------------------------------------------------------------ store
// For a run, a head, and keys or values: the largest finite magnitude, the page's
// exponent, the codes.  A thread takes eight channels of a token (keys) or of four
// tokens that lie in one word of a value page's channel (values: the page is
// transposed in registers); what it first loaded stays in registers until the exponent
// is known.  Bound by the rows' bytes, each read from memory once: 16384 tokens of 8
// heads of 128 in bf16, 101 MB in 20.9 us, 4.8 TB/s (value by value: 117 us).
struct StoreArgs {
  Cache c;
  const void *x[2];
  int64_t row[2], head[2];
  const int64_t *slots;
  const int32_t *runs, *counts;
  uint32_t n_rows;
  bool vec;  // rows start at multiples of 16 bytes
};

constexpr int kHeld = 4;  // pieces of eight values that a thread keeps

template <int T>
struct Eight {
  typedef typename Elem<T>::type Value;
  u32x4 w[sizeof(Value) / 2];
  __device__ __forceinline__ void load(const Value *x, bool vec) {
    if (vec) {
#pragma unroll
      for (int i = 0; i < (int)sizeof(Value) / 2; ++i) w[i] = ((const u32x4 *)x)[i];
    } else {
      Value v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = x[j];
      __builtin_memcpy(w, v, sizeof(w));
    }
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < (int)sizeof(Value) / 2; ++i) w[i] = u32x4{0, 0, 0, 0};
  }
  __device__ __forceinline__ void get(float *x) const {
    Value v[8];
    __builtin_memcpy(v, w, sizeof(w));
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = (float)v[j];
  }
};

// The codes of places 0 .. off - 1 again, where the page's scale grew.
template <int CODE>
__device__ void grow_page(uint8_t *codes, bool values, uint32_t off, uint32_t D, uint32_t P, uint32_t was, uint32_t e,
                          uint32_t tid, uint32_t threads) {
  const float down = pow2(max(127 + (int)was - (int)e, 0));
  for (uint32_t i = tid; i < off * D; i += threads) {
    uint8_t &c = codes[values ? i / off * P + i % off : i];
    c = (uint8_t)recode<CODE>(c, down);
  }
}

template <int T, int CODE, int THREADS, bool VALUES>
__device__ void store_run(const StoreArgs &a, uint32_t run, uint32_t h, uint32_t tid, float *part, uint32_t *odd_part) {
  typedef typename Elem<T>::type Value;
  const uint32_t D = a.c.dim, P = a.c.page, per = D / 8;
  const int32_t row = a.runs[2 * (size_t)run];
  int32_t n = a.runs[2 * (size_t)run + 1];
  if (row < 0 || n <= 0 || (uint32_t)row >= a.n_rows) return;
  const int64_t slot = a.slots[row];
  if (slot < 0 || (uint64_t)slot >= (uint64_t)a.c.n_pages << a.c.page_shift) return;
  const uint32_t page = (uint32_t)(slot >> a.c.page_shift), off = (uint32_t)slot & (P - 1);
  n = min((uint32_t)n, min(P - off, a.n_rows - (uint32_t)row));
  const uint32_t last = off + n;  // places off .. last - 1 of the page
  const int64_t stride = a.row[VALUES];
  // the row of place t of the page
  const Value *x = (const Value *)a.x[VALUES] + ((int64_t)row - off) * stride + (int64_t)h * a.head[VALUES];
  const size_t ph = (size_t)page * a.c.heads + h;
  uint8_t *codes = (VALUES ? a.c.v : a.c.k) + ph * P * D;
  uint8_t *exps = VALUES ? a.c.v_exp : a.c.k_exp;
  const uint32_t was = off ? exps[ph] : 0;

  // A piece: eight channels of one place; a unit: one piece (keys), or the four pieces of a word (values).
  constexpr uint32_t kUnit = VALUES ? 4 : 1;
  const uint32_t first = off / kUnit, count = ((last + kUnit - 1) / kUnit - first) * per;
  auto unit = [&](uint32_t i, uint32_t *t, uint32_t *d) {
    if (VALUES) {  // neighbours in a wave: 16 words of a channel (or what there are), so that stores join up
      const uint32_t words = (last + 3) / 4 - first;
      *t = 4 * (first + i % words);
      *d = 8 * (i / words);
    } else {
      *t = first + i / per;
      *d = 8 * (i % per);
    }
  };
  auto load = [&](uint32_t t, uint32_t d, Eight<T> *e) {
#pragma unroll
    for (uint32_t j = 0; j < kUnit; ++j) {
      if (t + j >= off && t + j < last) e[j].load(x + (int64_t)(t + j) * stride + d, a.vec);
      else e[j].zero();
    }
  };
  constexpr uint32_t kKeep = kHeld / kUnit;
  Eight<T> held[kHeld];
  float amax = 0;
  bool odd = false;
  auto scan = [&](const Eight<T> *e) {
#pragma unroll
    for (uint32_t j = 0; j < kUnit; ++j) {
      float v[8];
      e[j].get(v);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float f = fabsf(v[k]);
        const bool finite = f < INFINITY;
        odd = odd || !finite;
        amax = fmaxf(amax, finite ? f : 0.0f);
      }
    }
  };
#pragma unroll
  for (uint32_t k = 0; k < kKeep; ++k) {
    const uint32_t i = tid + k * THREADS;
    if (i < count) {
      uint32_t t, d;
      unit(i, &t, &d);
      load(t, d, held + k * kUnit);
    }
  }
#pragma unroll
  for (uint32_t k = 0; k < kKeep; ++k)
    if (tid + k * THREADS < count) scan(held + k * kUnit);
  for (uint32_t i = tid + kKeep * THREADS; i < count; i += THREADS) {
    uint32_t t, d;
    Eight<T> e[kUnit];
    unit(i, &t, &d);
    load(t, d, e);
    scan(e);
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) amax = fmaxf(amax, __shfl_xor(amax, o));
  odd = __any(odd);
  if (THREADS > 64) {
    if ((tid & 63) == 0) {
      part[tid >> 6] = amax;
      odd_part[tid >> 6] = odd;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
      amax = fmaxf(amax, part[w]);
      odd = odd || odd_part[w];
    }
  }
  const uint32_t e = max((uint32_t)exponent_for<CODE>(amax), was);
  if (tid == 0 && e != was) exps[ph] = (uint8_t)e;
  const float inv = pow2(254 - (int)e);
  odd = odd || e >= (uint32_t)Code<CODE>::kExpMax;  // there values may lie past the largest code

  auto put = [&](uint32_t t, uint32_t d, const Eight<T> *p) {
    float v[kUnit][8];
#pragma unroll
    for (uint32_t j = 0; j < kUnit; ++j) p[j].get(v[j]);
    if constexpr (VALUES) {
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        float of[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) of[j] = v[j][k];
        uint32_t w = 0;
        if (odd) {
#pragma unroll
          for (int j = 0; j < 4; ++j) w |= encode<CODE>(of[j], inv) << (8 * j);
        } else {
          w = encode4<CODE>(of, inv);
        }
        uint8_t *at = codes + (size_t)(d + k) * P + t;
        if (t >= off && t + 4 <= last) {
          *(uint32_t *)at = w;
        } else {
#pragma unroll
          for (uint32_t j = 0; j < 4; ++j)
            if (t + j >= off && t + j < last) at[j] = (uint8_t)(w >> (8 * j));
        }
      }
    } else {
      u32x2 w = {0, 0};
      if (odd) {
#pragma unroll
        for (int k = 0; k < 8; ++k) w[k / 4] |= encode<CODE>(v[0][k], inv) << (8 * (k % 4));
      } else {
        w = u32x2{encode4<CODE>(v[0], inv), encode4<CODE>(v[0] + 4, inv)};
      }
      *(u32x2 *)(codes + (size_t)t * D + d) = w;
    }
  };
#pragma unroll
  for (uint32_t k = 0; k < kKeep; ++k) {
    const uint32_t i = tid + k * THREADS;
    if (i < count) {
      uint32_t t, d;
      unit(i, &t, &d);
      put(t, d, held + k * kUnit);
    }
  }
  for (uint32_t i = tid + kKeep * THREADS; i < count; i += THREADS) {
    uint32_t t, d;
    Eight<T> p[kUnit];
    unit(i, &t, &d);
    load(t, d, p);
    put(t, d, p);
  }
  if (off && e > was) grow_page<CODE>(codes, VALUES, off, D, P, was, e, tid, THREADS);
}

// A run of one row by a wave: every lane a channel or a few, nothing but the row
// number needed to ask for them.  64 rows of 8 heads: 4.0 us, by workgroups 6.5.
template <int T, int CODE>
__device__ void store_one(const StoreArgs &a, bool values, int32_t row, uint32_t h, uint32_t lane) {
  typedef typename Elem<T>::type Value;
  const uint32_t D = a.c.dim, P = a.c.page;
  const Value *x = (const Value *)a.x[values] + (int64_t)row * a.row[values] + (int64_t)h * a.head[values];
  const int64_t slot = a.slots[row];
  float v[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = lane + 64 * j < D ? (float)x[lane + 64 * j] : 0.0f;
  if (slot < 0 || (uint64_t)slot >= (uint64_t)a.c.n_pages << a.c.page_shift) return;
  const uint32_t page = (uint32_t)(slot >> a.c.page_shift), off = (uint32_t)slot & (P - 1);
  const size_t ph = (size_t)page * a.c.heads + h;
  uint8_t *codes = (values ? a.c.v : a.c.k) + ph * P * D, *exps = values ? a.c.v_exp : a.c.k_exp;
  const uint32_t was = off ? exps[ph] : 0;
  float amax = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float f = fabsf(v[j]);
    amax = fmaxf(amax, f < INFINITY ? f : 0.0f);
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) amax = fmaxf(amax, __shfl_xor(amax, o));
  const uint32_t e = max((uint32_t)exponent_for<CODE>(amax), was);
  if (lane == 0 && e != was) exps[ph] = (uint8_t)e;
  const float inv = pow2(254 - (int)e);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t d = lane + 64 * j;
    if (d < D) codes[values ? d * P + off : off * D + d] = (uint8_t)encode<CODE>(v[j], inv);
  }
  if (off && e > was) grow_page<CODE>(codes, values, off, D, P, was, e, lane, 64);
}

// Runs of many rows: a workgroup for each run, head, and keys or values.
template <int T, int CODE>
__global__ __launch_bounds__(256) void store_kernel(StoreArgs a) {
  __shared__ float part[4];
  __shared__ uint32_t odd_part[4];
  if ((int32_t)blockIdx.x >= a.counts[1]) return;
  if (blockIdx.z == 0) store_run<T, CODE, 256, false>(a, blockIdx.x, blockIdx.y, threadIdx.x, part, odd_part);
  else store_run<T, CODE, 256, true>(a, blockIdx.x, blockIdx.y, threadIdx.x, part, odd_part);
}
// A wave for each run, whatever its length.
template <int T, int CODE>
__global__ __launch_bounds__(256) void store_few_kernel(StoreArgs a) {
  const uint32_t h = blockIdx.y * 4 + (threadIdx.x >> 6);
  const int32_t count = a.counts[1], row = a.runs[2 * (size_t)blockIdx.x], rows = a.runs[2 * (size_t)blockIdx.x + 1];
  if ((int32_t)blockIdx.x >= count || h >= a.c.heads || row < 0 || (uint32_t)row >= a.n_rows) return;
  if (rows == 1) store_one<T, CODE>(a, blockIdx.z != 0, row, h, threadIdx.x & 63);
  else if (blockIdx.z == 0) store_run<T, CODE, 64, false>(a, blockIdx.x, h, threadIdx.x & 63, nullptr, nullptr);
  else store_run<T, CODE, 64, true>(a, blockIdx.x, h, threadIdx.x & 63, nullptr, nullptr);
}

template <int T, int CODE>
void launch_store(const StoreArgs &a, uint32_t max_runs, hipStream_t stream) {
  // The host knows a bound on the runs, not their lengths.  A wave for each where the bound
  // allows a run for every other row: steps of single tokens, but also a few long runs among
  // many requests, which workgroups store faster (63 single rows and one run of 100: 12.5 us,
  // 7.4), and plans made for more rows (8192 rows in pages of 16: 11.6 us, workgroups 20.6).
  if (a.n_rows <= 2 * max_runs) store_few_kernel<T, CODE><<<dim3(max_runs, (a.c.heads + 3) / 4, 2), 256, 0, stream>>>(a);
  else store_kernel<T, CODE><<<dim3(max_runs, a.c.heads, 2), 256, 0, stream>>>(a);
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
      n_free >= INT32_MAX || max_pages > INT32_MAX)
    return UZIP_EINVAL;
  if (n_reqs && (!d_old || !d_new || !d_lens || (max_pages && !d_table))) return UZIP_EINVAL;
  if ((n_free && !d_free) || (n_rows && (!d_slots || !d_runs)) || !d_q_start || !d_counts) return UZIP_EINVAL;
  for (const void *p : {(const void *)d_old, (const void *)d_new, (const void *)d_free, (const void *)d_table,
                        (const void *)d_lens, (const void *)d_q_start, (const void *)d_runs, (const void *)d_counts,
                        (const void *)d_status})
    if (!aligned(p, 4)) return UZIP_EINVAL;
  if (!aligned(d_slots, 8)) return UZIP_EINVAL;
  if (n_reqs && (d_lens == d_old || d_lens == d_new)) return UZIP_EINVAL;
  if (const uzip_status s = device(nullptr); s != UZIP_OK) return s;
  PlanArgs a{d_old, d_new, d_free, d_table, d_lens, d_q_start, d_runs, d_counts, d_slots, (int *)d_status,
             n_reqs, n_free, (uint32_t)__builtin_ctz(page_tokens), n_rows, max_pages};
  const uint32_t grid = std::max(1u, (n_rows + kPlanThreads - 1) / kPlanThreads);
  plan_kernel<<<grid, kPlanThreads, (3 * n_reqs + 1) * sizeof(int32_t), stream>>>(a);
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
              {d_k, d_v}, {k_row, v_row}, {k_head, v_head}, d_slots, d_runs, d_counts, n_rows, false};
  const int64_t size = type_bytes(dtype);
  a.vec = aligned(d_k, 16) && aligned(d_v, 16);
  for (const int64_t s : {k_row, k_head, v_row, v_head}) a.vec = a.vec && s * size % 16 == 0;
  const bool e5 = cache->dtype == UZIP_E5M2;
  switch (dtype) {
    case UZIP_BF16: (e5 ? launch_store<UZIP_BF16, UZIP_E5M2> : launch_store<UZIP_BF16, UZIP_E4M3FN>)(a, max_runs, stream); break;
    case UZIP_FP16: (e5 ? launch_store<UZIP_FP16, UZIP_E5M2> : launch_store<UZIP_FP16, UZIP_E4M3FN>)(a, max_runs, stream); break;
    default: (e5 ? launch_store<UZIP_FP32, UZIP_E5M2> : launch_store<UZIP_FP32, UZIP_E4M3FN>)(a, max_runs, stream); break;
  }
  return hipGetLastError() == hipSuccess ? UZIP_OK : UZIP_EHIP;
}

}  // extern "C"
