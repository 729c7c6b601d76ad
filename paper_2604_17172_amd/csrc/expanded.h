// expanded.h -- attention in the expanded form: keys and values of a head in 16 bits,
// one rotary key a token for all heads, ragged and causal.
//
//   s_t = scale (q . k_t + p . r_t)   out = sum_t e^(s_t) v_t / sum_t e^(s_t)
// in one pass over the tokens with a running maximum.  A wave has a SIMD to itself and takes 64 rows (or 32),
// so that what it reads from LDS serves two products: with 32 rows and two waves a SIMD, LDS was the bound.
// In a round the weights of one tile of 32 tokens are worked out beside the scores of the next.  16 heads of 4096
// tokens, causal, 128 + 64 and 128 channels in bf16: 114 us, 750 TFLOP/s of 86 GFLOP.  A round takes 2500 cycles, of which
// the matrix unit works 1280: a wave issues 345 instructions and 32 exponentials in it.  A workgroup's
// begin and end take 12 us, of which there are two on each compute unit.
#pragma once

#include <utility>

#include "latent.h"

namespace uzip_kv {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

struct ExpandedArgs {
  const void *q, *k, *rot, *v;
  void *out;
  float *lse;
  int64_t q_row, q_head, k_row, k_head, rot_row, v_row, v_head, out_row, out_head;
  const int32_t *q_start, *k_start;
  uint32_t n_rows, n_keys, heads, n_reqs;
  float scale_log2;
  bool flip, flat;    // the scale was below zero, or zero: scale_log2 is its magnitude, or 1
  bool q_vec, out_vec;
};

// Chunks of 16 bytes; chunk c of token t lies at c ^ spread<chunks in a row>(t).  Neither a read of one chunk
// of 16 tokens nor a transposing read of four tokens by four chunks meets a bank twice.
template <int CHUNKS>
__device__ __forceinline__ uint32_t spread(uint32_t t) {
  if constexpr (CHUNKS == 16) return ((t & 3) << 2) | ((t >> 2) & 3);
  else if constexpr (CHUNKS == 8) return ((t & 2) << 1) | ((t >> 2) & 3);
  else return (t >> 2) & 3;
}

struct ExpandedBlock {
  int32_t first, rows;  // the block's rows
  int32_t base;         // place of the first
  int32_t key0, keys;   // the request's keys
};

// Block `index` of the requests' blocks of ROWS rows, last blocks of a request first; found by each wave.  A lane
// looks at a request (or at several in a row), the rows behind the last being one more.
template <int ROWS>
__device__ __forceinline__ bool find_expanded(const ExpandedArgs &a, uint32_t index, ExpandedBlock *out) {
  const uint32_t lane = threadIdx.x & 63, n = a.n_reqs + 1, each = (n + 63) / 64, lo = min(n, lane * each), hi = min(n, lo + each);
  struct Request {
    int32_t first, rows, key0, keys;
  };
  auto request = [&](uint32_t i) {
    const int64_t all = a.n_rows, most = a.n_keys;
    const bool one = i < a.n_reqs;
    const int64_t from = min(max((int64_t)(a.n_reqs ? a.q_start[i] : 0), (int64_t)0), all);
    const int64_t to = one ? min(max((int64_t)a.q_start[i + 1], from), all) : all;
    const int64_t k0 = one ? min(max((int64_t)a.k_start[i], (int64_t)0), most) : 0;
    const int64_t k1 = one ? min(max((int64_t)a.k_start[i + 1], k0), most) : 0;
    return Request{(int32_t)from, (int32_t)(to - from), (int32_t)k0, (int32_t)(k1 - k0)};
  };
  auto blocks_of = [](const Request &r) { return ((uint32_t)r.rows + ROWS - 1) / ROWS; };
  Request r{};
  uint32_t mine = 0;
  for (uint32_t i = lo; i < hi; ++i) {
    r = request(i);
    mine += blocks_of(r);
  }
  uint32_t upto = mine;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t y = __shfl_up(upto, o);
    if ((int)lane >= o) upto += y;
  }
  const bool here = index < upto && index >= upto - mine;
  const uint64_t who = __ballot(here);
  if (!who) return false;
  uint32_t at = upto - mine;
  if (here && each > 1)
    for (uint32_t i = lo; i < hi; ++i) {
      r = request(i);
      if (index - at < blocks_of(r)) break;
      at += blocks_of(r);
    }
  const int32_t block = (int32_t)(blocks_of(r) - 1 - (index - at)) * ROWS;
  const ExpandedBlock b{r.first + block, min((int32_t)ROWS, r.rows - block), r.keys - r.rows + block, r.key0, r.keys};
  const int from = __ffsll((unsigned long long)who) - 1;
  uint32_t words[sizeof(ExpandedBlock) / 4];
  __builtin_memcpy(words, &b, sizeof(b));
#pragma unroll
  for (uint32_t i = 0; i < sizeof(b) / 4; ++i) words[i] = __builtin_amdgcn_readlane(words[i], from);
  __builtin_memcpy(out, words, sizeof(b));
  return true;
}

// Four or eight waves of R times 32 rows: RG side by side share their tiles of 32 tokens, and SPLIT such groups take
// the tiles in turn; their sums are joined at the end.
template <int DN, int DR, int DV, int R, int RG, int SPLIT>
struct Expanded {
  static constexpr int kWaves = RG * SPLIT, kRows = 32 * R * RG, kThreads = 64 * kWaves, kTokens = 32, kMemory = 160 * 1024;
  struct Tile {
    uint8_t k[kTokens * DN * 2], rot[kTokens * DR * 2], v[kTokens * DV * 2];
  };
  // rounds that a tile is asked for ahead, and places for tiles
  static constexpr int kAsk = 3 * SPLIT * sizeof(Tile) <= kMemory ? 2 : 1, kPlaces = kAsk + 1;
  struct Notes {
    int32_t first_of[3][DV];  // the first token whose value is NaN, infinite, minus infinite
    uint32_t trouble, unused[3];
  };
  struct Join {
    float m[SPLIT][kRows], l[SPLIT][kRows];
    f32x4 part[R][DV / 32][SPLIT - 1][RG][4][64];
  };
  union Lds {
    Tile tile[kPlaces][SPLIT];
    Join join;
  };
  static_assert((kWaves == 4 || kWaves == 8) && sizeof(Lds) <= kMemory && sizeof(Join) + sizeof(Notes) <= sizeof(Lds), "the tiles' memory holds the rest");
};

template <int T, int DN, int DR, int DV, int R, int RG, int SPLIT, bool DIRECT>
__global__ __launch_bounds__(64 * RG * SPLIT, RG * SPLIT / 4) void expanded_kernel(ExpandedArgs a) {
  typedef Expanded<DN, DR, DV, R, RG, SPLIT> L;
  typedef typename Elem<T>::type Value;
  typedef typename LatentType<T>::Eight Eight;
  typedef __attribute__((address_space(3))) Eight LdsEight;
  constexpr int kSteps = (DN + DR) / 16, kBlocks = DV / 32, kTokens = L::kTokens;
  constexpr float kLag = 8;  // weights up to 2^8
  extern __shared__ __align__(16) uint8_t lds_bytes[];
  typename L::Lds &lds = *(typename L::Lds *)lds_bytes;
  const uint32_t lds0 = lds_at(lds_bytes);
  typename L::Notes &notes = *(typename L::Notes *)(lds_bytes + sizeof(lds) - sizeof(typename L::Notes));
  const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 31, h = lane >> 5;
  const uint32_t rg = wave % RG, group = wave / RG;
  const uint32_t head = blockIdx.x % a.heads;
  ExpandedBlock b;
  if (!find_expanded<L::kRows>(a, blockIdx.x / a.heads, &b)) return;

  int32_t at[R], at_min[R];  // places of this lane's rows, and of the first of each 32
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int32_t j = (int32_t)(32 * (R * rg + r));
    at[r] = j + (int32_t)col < b.rows ? b.base + j + (int32_t)col : -1;
    at_min[r] = b.base + min(j, b.rows - 1);
  }
  const int32_t seen = min(max(b.base + b.rows, 0), b.keys);
  const uint32_t tiles = ((uint32_t)seen + kTokens - 1) / kTokens, rounds = (tiles + SPLIT - 1) / SPLIT;
  const uint32_t mine = tiles > group ? (tiles - group + SPLIT - 1) / SPLIT : 0;  // this group's tiles

  Eight query[R][kSteps];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int32_t j = (int32_t)(32 * (R * rg + r) + col);
    const Value *src = (const Value *)a.q + (int64_t)(b.first + (j < b.rows ? j : 0)) * a.q_row + (int64_t)head * a.q_head + 8 * h;
    if (a.q_vec) {
#pragma unroll
      for (int s = 0; s < kSteps; ++s) query[r][s] = *(const Eight *)(src + 16 * s);
    } else {
#pragma unroll
      for (int s = 0; s < kSteps; ++s)
#pragma unroll
        for (int e = 0; e < 8; ++e) query[r][s][e] = src[16 * s + e];
    }
  }

  // What a row has in memory, `row` elements from one token to the next: this group's tiles one after another.
  // Past the last token that one is read again.
  struct From {
    const uint8_t *base;  // of the tile's first token
    int32_t left;         // tokens behind that
    int64_t row;          // in bytes
    __device__ __forceinline__ void next() {
      const bool more = left >= SPLIT * kTokens;
      base += more ? SPLIT * kTokens * row : 0;
      left = more ? left - SPLIT * kTokens : 0;  // no tile that is used comes after this one
    }
  };
  auto from = [&](const void *x, int64_t row, int64_t at_head) {
    const int64_t t0 = min(group * kTokens, (uint32_t)max(b.keys, 1) - 1);
    return From{(const uint8_t *)x + 2 * ((b.key0 + t0) * row + at_head), max(b.keys, 1) - 1 - (int32_t)t0, 2 * row};
  };
  constexpr uint32_t kRot = offsetof(typename L::Tile, rot), kValues = offsetof(typename L::Tile, v);
  // The n-th of this wave's loads of a tile's rows of `width` bytes; a load takes 1024 bytes.
  auto load = [&](auto width, const From &f, uint32_t to, int n) {
    constexpr int kBytes = decltype(width)::value, kChunks = kBytes / 16, kPer = 1024 / kBytes, kLoads = kTokens / kPer;
    static_assert(kLoads % RG == 0, "");
    const uint32_t k = n * RG + rg, t = k * kPer + lane / kChunks, c = (lane % kChunks) ^ spread<kChunks>(t), token = min(t, (uint32_t)f.left);
    if constexpr (DIRECT) {
      load_to_lds(f.base, __umul24(token, (uint32_t)f.row) + c * 16, to + k * 1024);
    } else {  // rows that are not at multiples of 16 bytes, or far apart
      const Value *x = (const Value *)(f.base + token * f.row) + c * 8;
      Eight y;
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = x[e];
      *(LdsEight *)(uintptr_t)(to + k * 1024 + lane * 16) = y;
    }
  };
  constexpr int kKeyLoads = kTokens * DN * 2 / 1024 / RG, kOwnKeys = kKeyLoads + kTokens * DR * 2 / 1024 / RG,  // loads of a wave
                kOwnValues = kTokens * DV * 2 / 1024 / RG;
  From keys{}, turned{}, values{};  // the tiles to be asked for next
  auto ask_key = [&](uint32_t to, int n) {
    if (n < kKeyLoads) load(std::integral_constant<int, DN * 2>{}, keys, to, n);
    else load(std::integral_constant<int, DR * 2>{}, turned, to + kRot, n - kKeyLoads);
  };
  auto ask_value = [&](uint32_t to, int n) { load(std::integral_constant<int, DV * 2>{}, values, to + kValues, n); };
  auto ask_keys = [&](uint32_t to) {
#pragma unroll
    for (int n = 0; n < kOwnKeys; ++n) ask_key(to, n);
    keys.next();
    turned.next();
  };
  auto ask_values = [&](uint32_t to) {
#pragma unroll
    for (int n = 0; n < kOwnValues; ++n) ask_value(to, n);
    values.next();
  };
  auto first_of_tile = [&](uint32_t i) { return (i * SPLIT + group) * kTokens; };

  // where this lane reads
  const uint32_t k_off = col * DN * 2 + ((h ^ spread<DN / 8>(col)) << 4);
  const uint32_t r_off = col * DR * 2 + ((h ^ spread<DR / 8>(col)) << 4);
  const uint32_t v_tok = 4 * h + ((lane & 15) >> 2);
  const uint32_t v_off = v_tok * DV * 2 + (((2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ spread<DV / 8>(v_tok)) << 4) + (lane & 1) * 8;

  f32x16 acc[R][kBlocks], s[2][R];  // scores of this round's tile and of the next
  u32x4 w[R][2];
  float m[R], l[R], most[R], ref[R];
  // Weights are 2^-lift times as large: in fp16 as large as they may be, since what is below 2^-25 becomes nothing.  (Past 2^24 a
  // reference 7 less could come out 8 less or more, and a weight past 2^16.)
  float lift = T == UZIP_FP16 ? kLag - 15 : 0;
  auto lifted = [&](float m) { return T == UZIP_FP16 && fabsf(m) >= 0x1p24f ? m : m + lift; };
  // `count` steps, each with a read from LDS: two are on their way while the two before them are used, and
  // beside(i) is what the vector units do meanwhile.  The order is the one written here: the wave has its SIMD for
  // itself, and only what stands beside a matrix instruction runs beside it.
  auto steps = [&](auto count, const auto &read, const auto &use, const auto &beside) {
    constexpr int kCount = decltype(count)::value, kAhead = 2;
    Eight x[2 * kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) x[i] = read(i);
#pragma unroll
    for (int i = 0; i < kCount; ++i) {
      if (i + kAhead < kCount) x[(i + kAhead) % (2 * kAhead)] = read(i + kAhead);
      use(i, x[i % (2 * kAhead)]);
      beside(i);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // to = the products of a tile's keys
  auto score = [&](uint32_t tile, f32x16 *to, const auto &beside) {
    const uint32_t at_keys = tile + k_off, at_turned = tile + kRot + r_off;
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int e = 0; e < 16; ++e) to[r][e] = 0;
    steps(std::integral_constant<int, kSteps>{},
          [&](int k) {
            if (k < DN / 16) return *(const LdsEight *)(uintptr_t)(at_keys ^ (k << 5));
            return *(const LdsEight *)(uintptr_t)(at_turned ^ ((k - DN / 16) << 5));
          },
          [&](int k, const Eight &x) {
#pragma unroll
            for (int r = 0; r < R; ++r) to[r] = mfma16(x, query[r][k], to[r]);
          },
          beside);
  };
  // the largest score of a tile's rows, what is past a row masked
  auto peak = [&](uint32_t i, f32x16 *x, int r) {
    const int32_t t0 = (int32_t)first_of_tile(i);
    if (a.flat) {  // a scale of zero: what is finite becomes 0
#pragma unroll
      for (int e = 0; e < 16; ++e) x[r][e] *= 0.0f;
    }
    if (t0 + kTokens - 1 > at_min[r]) {
      const int32_t upto = at[r] - t0 - 4 * (int)h;
#pragma unroll
      for (int e = 0; e < 16; ++e) x[r][e] = 8 * (e / 4) + e % 4 <= upto ? x[r][e] : -INFINITY;
    }
    float y = x[r][0];
#pragma unroll
    for (int e = 1; e < 16; ++e) y = fmaxf(y, x[r][e]);
    most[r] = y * a.scale_log2;
  };
  // where it is far above the reference, that is raised and the sums scaled
  auto settle = [&] {
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (__any(most[r] - m[r] > kLag)) {
        const float both = max_of_halves(most[r]);
        const float next = both - m[r] > kLag ? both : m[r], f = next == m[r] ? 1.0f : __builtin_amdgcn_exp2f(m[r] - next);
        m[r] = next;
        ref[r] = next == -INFINITY ? 0.0f : lifted(next);
        l[r] *= f;
#pragma unroll
        for (int n = 0; n < kBlocks; ++n)
#pragma unroll
          for (int e = 0; e < 16; ++e) acc[r][n][e] *= f;
      }
  };
  // two weights of every row: the first 4 R pairs are of the tile's first 16 tokens
  auto weigh = [&](f32x16 *x, int pair) {
    const int half = pair / (4 * R), r = pair / 4 % R, e = 2 * (pair % 4);
    typedef Value Two __attribute__((ext_vector_type(2)));
    Two y;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const float z = __builtin_amdgcn_exp2f(__builtin_fmaf(x[r][8 * half + e + k], a.scale_log2, -ref[r]));
      l[r] += z;
      y[k] = (Value)z;
    }
    uint32_t word = __builtin_bit_cast(uint32_t, y);
    asm volatile("" : "+v"(word), "+v"(l[r]));  // here, and not where they are used
    w[r][half][e / 2] = word;
  };
  // adds a tile's values
  auto add = [&](uint32_t tile, const auto &beside) {
    const uint32_t at_values = tile + kValues + v_off;
    steps(std::integral_constant<int, 2 * kBlocks>{},
          [&](int i) {
            const int k = i / kBlocks, n = i % kBlocks;
            union {
              Eight e;
              s16x4 p[2];
            } v;
#pragma unroll
            for (int p = 0; p < 2; ++p)
              v.p[p] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                  (__attribute__((address_space(3))) s16x4 *)(uintptr_t)((at_values ^ (n << 6) ^ (p << 5)) + (16 * k + 8 * p) * DV * 2));
            return v.e;
          },
          [&](int i, const Eight &x) {
#pragma unroll
            for (int r = 0; r < R; ++r) acc[r][i % kBlocks] = mfma16(x, __builtin_bit_cast(Eight, w[r][i / kBlocks]), acc[r][i % kBlocks]);
          },
          beside);
  };

  uint32_t place[L::kPlaces];  // of the tiles i, i + 1, ..., in turn
  auto ask_first = [&] {
#pragma unroll
    for (int i = 0; i < L::kPlaces; ++i) place[i] = lds0 + (i * SPLIT + group) * (uint32_t)sizeof(typename L::Tile);
    keys = from(a.k, a.k_row, (int64_t)head * a.k_head);
    turned = from(a.rot, a.rot_row, 0);
    values = from(a.v, a.v_row, (int64_t)head * a.v_head);
    if (mine > 0) {
      ask_keys(place[0]);
#pragma unroll
      for (int i = 0; i < L::kAsk; ++i) {
        ask_values(place[i]);
        ask_keys(place[i + 1]);
      }
    }
  };
  ask_first();
  if (a.flip) {  // a scale below zero: its sign is the queries', so that the largest product has the largest score
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int s = 0; s < kSteps; ++s) query[r][s] = __builtin_bit_cast(Eight, __builtin_bit_cast(s16x8, query[r][s]) ^ (short)0x8000);
  }
  if constexpr (L::kWaves == 4)  // half of the registers
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int s = 0; s < kSteps; ++s) asm volatile("" : "+a"(query[r][s]));  // in accumulation registers, which matrix instructions read as well
  bool careful = false;
  for (;;) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
#pragma unroll
      for (int n = 0; n < kBlocks; ++n)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[r][n][e] = 0;
      m[r] = -INFINITY;
      l[r] = ref[r] = 0;
    }
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    if (mine > 0) {
      score(place[0], s[0], [](int) {});
#pragma unroll
      for (int r = 0; r < R; ++r) peak(0, s[0], r);
      settle();
    }
    // Round i: the weights of tile i beside the scores of tile i + 1, then tile i's values beside what is left of
    // its weights and the next tile's largest score; in between, loads of tiles to come.  Past this group's
    // last tile they read its last token again, into places that nobody reads, and what is scored is masked.
    auto round = [&](uint32_t i, auto parity) {
      constexpr int kNow = decltype(parity)::value, kPairs = 8 * R, kFirst = kPairs - 4;  // pairs beside the scores
      constexpr int kOwn = kOwnKeys + kOwnValues;
      if (L::kAsk == 2 && DIRECT) __builtin_amdgcn_s_waitcnt(0x0070 | (kOwn & 15) | (kOwn >> 4) << 14);  // but for the last round's loads
      else __builtin_amdgcn_s_waitcnt(0);
      __syncthreads();  // everybody's part of the next keys and these values has arrived
      if (careful) {  // values that are NaN or infinite are left out
        if (i < mine)
          for (uint32_t c = rg * 64 + lane; c < kTokens * DV / 8; c += 64 * RG) {
            LdsEight *at_values = (LdsEight *)(uintptr_t)(place[0] + kValues + c * 16);
            Eight x = *at_values;
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = (float)x[e] - (float)x[e] == 0 ? x[e] : (Value)0.0f;
            *at_values = x;
          }
        __syncthreads();
      }
      if (i >= mine) return;
      const uint32_t for_keys = place[0], for_values = place[L::kAsk];
      score(place[1], s[1 - kNow], [&](int g) {
#pragma unroll
        for (int p = g * kFirst / kSteps; p < (g + 1) * kFirst / kSteps; ++p) weigh(s[kNow], p);
#pragma unroll
        for (int n = g * kOwnKeys / kSteps; n < (g + 1) * kOwnKeys / kSteps; ++n) ask_key(for_keys, n);
      });
      add(place[0], [&](int g) {
        if (g < kBlocks)
#pragma unroll
          for (int p = kFirst + g * 4 / kBlocks; p < kFirst + (g + 1) * 4 / kBlocks; ++p) weigh(s[kNow], p);
        else if (g < kBlocks + R)
          peak(i + 1, s[1 - kNow], g - kBlocks);
#pragma unroll
        for (int n = g * kOwnValues / (2 * kBlocks); n < (g + 1) * kOwnValues / (2 * kBlocks); ++n) ask_value(for_values, n);
      });
      keys.next();
      turned.next();
      values.next();
      const uint32_t p0 = place[0];
#pragma unroll
      for (int p = 0; p + 1 < L::kPlaces; ++p) place[p] = place[p + 1];
      place[L::kPlaces - 1] = p0;
      settle();
    };
    for (uint32_t i = 0; i < rounds; i += 2) {
      round(i, std::integral_constant<int, 0>{});
      if (i + 1 < rounds) round(i + 1, std::integral_constant<int, 1>{});
    }
    __builtin_amdgcn_s_waitcnt(0);  // the last loads, before the places serve for other things
    __syncthreads();
    if (careful) break;
    // sums that are not finite are computed again with care
    float odd = 0;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      odd = __builtin_fmaf(l[r], 0.0f, odd);
#pragma unroll
      for (int n = 0; n < kBlocks; ++n)
#pragma unroll
        for (int e = 0; e < 16; ++e) odd = __builtin_fmaf(acc[r][n][e], 0.0f, odd);
    }
    if (threadIdx.x == 0) notes.trouble = 0;
    __syncthreads();
    if (__any(odd != 0.0f) && lane == 0) notes.trouble = 1;
    __syncthreads();
    if (!notes.trouble) break;
    __syncthreads();
    careful = true;
    if (T == UZIP_BF16) lift = 32;  // sums of values near the type's largest stay finite
    ask_first();
  }

  if (careful) {  // where they are
    for (uint32_t i = threadIdx.x; i < 3 * DV; i += L::kThreads) (&notes.first_of[0][0])[i] = INT32_MAX;
    __syncthreads();
    const Value *x = (const Value *)a.v + (int64_t)b.key0 * a.v_row + (int64_t)head * a.v_head;
#pragma unroll 1
    for (uint32_t i = threadIdx.x; i < (uint32_t)seen * DV; i += L::kThreads) {
      const float y = (float)x[(int64_t)(i / DV) * a.v_row + i % DV];
      if (y - y != 0) atomicMin(&notes.first_of[y != y ? 0 : y > 0 ? 1 : 2][i % DV], (int32_t)(i / DV));
    }
  }
  // The groups' sums come together: block n of the channels is finished by group n % SPLIT.
  typename L::Join &join = lds.join;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const uint32_t j = 32 * (R * rg + r) + col;
    l[r] = sum_of_halves(l[r]);
    m[r] = lifted(m[r]);
    if (h == 0) {
      join.m[group][j] = m[r];
      join.l[group][j] = l[r];
    }
#pragma unroll
    for (int n = 0; n < kBlocks; ++n)
      if (n % SPLIT != (int)group)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          join.part[r][n][group < n % SPLIT ? group : group - 1][rg][g][lane] = f32x4{acc[r][n][4 * g], acc[r][n][4 * g + 1], acc[r][n][4 * g + 2], acc[r][n][4 * g + 3]};
  }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const uint32_t j = 32 * (R * rg + r) + col;
    float theirs[SPLIT], scale[SPLIT], all = -INFINITY, sum = 0;
#pragma unroll
    for (int g = 0; g < SPLIT; ++g) all = fmaxf(all, theirs[g] = join.m[g][j]);
#pragma unroll
    for (int g = 0; g < SPLIT; ++g) {
      scale[g] = theirs[g] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(theirs[g] - all);
      sum = __builtin_fmaf(join.l[g][j], scale[g], sum);
    }
    if ((int32_t)j >= b.rows) continue;
    // divided before they are added: a group's sums may be finite and all of them together not
    const float inverse = sum > 0 ? 1.0f / sum : sum == 0 ? 0.0f : NAN;
    const float f = m[r] == -INFINITY ? 0.0f * inverse : __builtin_amdgcn_exp2f(m[r] - all) * inverse;
#pragma unroll
    for (int g = 0; g < SPLIT; ++g) scale[g] *= inverse;
    Value *out = (Value *)a.out + (int64_t)(b.first + (int32_t)j) * a.out_row + (int64_t)head * a.out_head;
#pragma unroll
    for (int n = 0; n < kBlocks; ++n) {
      if (n % SPLIT != (int)group) continue;
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const uint32_t d = 32 * n + 8 * g + 4 * h;
        f32x4 x;
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] = acc[r][n][4 * g + k] * f;
#pragma unroll
        for (int o = 0; o < SPLIT; ++o)
          if (o != n % SPLIT) {
            const f32x4 y = join.part[r][n][o < n % SPLIT ? o : o - 1][rg][g][lane];
#pragma unroll
            for (int k = 0; k < 4; ++k) x[k] = __builtin_fmaf(y[k], scale[o], x[k]);
          }
        Value y[4] __attribute__((aligned(8)));
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          float z = x[k];
          if (careful) {
            if (at[r] >= notes.first_of[0][d + k]) z = NAN;
            if (at[r] >= notes.first_of[1][d + k]) z += INFINITY;
            if (at[r] >= notes.first_of[2][d + k]) z -= INFINITY;
          }
          y[k] = (Value)z;
        }
        if (a.out_vec) {
          *(u32x2 *)(out + d) = *(u32x2 *)y;
        } else {
#pragma unroll
          for (int k = 0; k < 4; ++k) out[d + k] = y[k];
        }
      }
    }
    if (h == 0 && group == 0 && a.lse)
      a.lse[(size_t)(b.first + (int32_t)j) * a.heads + head] = sum == 0 ? -INFINITY : (all + __builtin_amdgcn_logf(sum)) * 0.69314718055994530942f;
  }
}

}  // namespace uzip_kv
