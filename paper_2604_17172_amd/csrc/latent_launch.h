// latent_launch.h -- the launches of one width of latents; each latent_<width>.hip includes it
// with LATENT_DIM, so that the widths compile side by side.
#include <algorithm>

#include "kv_host.h"
#include "latent.h"
#include "latent_host.h"

namespace uzip_kv {

template <int T, int CODE, int RG>
static uzip_status launch(LatentCall &c) {
  typedef Latent<T, CODE, LATENT_DIM, RG> L;
  LatentArgs &a = c.a;
  const auto kernel = latent_kernel<T, CODE, LATENT_DIM, RG>;
  a.by_heads = FastDiv::of(a.heads);
  a.growth = (double)L::kRows / ((double)kTile * a.heads);
  // What a block's beginning and end cost a workgroup, in tiles.  Counted as 1, workgroups with the end of one block and the
  // beginning of the next were 30 % later than others.  A call, us with 1, 4, 6, 9 of 64 requests of 1000 to 8190 tokens: of 512 in bf16, 16
  // heads 53, 50, 48, 49, 128 heads 108, 101, 98, 98; in fp16 56, 53, 52, 53 and 125, 116, 113, 114; of 256 in bf16 41, 38, 38, 38 and 77,
  // 72, 71, 72, in fp16 43, 40, 41, 42 and 86, 79, 80, 81.  16 requests of 500 to 4000, 32 heads, few tiles to a workgroup: of 512
  // 29, 29, 32, 39, of 256 23, 22, 25, 30.  Two pieces behind 5000 and 8000, 12 heads: of 512 93, 91, 90, 91, of 256 68, 66, 66, 67.
  a.begin = LATENT_DIM == 512 ? 6 : 4;
  // At most how much work there is: blocks, and the tiles of each.
  const uint64_t rows = (uint64_t)a.n_rows * a.heads;
  const uint64_t blocks = std::min<uint64_t>(rows / L::kRows + a.n_reqs + 1, (uint64_t)a.n_rows * ((a.heads + L::kRows - 1) / L::kRows));
  const uint64_t tiles = (((uint64_t)a.max_pages << a.page_shift) + kTile - 1) / kTile;
  a.groups = (uint32_t)std::min<uint64_t>(c.units, std::max<uint64_t>(1, (blocks * (tiles + a.begin) + 2 * a.begin - 1) / (2 * a.begin)));
  if (hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(typename L::Lds)) != hipSuccess) return UZIP_EHIP;
  kernel<<<a.groups, L::kThreads, sizeof(typename L::Lds), c.stream>>>(a);
  if (a.groups > 1)
    latent_join_kernel<T, LATENT_DIM, RG><<<dim3(a.groups - 1, RG * 2 * L::kBlocks), 256, 0, c.stream>>>(a);
  return hipGetLastError() == hipSuccess ? UZIP_OK : UZIP_EHIP;
}

template <int T, int CODE>
static uzip_status launch(LatentCall &c) {
  return c.rows == 32 ? launch<T, CODE, 1>(c) : launch<T, CODE, 2>(c);
}

template <>
uzip_status launch_latent<LATENT_DIM>(LatentCall &c) {
  const bool e5 = c.code == UZIP_E5M2;
  if (c.type == UZIP_BF16) return e5 ? launch<UZIP_BF16, UZIP_E5M2>(c) : launch<UZIP_BF16, UZIP_E4M3FN>(c);
  return e5 ? launch<UZIP_FP16, UZIP_E5M2>(c) : launch<UZIP_FP16, UZIP_E4M3FN>(c);
}

}  // namespace uzip_kv
