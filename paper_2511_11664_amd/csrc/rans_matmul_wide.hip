// rans_matmul_wide.hip -- the matrix product with binary32 results, on the bf16 matrix instructions

#include <hip/hip_runtime.h>
#include <hip/hip_fp16.h>

#include <type_traits>

#include "rans_if.h"

#include "rans_host.h"
#include "rans_common.h"
#include "rans_blocks.h"
#include "rans_matmul_launch.h"
#include "rans_matmul.h"
#include "rans_matmul_pick.h"

int launch_matmul_wide(const MatmulArgs &p, int fmt, MatmulParts parts, void *ws, hipStream_t st) {
  const uint32_t units = compute_units() ? compute_units() : 256;
  const double medium = mm_cost_medium(p, units), small = mm_cost_small(p, units);
  const bool few = mm_few(p, small), fetch = mm_fetch_fits(p), deep = mm_deep(p, units, 1);
  return by_format(fmt, [&](auto fa, auto fb) {
    return by_scale(p, [&](auto scale) {
      constexpr int FA = decltype(fa)::value, FB = decltype(fb)::value, SCALE = decltype(scale)::value;
      if (few && p.m <= 16) return launch_few<1, 4, 8, FA, FB, SCALE, true>(p, st);
      if (few) return launch_few<2, 8, 4, FA, FB, SCALE, true>(p, st);
      return in_parts(p, parts, ws, st, [&](const MatmulArgs &q) {
        if (parts.n > 1 || small <= medium) return fetch ? launch_tiles<MmSmall, FA, FB, SCALE, true>(q, st) : launch_any<MmSmall, FA, FB, SCALE, true>(q, st);
        if (!fetch) return launch_any<std::conditional_t<SCALE == MM_F32_TILE, MmWide, MmBroad>, FA, FB, SCALE, true>(q, st);
        return deep ? launch_tiles<MmDeep, FA, FB, SCALE, true>(q, st) : launch_tiles<MmWide, FA, FB, SCALE, true>(q, st);
      });
    });
  });
}
