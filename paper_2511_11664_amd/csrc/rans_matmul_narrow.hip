// rans_matmul_narrow.hip -- the matrix product with 16-bit results, on the 8-bit matrix instructions

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

// Tiles by the least estimate.  B in E5M2, which no path of a training step has, takes the 128 x 128 tiles at every size.  The
// large tiles are not for binary32 scales of both operands' rows, which leave them too few registers (4096 x 4096 x 11231: 574
// us, 128 x 128 tiles 347).
int launch_matmul_narrow(const MatmulArgs &p, int fmt, MatmulParts parts, void *ws, hipStream_t st) {
  const uint32_t units = compute_units() ? compute_units() : 256;
  const double large = mm_cost_large(p, units), medium = mm_cost_medium(p, units), small = mm_cost_small(p, units);
  const bool few = mm_few(p, small), fetch = mm_fetch_fits(p), deep = mm_deep(p, units, 8);
  return by_format(fmt, [&](auto fa, auto fb) {
    return by_scale(p, [&](auto scale) {
      constexpr int FA = decltype(fa)::value, FB = decltype(fb)::value, SCALE = decltype(scale)::value;
      if (few && p.m <= 16) return launch_few<1, 4, 8, FA, FB, SCALE, false>(p, st);
      if (few) return launch_few<2, 8, 4, FA, FB, SCALE, false>(p, st);
      return in_parts(p, parts, ws, st, [&](const MatmulArgs &q) {
        if (!fetch) return parts.n > 1 || small <= medium ? launch_any<MmSmall, FA, FB, SCALE, false>(q, st) : launch_any<MmWide, FA, FB, SCALE, false>(q, st);
        if constexpr (FB == 0) {
          if (parts.n > 1 || (small <= medium && (small <= large || SCALE == MM_F32_ROW))) return launch_tiles<MmSmall, FA, FB, SCALE, false>(q, st);
          if constexpr (SCALE != MM_F32_ROW)
            if (large < medium) return launch_tiles<MmLarge, FA, FB, SCALE, false>(q, st);
        }
        return deep ? launch_tiles<MmDeep, FA, FB, SCALE, false>(q, st) : launch_tiles<MmMedium, FA, FB, SCALE, false>(q, st);
      });
    });
  });
}

MatmulParts matmul_parts(uint64_t m, uint64_t n, uint64_t k, uint32_t units) {
  const uint64_t tiles = (m + MmSmall::bm - 1) / MmSmall::bm * ((n + MmSmall::bn - 1) / MmSmall::bn), nb = (k + kBlk - 1) / kBlk;
  if (!tiles || 2 * tiles > units || nb < 32) return MatmulParts{1, 0};
  MatmulArgs p = {};
  p.m = (uint32_t)m, p.n = (uint32_t)n, p.k = (uint32_t)k;
  if (mm_few(p, mm_cost_small(p, units))) return MatmulParts{1, 0};
  uint64_t parts = units / tiles < nb / 8 ? units / tiles : nb / 8;
  const uint64_t blocks = ((nb + parts - 1) / parts + MmSmall::stages - 1) / MmSmall::stages * MmSmall::stages;  // whole rounds of the ring
  parts = (nb + blocks - 1) / blocks;
  return parts < 2 ? MatmulParts{1, 0} : MatmulParts{(uint32_t)parts, (uint32_t)blocks};
}
