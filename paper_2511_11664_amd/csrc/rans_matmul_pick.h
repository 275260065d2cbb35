// rans_matmul_pick.h -- which kernel a matrix product takes
//
// Part of the translation units rans_matmul_narrow.hip and rans_matmul_wide.hip; not a stand-alone header.
#pragma once

namespace {

typedef MmTile<2, 4, 8, 4, 2> MmLarge;   // 256 x 256, eight waves
typedef MmTile<2, 4, 4, 2, 2> MmMedium;  // 128 x 128, eight waves
typedef MmTile<2, 4, 4, 2, 4> MmDeep;    // the same with four stages, which leave room for one work-group on a compute unit
typedef MmTile<2, 2, 4, 4, 2> MmWide;    // 128 x 128, four waves: widened operands, and operands of any alignment
typedef MmTile<4, 2, 4, 4, 2> MmBroad;   // 128 rows of A x 256, eight waves: both, scales of each row of B (4096 x 4096 x 4096 224 -> 173 us)
typedef MmTile<2, 2, 2, 2, 4> MmSmall;   // 64 x 64, four waves, four stages

template <typename TILE> uint64_t mm_tiles(const MatmulArgs &p) { return ((p.m + TILE::bm - 1) / TILE::bm) * (uint64_t)((p.n + TILE::bn - 1) / TILE::bn); }

inline uint32_t mm_parts_of(const MatmulArgs &p) { return p.part_blocks ? ((p.k + kBlk - 1) / kBlk + p.part_blocks - 1) / p.part_blocks : 1; }

template <typename TILE, int FA, int FB, int SCALE, bool EXACT> int launch_tiles(const MatmulArgs &p, hipStream_t st) {
  const uint32_t tiles_m = (p.m + TILE::bm - 1) / TILE::bm, tiles_n = (p.n + TILE::bn - 1) / TILE::bn;
  constexpr int kid = std::is_same<TILE, MmSmall>::value ? KID_BLOCK_MATMUL : std::is_same<TILE, MmLarge>::value ? KID_BLOCK_MATMUL_256
                      : std::is_same<TILE, MmDeep>::value ? KID_BLOCK_MATMUL_DEEP : KID_BLOCK_MATMUL_128;
  PROF_LAUNCH(kid, (k_block_matmul<TILE, FA, FB, SCALE, EXACT>), dim3(tiles_m * tiles_n, mm_parts_of(p)), dim3(TILE::threads), 0, st, p, tiles_m,
              tiles_n);
  LAUNCH_CHECK();
  return RANS_OK;
}
template <typename TILE, int FA, int FB, int SCALE, bool EXACT> int launch_any(const MatmulArgs &p, hipStream_t st) {
  const uint32_t tiles_m = (p.m + TILE::bm - 1) / TILE::bm, tiles_n = (p.n + TILE::bn - 1) / TILE::bn;
  constexpr int kid = std::is_same<TILE, MmSmall>::value ? KID_BLOCK_MATMUL_ANY : KID_BLOCK_MATMUL_ANY_128;
  PROF_LAUNCH(kid, (k_block_matmul_any<TILE, FA, FB, SCALE, EXACT>), dim3(tiles_m * tiles_n, mm_parts_of(p)), dim3(TILE::threads), 0, st, p, tiles_m,
              tiles_n);
  LAUNCH_CHECK();
  return RANS_OK;
}
template <int MT, int W, int AHEAD, int FA, int FB, int SCALE, bool EXACT> int launch_few(const MatmulArgs &p, hipStream_t st) {
  PROF_LAUNCH(KID_BLOCK_MATMUL_FEW, (k_block_matmul_few<FA, FB, SCALE, EXACT, MT, W, AHEAD>), dim3((p.n + 15) / 16), dim3(W * 64), 0, st, p);
  LAUNCH_CHECK();
  return RANS_OK;
}

// Rounds of work-groups times what a round takes, us a block: `alone` with one work-group on a compute unit, `both` with two
// (K = 4096, 256 units; 48 to 1024 rows of A, 1024 to 12288 of B).  Widened operands and operands of any alignment take
// longer, but change between 64 x 64 and 128 x 128 tiles at the same sizes.  K = 4096, 64 x 64 / larger, us: 395 x 4096
// widened 27 / 43, any alignment 31 / 40, both 39 / 84; 2048 x 4096 103 / 76, 88 / 57, 116 / 88.
// 128 x 128 / 256 x 256 tiles beyond those rows, us, binary32 scales (powers of two): K = 4096, 1024 x 12288 61 / 61 (59 / 56), 2048 x
// 12288 115 / 122 (107 / 109), which the estimate has the other way round, 4096 x 4096 80 / 69 (74 / 61), 16384 x 12288 960 / 816
// (901 / 740); K = 12288, 2048 x 4096 116 / 171 (107 / 151), 4096 x 4096 225 / 186 (208 / 163), 16384 x 4096 937 / 827 (887 / 728).
inline double mm_cost(uint64_t tiles, uint32_t units, double alone, double both) {
  const uint64_t slots = both > 0 ? 2ull * units : units, whole = tiles / slots, rest = tiles % slots;
  const double full = both > 0 ? both : alone;
  return whole * full + (rest == 0 ? 0 : rest <= units ? alone : full);
}
inline double mm_cost_large(const MatmulArgs &p, uint32_t units) { return mm_cost(mm_tiles<MmLarge>(p), units, 1.6, 0); }
inline double mm_cost_medium(const MatmulArgs &p, uint32_t units) { return mm_cost(mm_tiles<MmMedium>(p), units, 0.64, 1.1); }
inline double mm_cost_small(const MatmulArgs &p, uint32_t units) { return mm_cost(mm_tiles<MmSmall>(p), units, 0.36, 0.5); }

// Four stages where each 128 x 128 tile has a compute unit to itself anyway, and K lasts a few rounds of them.  1024 x 4096,
// us, with two / four stages: K = 512 6.9 / 7.5, 4096 28.9 / 26.0 (powers of two 28.4 / 23.7), 12288 77.5 / 73.6 (82.5 / 71.7);
// widened, over four waves with two stages, 12.2 / 11.9, 51.2 / 49.1, 136 / 131, and 700 x 4096 x 4096 47.7 / 44.5.
inline bool mm_deep(const MatmulArgs &p, uint32_t units, uint32_t least_blocks) {
  return mm_tiles<MmDeep>(p) <= units && p.k >= least_blocks * kBlk;
}

// Few rows of A: the kernel for them takes about 2.6 us and what B, and A once for every 16 rows of B, take at 7.9 MB a us;
// `tiles` is what the tile kernel would take for a block.  1 / 16 / 32 rows, K = 4096, us, few rows over 64 x 64 tiles:
// 4096 rows of B 4.3 / 7.2 / 9.8 over 12, 12288 rows of B 9.6 / 15.3 / 24.7 over 13.
inline bool mm_few(const MatmulArgs &p, double tiles) {
  if (p.m > 32) return false;
  const double bytes = (double)p.n * p.k * (1 + p.m / 16.0), nb = (p.k + kBlk - 1) / kBlk;
  return 2.6 + bytes / 7.9e6 < 1 + tiles * nb;
}
inline bool mm_fetch_fits(const MatmulArgs &p) {
  return aligned_to(p.a, 16) && aligned_to(p.b, 16) && p.lda % 16 == 0 && p.ldb % 16 == 0 && p.lda <= kMmMaxLd && p.ldb <= kMmMaxLd;
}

// The product with its K in parts: `go` launches the tiles, whose sums then become the result.
template <typename F> int in_parts(const MatmulArgs &p, MatmulParts parts, void *ws, hipStream_t st, F go) {
  if (parts.n < 2) return go(p);
  MatmulArgs q = p;
  q.c = ws, q.ldc = matmul_part_ld(p.n), q.out = RANS_F32, q.part_blocks = parts.blocks;
  const int rc = go(q);
  if (rc) return rc;
  PROF_LAUNCH(KID_BLOCK_MATMUL_SUM, k_block_matmul_sum, dim3((p.n + 4 * kWG - 1) / (4 * kWG), p.m), dim3(kWG), 0, st, p, (const float *)ws, parts.n, q.ldc);
  LAUNCH_CHECK();
  return RANS_OK;
}

template <typename F> int by_format(int fmt, F f) {
  typedef std::integral_constant<int, 0> E4;
  typedef std::integral_constant<int, 1> E5;
  return fmt & 2 ? (fmt & 1 ? f(E5{}, E5{}) : f(E5{}, E4{})) : (fmt & 1 ? f(E4{}, E5{}) : f(E4{}, E4{}));
}
template <typename F> int by_scale(const MatmulArgs &p, F f) {
  if (p.e8m0) return f(std::integral_constant<int, MM_E8M0>{});
  if (p.b_tile) return f(std::integral_constant<int, MM_F32_TILE>{});
  return f(std::integral_constant<int, MM_F32_ROW>{});
}

}  // namespace
