// rans_matmul_launch.h -- the matrix product's arguments, and its launches from the units that hold its kernels
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

struct MatmulArgs {
  const uint8_t *a, *b;
  const void *sa, *sb;
  void *c;
  uint64_t lda, ldb, ldsa, ldsb, ldc;
  uint32_t m, n, k;
  uint32_t part_blocks;  // K in parts of so many blocks, a work-group row each, whose sums go to c one m x ldc matrix behind the other
  uint32_t e8m0, b_tile;
  uint32_t out;  // RANS_F32 / F16 / BF16
};

// How a product of few tiles and a long K is cut along K: `n` parts (1: not at all) of `blocks` blocks, whose sums take another
// launch.  As many parts as fill the compute units once, of eight blocks at least, where K has 32 blocks or more.  Whole / in
// parts, us: K = 4096, 256 x 256 11.5 / 9.5 (binary32 17.9 / 10.9); K = 16384, 64 x 64 36.5 / 8.5, 704 x 704 39.3 / 26.0;
// K = 2048, 256 x 256 7.2 / 8.4.
// m, n: rows of A and of B in one launch; units: compute units.
struct MatmulParts {
  uint32_t n, blocks;
};
__attribute__((visibility("hidden"))) MatmulParts matmul_parts(uint64_t m, uint64_t n, uint64_t k, uint32_t units);
inline uint64_t matmul_part_ld(uint64_t n) { return (n + 3) & ~3ull; }
inline uint64_t matmul_part_bytes(MatmulParts parts, uint64_t m, uint64_t n) { return parts.n < 2 ? 0 : parts.n * m * matmul_part_ld(n) * 4; }

// p.c, p.ldc: the result's; ws: matmul_part_bytes() of p's rows.  fmt: 2 where A's codes are E5M2, and 1 where B's are.  Results of 16 bits / binary32 results.
__attribute__((visibility("hidden"))) int launch_matmul_narrow(const MatmulArgs &p, int fmt, MatmulParts parts, void *ws, hipStream_t st);
__attribute__((visibility("hidden"))) int launch_matmul_wide(const MatmulArgs &p, int fmt, MatmulParts parts, void *ws, hipStream_t st);
