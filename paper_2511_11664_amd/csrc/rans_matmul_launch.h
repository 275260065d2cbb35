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
  uint32_t e8m0, b_tile;
  uint32_t out;  // RANS_F32 / F16 / BF16
};

// fmt: 2 where A's codes are E5M2, and 1 where B's are.  Results of 16 bits / binary32 results.
__attribute__((visibility("hidden"))) int launch_matmul_narrow(const MatmulArgs &p, int fmt, hipStream_t st);
__attribute__((visibility("hidden"))) int launch_matmul_wide(const MatmulArgs &p, int fmt, hipStream_t st);
