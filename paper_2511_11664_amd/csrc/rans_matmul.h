// rans_matmul.h -- C = A B^T of two matrices of 8-bit codes with block scales
//
// Part of the translation unit rans_blocks.hip; not a stand-alone header.
//
//   C[m, n] = sum over blocks b of sA[m, b] * sB[n or its tile, b] * (sum over k in b of A[m, k] * B[n, k])
//
// B's rows go to the matrix instruction's row operand and A's to its column operand: a lane then holds four neighbouring
// columns of one row of C, stores them at once, and needs one scale of A for them.  A K-step is one block, 128 bytes of a row.
//
// Sums.  The 8-bit matrix instructions add 128 products in binary32 with the smaller ones cut off below the largest one's
// leading bits (an error of about 1e-5 of the result for normally distributed data, 6e-5 where magnitudes spread over
// several powers of two, whatever K is).  That is far below half a step of a 16-bit result.  For binary32 results the codes
// are widened to bf16, which holds both formats exactly, and go through the bf16 instruction, which adds them in binary32
// without such a loss (8e-8 at K = 4096) at half the rate.
#pragma once

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

struct MatmulArgs {
  const uint8_t *a, *b;
  const void *sa, *sb;
  void *c;
  uint64_t lda, ldb, ldsa, ldsb, ldc;
  uint32_t m, n, k;
  uint32_t e8m0, b_tile;
  uint32_t out;  // RANS_F32 / F16 / BF16
  int vec_c;     // four neighbouring elements of C may be stored at once
};

// 16 codes of a row from k on, those from K on are zero.  Rows may start anywhere.
__device__ inline u32x4 load_codes16(const uint8_t *row, uint32_t k, uint32_t K) {
  u32x4 w = {0, 0, 0, 0};
  if (k + 16 <= K) {
    __builtin_memcpy(&w, row + k, 16);
  } else {
    for (uint32_t i = 0; i < 16; i++)
      if (k + i < K) w[i >> 2] |= (uint32_t)row[k + i] << (8 * (i & 3));
  }
  return w;
}

// bf16 of eight codes (two registers).
template <int FMT> __device__ inline bf16x8 bf16_of(uint32_t lo, uint32_t hi) {
  bf16x8 r;
#pragma unroll
  for (int h = 0; h < 2; h++) {
    const uint32_t w = h ? hi : lo;
    const bf16x2 a = FMT ? __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w, 1.0f, false) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false);
    const bf16x2 b = FMT ? __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w, 1.0f, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true);
    r[4 * h] = a[0], r[4 * h + 1] = a[1], r[4 * h + 2] = b[0], r[4 * h + 3] = b[1];
  }
  return r;
}

__device__ inline float matmul_scale(const void *s, uint64_t at, uint32_t e8m0) {
  return e8m0 ? load_scale<true>(s, at) : load_scale<false>(s, at);
}

__device__ inline void store_c4(const MatmulArgs &p, uint32_t m, uint32_t n, f32x4 v) {
  const uint64_t at = m * p.ldc + n;
  if (p.vec_c && n + 4 <= p.n) {
    if (p.out == RANS_F32) {
      *(f32x4 *)((float *)p.c + at) = v;
    } else if (p.out == RANS_F16) {
      typedef _Float16 h4 __attribute__((ext_vector_type(4)));
      *(h4 *)((_Float16 *)p.c + at) = (h4){(_Float16)v[0], (_Float16)v[1], (_Float16)v[2], (_Float16)v[3]};
    } else {
      typedef __bf16 b4 __attribute__((ext_vector_type(4)));
      *(b4 *)((__bf16 *)p.c + at) = (b4){(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; i++) {
    if (n + i >= p.n) break;
    if (p.out == RANS_F32) ((float *)p.c)[at + i] = v[i];
    else if (p.out == RANS_F16) ((_Float16 *)p.c)[at + i] = (_Float16)v[i];
    else ((__bf16 *)p.c)[at + i] = (__bf16)v[i];
  }
}

// A 128 x 128 tile of C, four waves of 64 x 64.  Rows of codes lie in LDS as eight chunks of 16 bytes, chunk c of row r at
// place c ^ (r & 7): the 16 rows that a matrix operand takes the same chunk of then lie in different banks.
constexpr uint32_t kMmTile = 128;
template <int FA, int FB, bool EXACT>
__global__ __launch_bounds__(kWG) void k_block_matmul(MatmulArgs p, uint32_t tiles_m) {
  __shared__ __attribute__((aligned(16))) uint8_t s_a[kMmTile * kBlk], s_b[kMmTile * kBlk];
  const uint32_t t = threadIdx.x, lane = t & 63, r16 = lane & 15, g = lane >> 4;
  const uint32_t wm = (t >> 6) & 1, wn = t >> 7;
  const uint32_t m0 = (blockIdx.x % tiles_m) * kMmTile, n0 = (blockIdx.x / tiles_m) * kMmTile;
  const uint32_t nb = (p.k + kBlk - 1) / kBlk;
  f32x4 acc[4][4];
#pragma unroll
  for (int i = 0; i < 4; i++)
#pragma unroll
    for (int j = 0; j < 4; j++) acc[i][j] = (f32x4){0, 0, 0, 0};
  for (uint32_t kb = 0; kb < nb; kb++) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const uint32_t r = i * 32 + (t >> 3), ch = t & 7;
      const uint32_t ma = m0 + r < p.m ? m0 + r : p.m - 1, mb = n0 + r < p.n ? n0 + r : p.n - 1;
      *(u32x4 *)(s_a + r * kBlk + (ch ^ (r & 7)) * 16) = load_codes16(p.a + ma * p.lda, kb * kBlk + ch * 16, p.k);
      *(u32x4 *)(s_b + r * kBlk + (ch ^ (r & 7)) * 16) = load_codes16(p.b + mb * p.ldb, kb * kBlk + ch * 16, p.k);
    }
    __syncthreads();
    auto frag = [&](const uint8_t *s, uint32_t row) {
      const u32x4 lo = *(const u32x4 *)(s + row * kBlk + (g ^ (row & 7)) * 16);
      const u32x4 hi = *(const u32x4 *)(s + row * kBlk + ((g + 4) ^ (row & 7)) * 16);
      return (i32x8){(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
    };
    i32x8 fa[4], fb[4];
    float sa[4];
    f32x4 sb[4];
#pragma unroll
    for (int i = 0; i < 4; i++) {
      fa[i] = frag(s_a, wm * 64 + i * 16 + r16);
      fb[i] = frag(s_b, wn * 64 + i * 16 + r16);
      const uint32_t m = m0 + wm * 64 + i * 16 + r16;
      sa[i] = matmul_scale(p.sa, (m < p.m ? m : p.m - 1) * p.ldsa + kb, p.e8m0);
#pragma unroll
      for (int j = 0; j < 4; j++) {
        uint32_t n = n0 + wn * 64 + i * 16 + g * 4 + j;
        n = n < p.n ? n : p.n - 1;
        sb[i][j] = matmul_scale(p.sb, (p.b_tile ? n / kBlk : n) * p.ldsb + kb, p.e8m0);
      }
    }
#pragma unroll
    for (int i = 0; i < 4; i++)
#pragma unroll
      for (int j = 0; j < 4; j++) {
        f32x4 d = {0, 0, 0, 0};
        if (EXACT) {
#pragma unroll
          for (int q = 0; q < 4; q++)
            d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bf16_of<FB>(fb[i][2 * q], fb[i][2 * q + 1]), bf16_of<FA>(fa[j][2 * q], fa[j][2 * q + 1]), d, 0, 0, 0);
        } else {
          d = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fb[i], fa[j], d, FB, FA, 0, 0, 0, 0);
        }
#pragma unroll
        for (int e = 0; e < 4; e++) acc[i][j][e] = __builtin_fmaf(d[e], sa[j] * sb[i][e], acc[i][j][e]);
      }
  }
#pragma unroll
  for (int i = 0; i < 4; i++)
#pragma unroll
    for (int j = 0; j < 4; j++) {
      const uint32_t m = m0 + wm * 64 + j * 16 + r16, n = n0 + wn * 64 + i * 16 + g * 4;
      if (m < p.m && n < p.n) store_c4(p, m, n, acc[i][j]);
    }
}

}  // namespace
