// rans_blocks.h -- matrices of 8-bit floating-point codes with a scale for each block of 128: quantise and dequantise
//
// Part of the translation unit rans_blocks.hip; not a stand-alone header.
//
// A block is 128 columns of one row, or a 128 x 128 tile.  With a = the largest finite |x| of a block and v the format's
// largest number (448 for E4M3, 57344 for E5M2):
//   binary32 scales   s = max(a / v, 2^-126), code = rne8(x * (1 / s))
//   powers of two     s = 2^e with the least e >= -126 for which v * 2^e >= a, code = rne8(x * 2^-e)
// and s = 1 where a = 0.  Both v are 1.75 * 2^k, so e follows from a's exponent and one comparison of its mantissa.
// Products are binary32 (those with 2^-e exact), rne8 is the conversion instruction: round to nearest, ties to even,
// subnormals kept.  |x * (1 / s)| <= v * (1 + 2^-22), which rounds to v, so nothing saturates.  NaN stays NaN; an
// infinity becomes NaN in E4M3, which has none, and stays one in E5M2.
//
// Bound by memory: 3 bytes an element for 16-bit input, some five operations.
#pragma once

namespace {

constexpr uint32_t kBlk = 128;              // columns (and rows of a tile) that share a scale
constexpr uint64_t kBlkMaxDim = 1ull << 30; // rows, columns
constexpr uint64_t kBlkMaxLd = 1ull << 32;  // elements from a row to the next

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// ------------------------------------------------------------------ element types: eight neighbours at a time

// Aligned to an element only: the loads and stores stay 16 bytes wide, and cost more where they cross a cache line.
template <typename T> struct Vec8;
template <> struct Vec8<float> { typedef float type __attribute__((ext_vector_type(8), aligned(4))); };
template <> struct Vec8<_Float16> { typedef _Float16 type __attribute__((ext_vector_type(8), aligned(2))); };
template <> struct Vec8<__bf16> { typedef __bf16 type __attribute__((ext_vector_type(8), aligned(2))); };
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(1)));

// Elements c .. c + 7 of a row of n as they lie in memory; those from n on are zero.
// ONCE: read past the caches, for what nobody reads again soon (16384 x 4096 fp16 to codes: 41.6 -> 34.3 us, with two
// blocks instead of four for a lane).
template <bool ONCE = false, typename T> __device__ inline typename Vec8<T>::type load8_raw(const T *row, uint32_t c, uint32_t n) {
  typedef typename Vec8<T>::type V;
  if (c + 8 <= n) {
    if (!ONCE) return *(const V *)(row + c);
    struct Words {
      u32x4 w[sizeof(V) / 16];
    } q;
#pragma unroll
    for (size_t i = 0; i < sizeof(V) / 16; i++) q.w[i] = __builtin_nontemporal_load((const u32x4_any *)(row + c) + i);
    return __builtin_bit_cast(V, q);
  }
  V v;
#pragma unroll
  for (int i = 0; i < 8; i++) v[i] = c + i < n ? row[c + i] : (T)0.0f;
  return v;
}
template <typename V> __device__ inline f32x8 float8_of(V v) {
  f32x8 r;
#pragma unroll
  for (int i = 0; i < 8; i++) r[i] = (float)v[i];
  return r;
}
template <bool ONCE = false, typename T> __device__ inline f32x8 load8(const T *row, uint32_t c, uint32_t n) {
  return float8_of(load8_raw<ONCE>(row, c, n));
}

// The element type's rounding (to nearest even) of eight binary32 values, kept if in the row.
template <typename T> __device__ inline void store8(T *row, uint32_t c, uint32_t n, f32x8 v) {
  if (c + 8 <= n) {
    typename Vec8<T>::type o;
#pragma unroll
    for (int i = 0; i < 8; i++) o[i] = (T)v[i];
    *(typename Vec8<T>::type *)(row + c) = o;
  } else {
#pragma unroll
    for (int i = 0; i < 8; i++)
      if (c + i < n) row[c + i] = (T)v[i];
  }
}

// ------------------------------------------------------------------ scales and codes

// Bits of |x|, 0 where x is no finite number: as unsigned integers they compare like the numbers.
__device__ inline uint32_t abs_bits_finite(float x) {
  const uint32_t b = __float_as_uint(x) & 0x7fffffffu;
  return b < 0x7f800000u ? b : 0u;
}
__device__ inline uint32_t abs_max8(f32x8 v) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; i++) {
    const uint32_t b = abs_bits_finite(v[i]);
    m = b > m ? b : m;
  }
  return m;
}

// Largest of 16 neighbouring lanes, in all of them.
__device__ inline uint32_t max16(uint32_t m) {
#define STEP(ctrl)                                                                                \
  {                                                                                               \
    const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp((int)m, (int)m, ctrl, 0xf, 0xf, true); \
    m = o > m ? o : m;                                                                            \
  }
  STEP(0x128) STEP(0x124) STEP(0x122) STEP(0x121)  // rotations by 8, 4, 2, 1 inside a row of 16
#undef STEP
  return m;
}

// Scale of a block whose largest magnitude has the bits `amax`: what is stored (float or exponent byte), and the factor
// that x is multiplied by.
struct BlockScale {
  float scale, factor;
  uint32_t e8m0;
};
template <bool E8M0> __device__ inline BlockScale block_scale(uint32_t amax, uint32_t e5m2) {
  BlockScale s;
  if (E8M0) {
    // a = m * 2^x, v = 1.75 * 2^k: the least e with 1.75 * 2^(k+e) >= a is x - k, one more for m > 1.75
    int e = (int)(amax >> 23) - (e5m2 ? 15 : 8) + ((amax & 0x7fffffu) > 0x600000u ? 1 : 0);
    e = e < 1 ? 1 : e;
    if (amax == 0) e = 127;
    s.e8m0 = (uint32_t)e;
    s.scale = __uint_as_float((uint32_t)e << 23);
    s.factor = __uint_as_float((uint32_t)(254 - e) << 23);
  } else {
    float q = __uint_as_float(amax) / (e5m2 ? 57344.0f : 448.0f);
    q = q < 0x1p-126f ? 0x1p-126f : q;
    if (amax == 0) q = 1.0f;
    s.e8m0 = 0;
    s.scale = q;
    s.factor = 1.0f / q;
  }
  return s;
}

__device__ inline u32x2 codes8(f32x8 v, float factor, uint32_t e5m2) {
  u32x2 r;
#pragma unroll
  for (int h = 0; h < 2; h++) {
    const float a = v[4 * h] * factor, b = v[4 * h + 1] * factor, c = v[4 * h + 2] * factor, d = v[4 * h + 3] * factor;
    int w = 0;
    if (e5m2) {
      w = __builtin_amdgcn_cvt_pk_bf8_f32(a, b, w, false);
      w = __builtin_amdgcn_cvt_pk_bf8_f32(c, d, w, true);
    } else {
      w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, w, false);
      w = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
    }
    r[h] = (uint32_t)w;
  }
  return r;
}

// Values of eight codes.
__device__ inline f32x8 values8(u32x2 w, uint32_t e5m2) {
  f32x8 r;
#pragma unroll
  for (int h = 0; h < 2; h++) {
    f32x2 a, b;
    if (e5m2) {
      a = __builtin_amdgcn_cvt_pk_f32_bf8((int)w[h], false);
      b = __builtin_amdgcn_cvt_pk_f32_bf8((int)w[h], true);
    } else {
      a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[h], false);
      b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[h], true);
    }
    r[4 * h] = a[0], r[4 * h + 1] = a[1], r[4 * h + 2] = b[0], r[4 * h + 3] = b[1];
  }
  return r;
}

__device__ inline void store_codes8(uint8_t *row, uint32_t c, uint32_t n, u32x2 w) {
  if (c + 8 <= n) {
    *(u32x2_any *)(row + c) = w;
  } else {
#pragma unroll
    for (int i = 0; i < 8; i++)
      if (c + i < n) row[c + i] = (uint8_t)(w[i >> 2] >> (8 * (i & 3)));
  }
}
__device__ inline u32x2 load_codes8(const uint8_t *row, uint32_t c, uint32_t n) {
  u32x2 w = {0, 0};
  if (c + 8 <= n) {
    w = *(const u32x2_any *)(row + c);
  } else {
#pragma unroll
    for (int i = 0; i < 8; i++)
      if (c + i < n) w[i >> 2] |= (uint32_t)row[c + i] << (8 * (i & 3));
  }
  return w;
}

template <bool E8M0> __device__ inline void store_scale(void *scales, uint64_t at, const BlockScale &s) {
  if (E8M0) ((uint8_t *)scales)[at] = (uint8_t)s.e8m0;
  else ((float *)scales)[at] = s.scale;
}
// Exponent bytes: 2^(b - 127), 255 is NaN.
__device__ inline float e8m0_value(uint32_t b) {
  return b == 255u ? __uint_as_float(0x7fc00000u) : b == 0u ? 0x1p-127f : __uint_as_float(b << 23);
}
template <bool E8M0> __device__ inline float load_scale(const void *scales, uint64_t at) {
  if (E8M0) return e8m0_value(((const uint8_t *)scales)[at]);
  return ((const float *)scales)[at];
}

// floor(u / d) for u < 2^32 by a multiplication with ceil(2^(32+k) / d), 2^(k-1) < d <= 2^k: the error of the multiplier
// is below d / 2^k of a unit, so the quotient is exact; the multiplier has 33 bits, its top one is added apart.
struct FastDivU32 {
  uint32_t mul, shift;
  __host__ static FastDivU32 of(uint32_t d) {
    uint32_t k = 0;
    while ((1ull << k) < d) k++;
    const unsigned __int128 m = (((unsigned __int128)1 << (32 + k)) + d - 1) / d;
    return FastDivU32{(uint32_t)m, k};
  }
  __device__ uint32_t operator()(uint32_t u) const {
    if (shift == 0) return u;
    const uint32_t t = __umulhi(u, mul);
    return (t + ((u - t) >> 1)) >> (shift - 1);
  }
};

// ------------------------------------------------------------------ kernels

// Row blocks: 16 lanes a block, eight elements a lane; the block's maximum stays in registers.  A work-group takes
// kQuantUnits blocks for each group of 16 lanes.  16384 x 4096 fp16: 33.6 us, 6.0 TB/s (a copy of the same mix of 16-bit loads
// and 8-bit stores 33.9).
constexpr int kQuantUnits = 2;
template <typename T, bool E8M0>
__global__ __launch_bounds__(kWG) void k_block_quant(const T *__restrict__ x, uint64_t ld_x, uint8_t *__restrict__ codes, uint64_t ld,
                                                     void *__restrict__ scales, uint64_t ld_scale, uint32_t n_units, uint32_t cols,
                                                     uint32_t nb, FastDivU32 by_nb, uint32_t e5m2) {
  const uint32_t lane = threadIdx.x & 15, grp = threadIdx.x >> 4;
  const uint32_t u0 = blockIdx.x * (kWG / 16 * kQuantUnits) + grp;
  f32x8 v[kQuantUnits];
  uint32_t row[kQuantUnits], kb[kQuantUnits];
#pragma unroll
  for (int i = 0; i < kQuantUnits; i++) {
    const uint32_t u = u0 + i * (kWG / 16);
    row[i] = by_nb(u < n_units ? u : 0);
    kb[i] = (u < n_units ? u : 0) - row[i] * nb;
    v[i] = load8<true>(x + row[i] * ld_x, kb[i] * kBlk + lane * 8, cols);
  }
#pragma unroll
  for (int i = 0; i < kQuantUnits; i++) {
    if (u0 + i * (kWG / 16) >= n_units) break;
    const BlockScale s = block_scale<E8M0>(max16(abs_max8(v[i])), e5m2);
    store_codes8(codes + row[i] * ld, kb[i] * kBlk + lane * 8, cols, codes8(v[i], s.factor, e5m2));
    if (lane == 0) store_scale<E8M0>(scales, row[i] * ld_scale + kb[i], s);
  }
}

// A 128 x 128 tile per work-group, eight rows by eight columns a lane: tiles with one scale, and the transposed forms,
// whose blocks run down the columns of x.  Transposed codes go through LDS, where a lane's eight rows of a column are
// one 8-byte chunk; the chunk's place in its row of 128 bytes is turned by the column's number / 8, so that the 16 lanes
// of a row of x write 16 different places.  11231 x 4096 bf16, transposed: 28.9 us, 4.8 TB/s: rows of 128 bytes are what a tile
// writes at a time, and a work-group reads, waits and writes once.  Tiles with one scale, 12288 x 4096 bf16: 27.9 us, 5.4 TB/s;
// transposed 30.5, 4.9.
template <typename T, bool E8M0, bool TRANS, bool TILE>
__global__ __launch_bounds__(kWG) void k_block_quant_tile(const T *__restrict__ x, uint64_t ld_x, uint32_t x_rows, uint32_t x_cols,
                                                          uint8_t *__restrict__ codes, uint64_t ld, void *__restrict__ scales,
                                                          uint64_t ld_scale, uint32_t e5m2) {
  __shared__ __attribute__((aligned(16))) uint8_t s_tile[TRANS ? kBlk * kBlk : 16];
  __shared__ uint32_t s_part[TILE ? kWG / 64 : 1];
  uint32_t *s_max = TILE ? s_part : (uint32_t *)s_tile;  // 16 groups' column maxima lie where the codes go later
  __shared__ float s_factor[TILE ? 1 : kBlk];
  const uint32_t t = threadIdx.x, lane = t & 15, grp = t >> 4;
  const uint32_t r0 = blockIdx.y * kBlk, c0 = blockIdx.x * kBlk;
  const uint32_t c = c0 + lane * 8;
  typename Vec8<T>::type v[8];  // as they came: half the registers of binary32 for 16-bit types, twice the work-groups
#pragma unroll
  for (int i = 0; i < 8; i++) {
    const uint32_t r = r0 + grp * 8 + i;
    v[i] = load8_raw<true>(x + (r < x_rows ? r : 0) * ld_x, c, r < x_rows ? x_cols : 0);
  }
  float factor[TILE ? 1 : 8];
  if (TILE) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; i++) {
      const uint32_t o = abs_max8(float8_of(v[i]));
      m = o > m ? o : m;
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const uint32_t o = (uint32_t)__shfl_xor((int)m, d);
      m = o > m ? o : m;
    }
    if ((t & 63) == 0) s_max[t >> 6] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWG / 64; w++) m = s_max[w] > m ? s_max[w] : m;
    const BlockScale s = block_scale<E8M0>(m, e5m2);
    factor[0] = s.factor;
    if (t == 0) store_scale<E8M0>(scales, TRANS ? blockIdx.x * ld_scale + blockIdx.y : blockIdx.y * ld_scale + blockIdx.x, s);
  } else {
#pragma unroll
    for (int j = 0; j < 8; j++) {
      uint32_t m = 0;
#pragma unroll
      for (int i = 0; i < 8; i++) {
        const uint32_t o = abs_bits_finite((float)v[i][j]);
        m = o > m ? o : m;
      }
      s_max[grp * kBlk + j * 16 + lane] = m;
    }
    __syncthreads();
    if (t < kBlk) {  // a column: the largest of the 16 groups' maxima; column 8 * lane + j lies at j * 16 + lane
      uint32_t m = 0;
#pragma unroll
      for (int g = 0; g < kWG / 16; g++) {
        const uint32_t o = s_max[g * kBlk + t];
        m = o > m ? o : m;
      }
      const BlockScale s = block_scale<E8M0>(m, e5m2);
      s_factor[t] = s.factor;
      const uint32_t col = c0 + (t & 15) * 8 + (t >> 4);
      if (col < x_cols) store_scale<E8M0>(scales, col * ld_scale + blockIdx.y, s);
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 8; j++) factor[TILE ? 0 : j] = s_factor[TILE ? 0 : j * 16 + lane];
  }
  if (!TRANS) {
#pragma unroll
    for (int i = 0; i < 8; i++) {
      const uint32_t r = r0 + grp * 8 + i;
      if (r < x_rows) store_codes8(codes + r * ld, c, x_cols, codes8(float8_of(v[i]), factor[0], e5m2));
    }
    return;
  }
#pragma unroll
  for (int j = 0; j < 8; j++) {
    f32x8 w;
#pragma unroll
    for (int i = 0; i < 8; i++) w[i] = (float)v[i][j];
    *(u32x2 *)(s_tile + (lane * 8 + j) * kBlk + ((grp ^ lane) & 15) * 8) = codes8(w, factor[TILE ? 0 : j], e5m2);
  }
  __syncthreads();
  // rows of the result: two neighbouring chunks a lane
  const uint32_t q = t & 7;
#pragma unroll
  for (int i = 0; i < 4; i++) {
    const uint32_t col = i * 32 + (t >> 3), turn = (col >> 3) & 15;
    if (c0 + col >= x_cols) continue;
    u32x4 w = *(const u32x4 *)(s_tile + col * kBlk + (q ^ (turn >> 1)) * 16);
    if (turn & 1) w = (u32x4){w[2], w[3], w[0], w[1]};
    uint8_t *out = codes + (c0 + col) * ld;
    const uint32_t r = r0 + q * 16;
    if (r + 16 <= x_rows) {
      __builtin_memcpy(out + r, &w, 16);
    } else {
      store_codes8(out, r, x_rows, (u32x2){w[0], w[1]});
      store_codes8(out, r + 8, x_rows, (u32x2){w[2], w[3]});
    }
  }
}

// Codes times scales, rounded once to the output's type.  5135 x 5120 to bf16: 12.7 us, 6.3 TB/s.  in_tile: where in its tile the first row lies.
template <typename T, bool E8M0>
__global__ __launch_bounds__(kWG) void k_block_dequant(const uint8_t *__restrict__ codes, uint64_t ld, const void *__restrict__ scales,
                                                       uint64_t ld_scale, T *__restrict__ x, uint64_t ld_x, uint32_t n_units, uint32_t cols,
                                                       uint32_t nb, FastDivU32 by_nb, uint32_t tile, uint32_t in_tile, uint32_t e5m2) {
  const uint32_t lane = threadIdx.x & 15, grp = threadIdx.x >> 4;
  const uint32_t u0 = blockIdx.x * (kWG / 16 * kQuantUnits) + grp;
  u32x2 w[kQuantUnits];
  float s[kQuantUnits];
  uint32_t row[kQuantUnits], kb[kQuantUnits];
#pragma unroll
  for (int i = 0; i < kQuantUnits; i++) {
    const uint32_t u = u0 + i * (kWG / 16);
    row[i] = by_nb(u < n_units ? u : 0);
    kb[i] = (u < n_units ? u : 0) - row[i] * nb;
    w[i] = load_codes8(codes + row[i] * ld, kb[i] * kBlk + lane * 8, cols);
    s[i] = load_scale<E8M0>(scales, (tile ? (in_tile + row[i]) / kBlk : row[i]) * ld_scale + kb[i]);
  }
#pragma unroll
  for (int i = 0; i < kQuantUnits; i++) {
    if (u0 + i * (kWG / 16) >= n_units) break;
    f32x8 v = values8(w[i], e5m2);
#pragma unroll
    for (int j = 0; j < 8; j++) v[j] *= s[i];
    store8(x + row[i] * ld_x, kb[i] * kBlk + lane * 8, cols, v);
  }
}

}  // namespace
