// rans_matmul.h -- C = A B^T of two matrices of 8-bit codes with block scales
//
// Part of the translation units rans_matmul_narrow.hip and rans_matmul_wide.hip; not a stand-alone header.
//
//   C[m, n] = sum over blocks b of sA[m, b] * sB[n or its tile, b] * (sum over k in b of A[m, k] * B[n, k])
//
// B's rows go to the matrix instruction's row operand and A's to its column operand: a lane then holds four neighbouring
// columns of one row of C, stores them at once, and needs one scale of A for them.  A K-step is one block, 128 bytes of a row.
//
// Sums.  The 8-bit matrix instructions add 128 products in binary32 with the smaller ones cut off below the leading bits of the
// largest of eight.  The error goes with |A| |B|^T and not with the element of C: at worst 7 * 2^-13 of it.  As a norm, over
// that of C, at K = 512 and 4096: normally distributed data 1.5e-5, with 1 % of the columns times 20 4.5e-5, log-normal magnitudes
// (one unit of the natural logarithm, both operands) 7e-5.  The result's own rounding is 2e-4 (binary16) or 1.7e-3 (bf16) on
// the same scale, so most elements are rounded as from exact sums: of normal data 2.5 % (binary16) and 0.3 % (bf16) lie on the
// other side of a tie or further off, and elements that cancel to little beside |A| |B|^T may be many of their own steps off.
// For binary32 results the codes are widened to bf16, which holds both formats exactly, and go through the bf16 instruction,
// which adds them in binary32 without such a loss (8e-8 as a norm at K = 4096) at half the rate.
#pragma once

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// 16 codes of a row from k on, those from K on are zero.  Rows may start anywhere.  The 16 around the row's end are its last
// 16, moved down (byte by byte is a trip to memory for each).
__device__ inline u32x4 load_codes16(const uint8_t *row, uint32_t k, uint32_t K) {
  u32x4 w = {0, 0, 0, 0};
  if (k + 16 <= K) {
    __builtin_memcpy(&w, row + k, 16);
  } else if (K >= 16) {
    if (k < K) {
      uint64_t q[2];
      __builtin_memcpy(q, row + K - 16, 16);
      const uint32_t by = (k + 16 - K) * 8;  // 8 to 120 bits
      const uint64_t lo = by < 64 ? q[0] >> by | q[1] << (64 - by) : q[1] >> (by - 64), hi = by < 64 ? q[1] >> by : 0;
      w = (u32x4){(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
    }
  } else {
    for (uint32_t i = 0; i < 16; i++)
      if (k + i < K) w[i >> 2] |= (uint32_t)row[k + i] << (8 * (i & 3));
  }
  return w;
}
__device__ inline i32x8 join8(u32x4 lo, u32x4 hi) {
  return (i32x8){(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
}

// An operand of 16 rows x 128 codes widened to bf16, as the bf16 instruction's four steps of 32 take it.  Both operands take
// their codes in the same order, so which 32 of the 128 a step holds does not matter.
struct Bf16Operand {
  bf16x8 q[4];
};
template <int FMT> __device__ inline Bf16Operand widen(i32x8 f) {
  Bf16Operand r;
#pragma unroll
  for (int i = 0; i < 8; i++) {
    const uint32_t w = (uint32_t)f[i];
    const bf16x2 a = FMT ? __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w, 1.0f, false) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false);
    const bf16x2 b = FMT ? __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w, 1.0f, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true);
    bf16x8 &o = r.q[i >> 1];
    const int at = 4 * (i & 1);
    o[at] = a[0], o[at + 1] = a[1], o[at + 2] = b[0], o[at + 3] = b[1];
  }
  return r;
}
__device__ inline f32x4 mfma_bf16(const Bf16Operand &b, const Bf16Operand &a) {
  f32x4 d = {0, 0, 0, 0};
#pragma unroll
  for (int q = 0; q < 4; q++) d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b.q[q], a.q[q], d, 0, 0, 0);
  return d;
}
template <int FA, int FB> __device__ inline f32x4 mfma_8bit(i32x8 b, i32x8 a) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, (f32x4){0, 0, 0, 0}, FB, FA, 0, 0, 0, 0);
}

__device__ inline float matmul_scale(const void *s, uint64_t at, uint32_t e8m0) {
  return e8m0 ? load_scale<true>(s, at) : load_scale<false>(s, at);
}

// ------------------------------------------------------------------ results

template <int OUT> __device__ inline uint32_t pack2(float a, float b) {
  typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
  if (OUT == RANS_F16) return __builtin_bit_cast(uint32_t, (f16x2){(_Float16)a, (_Float16)b});
  return __builtin_bit_cast(uint32_t, (bf16x2){(__bf16)a, (__bf16)b});
}
// Columns n .. n + 3 of row m.
__device__ inline void store_c4(const MatmulArgs &p, uint32_t m, uint32_t n, f32x4 v) {
  const uint64_t at = m * p.ldc + n;
  if (n + 4 <= p.n) {  // at once, wherever the row starts
    if (p.out == RANS_F32) {
      __builtin_memcpy((float *)p.c + at, &v, 16);
    } else {
      const u32x2 w = p.out == RANS_F16 ? (u32x2){pack2<RANS_F16>(v[0], v[1]), pack2<RANS_F16>(v[2], v[3])} : (u32x2){pack2<RANS_BF16>(v[0], v[1]), pack2<RANS_BF16>(v[2], v[3])};
      __builtin_memcpy((uint16_t *)p.c + at, &w, 8);
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

// A wave's part of a tile that lies inside C, 16-bit results: two neighbouring operands' results change places between
// lanes, so that a lane holds eight neighbouring columns and a row gets 64 bytes at once (32 without: 4096 x 8192 x 4096
// with power-of-two scales 146 -> 114 us).
template <int OUT, int NT, int MT> __device__ inline void store_c16(const MatmulArgs &p, uint32_t m, uint32_t n, uint32_t g, const f32x4 (&acc)[NT][MT]) {
#pragma unroll
  for (int j = 0; j < MT; j++) {
    uint16_t *row = (uint16_t *)p.c + (uint64_t)(m + j * 16) * p.ldc + n + (g & 1) * 16 + (g >> 1) * 8;
#pragma unroll
    for (int i = 0; i < NT; i += 2) {
      const auto lo = __builtin_amdgcn_permlane16_swap(pack2<OUT>(acc[i][j][0], acc[i][j][1]), pack2<OUT>(acc[i + 1][j][0], acc[i + 1][j][1]), false, false);
      const auto hi = __builtin_amdgcn_permlane16_swap(pack2<OUT>(acc[i][j][2], acc[i][j][3]), pack2<OUT>(acc[i + 1][j][2], acc[i + 1][j][3]), false, false);
      const u32x4 w = {lo[0], hi[0], lo[1], hi[1]};
      __builtin_memcpy(row + i * 16, &w, 16);
    }
  }
}

// ------------------------------------------------------------------ few rows of A

enum { MM_F32_TILE, MM_F32_ROW, MM_E8M0 };  // scales: binary32 with one of B for the wave's columns, binary32, powers of two

// Up to 16 MT rows of A: the work is reading B once.  A wave takes 16 rows of B and every W-th block of K, straight from
// memory into the operand's registers (no byte of B is used twice, so LDS would only add a copy), AHEAD blocks requested
// before the first is used; the waves' sums meet in LDS in a fixed order.  Rows behind the last one repeat it.  1 x 12288 x 4096:
// 10.3 us, 4.9 TB/s (bound by memory), powers of two 12.8; 16 rows 15.2, A read again for every 16 rows of B.
template <int FA, int FB, int SCALE, bool EXACT, int MT, int W, int AHEAD>
__global__ __launch_bounds__(W * 64) void k_block_matmul_few(MatmulArgs p) {
  __shared__ f32x4 s_sum[W][MT][64];
  const uint32_t t = threadIdx.x, lane = t & 63, r16 = lane & 15, g = lane >> 4, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const uint32_t n0 = blockIdx.x * 16, nb = (p.k + kBlk - 1) / kBlk, full = p.k / kBlk;
  constexpr size_t SB = SCALE == MM_E8M0 ? 1 : 4;
  constexpr bool HW = SCALE == MM_E8M0 && !EXACT;  // the instruction applies the scales
  constexpr int NS = SCALE == MM_F32_TILE || HW ? 1 : 4;  // scales of B that a lane needs
  const uint8_t *arow[MT], *sa[MT], *sb[NS];
  const uint32_t n = n0 + r16 < p.n ? n0 + r16 : p.n - 1;
  const uint8_t *brow = p.b + n * p.ldb + g * 16;
#pragma unroll
  for (int e = 0; e < NS; e++) {
    // 16 rows of B never span two tiles; exponents go to the instruction, which takes its row operand's from the row's lane
    const uint32_t ne = NS == 4 ? (n0 + g * 4 + e < p.n ? n0 + g * 4 + e : p.n - 1) : SCALE == MM_F32_TILE ? n0 : n;
    sb[e] = (const uint8_t *)p.sb + (p.b_tile ? ne / kBlk : ne) * p.ldsb * SB;
  }
#pragma unroll
  for (int j = 0; j < MT; j++) {
    const uint32_t m = j * 16 + r16 < p.m ? j * 16 + r16 : p.m - 1;
    arow[j] = p.a + m * p.lda + g * 16;
    sa[j] = (const uint8_t *)p.sa + m * p.ldsa * SB;
  }
  f32x4 acc[MT];
#pragma unroll
  for (int j = 0; j < MT; j++) acc[j] = (f32x4){0, 0, 0, 0};
  auto scale = [&](const uint8_t *q, uint32_t kb) {
    if (SCALE != MM_E8M0) return ((const uint32_t *)q)[kb];
    return HW ? (uint32_t)q[kb] : __float_as_uint(e8m0_value(q[kb]));
  };
  // ALL: AHEAD whole blocks, loads without conditions
  auto blocks = [&](uint32_t kb0, auto all_tag) {
    constexpr bool ALL = decltype(all_tag)::value;
    u32x4 b[AHEAD][2], a[AHEAD][MT][2];
    uint32_t va[AHEAD][MT], vb[AHEAD][NS];
    auto get = [&](const uint8_t *row, uint32_t k) {
      if (!ALL) return k + g * 16 < p.k ? load_codes16(row - g * 16, k + g * 16, p.k) : (u32x4){0, 0, 0, 0};
      u32x4 w;
      __builtin_memcpy(&w, row + k, 16);
      return w;
    };
#pragma unroll
    for (int u = 0; u < AHEAD; u++) {
      const uint32_t kb = kb0 + u * W;
      if (!ALL && kb >= nb) break;
      const uint32_t k = kb * kBlk;
      b[u][0] = get(brow, k), b[u][1] = get(brow, k + 64);
#pragma unroll
      for (int e = 0; e < NS; e++) vb[u][e] = scale(sb[e], kb);
#pragma unroll
      for (int j = 0; j < MT; j++) {
        a[u][j][0] = get(arow[j], k), a[u][j][1] = get(arow[j], k + 64);
        va[u][j] = scale(sa[j], kb);
      }
    }
#pragma unroll
    for (int u = 0; u < AHEAD; u++) {
      if (!ALL && kb0 + u * W >= nb) break;
      const i32x8 fb = join8(b[u][0], b[u][1]);
      Bf16Operand wb;
      if (EXACT) wb = widen<FB>(fb);
#pragma unroll
      for (int j = 0; j < MT; j++) {
        const i32x8 fa = join8(a[u][j][0], a[u][j][1]);
        if (HW) {
          acc[j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fb, fa, acc[j], FB, FA, 0, (int)vb[u][0], 0, (int)va[u][j]);
          continue;
        }
        const f32x4 d = EXACT ? mfma_bf16(wb, widen<FA>(fa)) : mfma_8bit<FA, FB>(fb, fa);
#pragma unroll
        for (int e = 0; e < 4; e++) acc[j][e] = __builtin_fmaf(d[e], __uint_as_float(va[u][j]) * __uint_as_float(vb[u][NS == 4 ? e : 0]), acc[j][e]);
      }
    }
  };
  uint32_t kb0 = wave;
  for (; kb0 + W * (AHEAD - 1) < full; kb0 += W * AHEAD) blocks(kb0, std::true_type{});
  for (; kb0 < nb; kb0 += W * AHEAD) blocks(kb0, std::false_type{});
#pragma unroll
  for (int j = 0; j < MT; j++) s_sum[wave][j][lane] = acc[j];
  __syncthreads();
  if (wave < MT) {
    f32x4 v = s_sum[0][wave][lane];
#pragma unroll
    for (int w = 1; w < W; w++) v += s_sum[w][wave][lane];
    const uint32_t m = wave * 16 + r16, c = n0 + g * 4;
    if (m < p.m && c < p.n) store_c4(p, m, c, v);
  }
}

// ------------------------------------------------------------------ tiles through LDS

// A tile of C: WN x WM waves, each NT x MT operands of 16 rows of B and of A; STAGES blocks of codes, and twice as many blocks'
// scales, in LDS.
template <int WN, int WM, int NT, int MT, int STAGES> struct MmTile {
  static constexpr int wn = WN, wm = WM, nt = NT, mt = MT, stages = STAGES, threads = 64 * WN * WM, bn = WN * NT * 16, bm = WM * MT * 16, rows = bm + bn;
};
constexpr uint64_t kMmMaxLd = 1u << 23;  // rows of codes up to this far apart: 32-bit offsets inside a tile

// Work-groups go round robin over the eight dies: gives each die consecutive tiles, and those in groups of eight tiles of A,
// so that the tiles a die works on at a time share rows of A and of B in its L2.
__device__ inline void mm_tile_of(uint32_t bid, uint32_t tiles_m, uint32_t tiles_n, uint32_t *tm, uint32_t *tn) {
  const uint32_t total = tiles_m * tiles_n, per = total / 8, more = total % 8, xcd = bid % 8;
  const uint32_t i = xcd * per + (xcd < more ? xcd : more) + bid / 8;
  constexpr uint32_t gm = 8;
  const uint32_t group = i / (gm * tiles_n), first = group * gm, rows = tiles_m - first < gm ? tiles_m - first : gm;
  const uint32_t in = i - group * gm * tiles_n;
  *tm = first + in % rows;
  *tn = in / rows;
}

// A row's scales of `stages` blocks in LDS: as many words of binary32, or a word of as many exponents where the instruction
// applies them.  For widened products exponents become numbers here, once a block and not with each use (4096 x 4096 x 11231
// 557 -> 435 us).
template <int SCALE, bool EXACT> constexpr bool mm_bytes = SCALE == MM_E8M0 && !EXACT;
template <typename TILE, int SCALE, bool EXACT> __device__ __forceinline__ void mm_put_scale(uint32_t *scales, uint32_t row, u32x4 v) {
  if (mm_bytes<SCALE, EXACT>) {
    scales[row] = v[0];
    return;
  }
  if (SCALE == MM_E8M0) {
    const uint32_t w = v[0];
#pragma unroll
    for (int j = 0; j < TILE::stages; j++) v[j] = __float_as_uint(e8m0_value(w >> (8 * j) & 255u));
  }
  if (TILE::stages == 4) *(u32x4 *)(scales + row * 4) = v;
  else *(u32x2 *)(scales + row * 2) = (u32x2){v[0], v[1]};
}
template <typename TILE, int SCALE, bool EXACT> __device__ __forceinline__ uint32_t mm_scale(const uint32_t *scales, uint32_t row, uint32_t step) {
  if (!mm_bytes<SCALE, EXACT>) return scales[row * TILE::stages + step];
  return scales[row] >> (8 * step);  // the instruction takes the lowest byte
}

// One K-step of a wave: its operands and scales from LDS, its products.  A row's eight chunks of 16 bytes lie turned, chunk c
// of row r at place c ^ (r & 7), so that the 16 rows that an operand takes the same chunk of are read from different banks.
// The order is pinned: an operand of B is read while the products of the one before it run, and binary32 scales are applied
// to the products before those that run.
template <typename TILE, int FA, int FB, int SCALE, bool EXACT>
__device__ __forceinline__ void mm_step(const uint8_t *__restrict__ code, const uint32_t *scales, uint32_t step, uint32_t wm, uint32_t wn, uint32_t lane,
                                        f32x4 (&acc)[TILE::nt][TILE::mt]) {
  constexpr int NT = TILE::nt, MT = TILE::mt;
  constexpr bool HW = SCALE == MM_E8M0 && !EXACT;       // the instruction applies the scales
  constexpr bool ROWS4 = !HW && SCALE != MM_F32_TILE;   // each row of B has its own
  const uint32_t r16 = lane & 15, g = lane >> 4, turned = r16 * kBlk + (g ^ (r16 & 7)) * 16;
  const uint32_t ra = wm * MT * 16, rb = TILE::bm + wn * NT * 16;
  auto frag = [&](uint32_t row) {
    const uint8_t *at = code + row * kBlk;
    return join8(*(const u32x4 *)(at + turned), *(const u32x4 *)(at + (turned ^ 64)));
  };
  auto scale8 = [&](int i) { return HW ? mm_scale<TILE, SCALE, EXACT>(scales, rb + i * 16 + r16, step) : 0u; };
  auto scale4 = [&](int i) {
    f32x4 v = {0, 0, 0, 0};
    if (ROWS4) {
#pragma unroll
      for (int e = 0; e < 4; e++) v[e] = __uint_as_float(mm_scale<TILE, SCALE, EXACT>(scales, rb + i * 16 + g * 4 + e, step));
    }
    return v;
  };
  i32x8 fa[EXACT ? 1 : MT];
  Bf16Operand wa[EXACT ? MT : 1];
  uint32_t sa[MT];
#pragma unroll
  for (int j = 0; j < MT; j++) {
    if (EXACT) wa[j] = widen<FA>(frag(ra + j * 16));
    else fa[j] = frag(ra + j * 16);
    sa[j] = mm_scale<TILE, SCALE, EXACT>(scales, ra + j * 16 + r16, step);
  }
  i32x8 fb = frag(rb);
  uint32_t sb8 = scale8(0);
  f32x4 d[2][MT], sb4[3];
  sb4[0] = scale4(0);
  if (SCALE == MM_F32_TILE) {
    const float sb = __uint_as_float(mm_scale<TILE, SCALE, EXACT>(scales, rb, step));
#pragma unroll
    for (int j = 0; j < MT; j++) sa[j] = __float_as_uint(__uint_as_float(sa[j]) * sb);
  }
  auto apply = [&](int i) {
#pragma unroll
    for (int j = 0; j < MT; j++)
#pragma unroll
      for (int e = 0; e < 4; e++) {
        const float s = ROWS4 ? __uint_as_float(sa[j]) * sb4[i % 3][e] : __uint_as_float(sa[j]);
        acc[i][j][e] = __builtin_fmaf(d[i & 1][j][e], s, acc[i][j][e]);
      }
  };
#pragma unroll
  for (int i = 0; i < NT; i++) {
    i32x8 fb_next = fb;
    uint32_t sb8_next = sb8;
    if (i + 1 < NT) {
      fb_next = frag(rb + (i + 1) * 16);
      sb8_next = scale8(i + 1);
      sb4[(i + 1) % 3] = scale4(i + 1);
    }
    __builtin_amdgcn_sched_barrier(0);
    if (EXACT) {
      const Bf16Operand wb = widen<FB>(fb);
#pragma unroll
      for (int q = 0; q < 4; q++)  // a sum's four steps depend on one another: in turn with the other sums'
#pragma unroll
        for (int j = 0; j < MT; j++)
          d[i & 1][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wb.q[q], wa[EXACT ? j : 0].q[q], q ? d[i & 1][j] : (f32x4){0, 0, 0, 0}, 0, 0, 0);
    } else {
#pragma unroll
      for (int j = 0; j < MT; j++) {
        if (HW)
          acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fb, fa[EXACT ? 0 : j], acc[i][j], FB, FA, 0, (int)sb8, 0, (int)sa[j]);
        else
          d[i & 1][j] = mfma_8bit<FA, FB>(fb, fa[EXACT ? 0 : j]);
      }
    }
    if (!HW && i > 0) apply(i - 1);
    __builtin_amdgcn_sched_barrier(0);
    fb = fb_next;
    sb8 = sb8_next;
  }
  if (!HW) apply(NT - 1);
  // the products stay in front of the next block's reads, whose operands would need registers beside this block's otherwise
#pragma unroll
  for (int i = 0; i < NT; i++)
#pragma unroll
    for (int j = 0; j < MT; j++) asm volatile("" : "+v"(acc[i][j]));
}

// The part of K that a work-group takes (blockIdx.y), as a product of its own.
template <int SCALE> __device__ __forceinline__ void mm_part(MatmulArgs &p) {
  const uint32_t z = blockIdx.y, k0 = z * p.part_blocks * kBlk, left = p.k - k0, most = p.part_blocks * kBlk;
  p.a += k0;
  p.b += k0;
  p.sa = (const uint8_t *)p.sa + z * p.part_blocks * (SCALE == MM_E8M0 ? 1 : 4);
  p.sb = (const uint8_t *)p.sb + z * p.part_blocks * (SCALE == MM_E8M0 ? 1 : 4);
  p.c = (float *)p.c + z * (uint64_t)p.m * p.ldc;
  p.k = left < most ? left : most;
}

// The parts' sums in their order, rounded once: four columns a lane.
__global__ __launch_bounds__(kWG) void k_block_matmul_sum(MatmulArgs p, const float *__restrict__ part, uint32_t parts, uint64_t ld) {
  const uint32_t n = (blockIdx.x * kWG + threadIdx.x) * 4;
  const uint32_t m = blockIdx.y;
  if (n >= p.n) return;
  f32x4 v = {0, 0, 0, 0};
  part += m * ld + n;
#pragma unroll 8
  for (uint32_t s = 0; s < parts; s++) v += *(const f32x4 *)(part + s * p.m * ld);
  store_c4(p, m, n, v);
}

// A wave's results of a tile.
template <typename TILE> __device__ __forceinline__ void mm_store(const MatmulArgs &p, uint32_t m0, uint32_t n0, uint32_t wm, uint32_t wn, uint32_t lane, const f32x4 (&acc)[TILE::nt][TILE::mt]) {
  constexpr int NT = TILE::nt, MT = TILE::mt;
  const uint32_t g = lane >> 4, m = m0 + wm * MT * 16 + (lane & 15), n = n0 + wn * NT * 16;
  if (p.out != RANS_F32 && m0 + TILE::bm <= p.m && n0 + TILE::bn <= p.n) {
    if (p.out == RANS_F16) store_c16<RANS_F16>(p, m, n, g, acc);
    else store_c16<RANS_BF16>(p, m, n, g, acc);
    return;
  }
#pragma unroll
  for (int i = 0; i < NT; i++)
#pragma unroll
    for (int j = 0; j < MT; j++)
      if (m + j * 16 < p.m && n + i * 16 + g * 4 < p.n) store_c4(p, m + j * 16, n + i * 16 + g * 4, acc[i][j]);
}

// Codes and scales of a tile through registers: any alignment, zeros behind the end of a row.
template <typename TILE, int SCALE, bool EXACT> struct MmRegs {
  static constexpr int NTH = TILE::threads, LA = TILE::bm * 8 / NTH, LOADS = TILE::rows * 8 / NTH, SROWS = (TILE::rows + NTH - 1) / NTH;
  static constexpr int S = TILE::stages;
  u32x4 st[LOADS];
  u32x4 sc[SROWS];
  __device__ __forceinline__ void load(const MatmulArgs &p, uint32_t m0, uint32_t n0, uint32_t kb) {
    const uint32_t t = threadIdx.x;
#pragma unroll
    for (int i = 0; i < LOADS; i++) {
      const uint32_t r = (i < LA ? i : i - LA) * (NTH / 8) + (t >> 3);
      const uint32_t m = m0 + r < p.m ? m0 + r : p.m - 1, n = n0 + r < p.n ? n0 + r : p.n - 1;
      st[i] = load_codes16(i < LA ? p.a + m * p.lda : p.b + n * p.ldb, kb * kBlk + (t & 7) * 16, p.k);
    }
  }
  __device__ __forceinline__ void put(uint8_t *code) const {
    const uint32_t t = threadIdx.x;
#pragma unroll
    for (int i = 0; i < LOADS; i++) {
      const uint32_t r = (i < LA ? i : i - LA) * (NTH / 8) + (t >> 3);
      *(u32x4 *)(code + (i < LA ? 0 : TILE::bm * kBlk) + r * kBlk + (((t & 7) ^ (r & 7)) * 16)) = st[i];
    }
  }
  __device__ __forceinline__ void load_scales(const MatmulArgs &p, uint32_t m0, uint32_t n0, uint32_t kb0, uint32_t nb) {
#pragma unroll
    for (int i = 0; i < SROWS; i++) {
      const uint32_t r = i * NTH + threadIdx.x;
      const bool is_a = r < (uint32_t)TILE::bm;
      const uint32_t m = m0 + r < p.m ? m0 + r : p.m - 1, n = n0 + (r - TILE::bm) < p.n ? n0 + (r - TILE::bm) : p.n - 1;
      const uint64_t at = is_a ? m * p.ldsa : (uint64_t)(p.b_tile ? n / kBlk : n) * p.ldsb;
      const void *s = is_a ? p.sa : p.sb;
      sc[i] = (u32x4){0, 0, 0, 0};
#pragma unroll
      for (int j = 0; j < S; j++) {
        const uint32_t kb = kb0 + j < nb ? kb0 + j : nb - 1;
        if (SCALE == MM_E8M0) sc[i][0] |= (uint32_t)((const uint8_t *)s)[at + kb] << (8 * j);
        else sc[i][j] = ((const uint32_t *)s)[at + kb];
      }
    }
  }
  __device__ __forceinline__ void put_scales(uint32_t *scales) const {
#pragma unroll
    for (int i = 0; i < SROWS; i++) {
      const uint32_t r = i * NTH + threadIdx.x;
      if (TILE::rows % NTH == 0 || r < (uint32_t)TILE::rows) mm_put_scale<TILE, SCALE, EXACT>(scales, r, sc[i]);
    }
  }
};

// Operands of any alignment: two stages, the next block in registers while this one's products run.  With widened operands
// those registers are too many: 128 x 256 tiles spill 109 (binary32 scales) or 31 (powers of two), 128 x 128 ones 30.
template <typename TILE, int FA, int FB, int SCALE, bool EXACT>
__global__ __launch_bounds__(TILE::threads, 2) void k_block_matmul_any(MatmulArgs p, uint32_t tiles_m, uint32_t tiles_n) {
  if (p.part_blocks) mm_part<SCALE>(p);
  __shared__ __attribute__((aligned(16))) uint8_t s_code[2][TILE::rows * kBlk];
  __shared__ __attribute__((aligned(16))) uint32_t s_scale[2][TILE::rows * (mm_bytes<SCALE, EXACT> ? 1 : TILE::stages)];
  const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave % TILE::wm, wn = wave / TILE::wm;
  uint32_t tm, tn;
  mm_tile_of(blockIdx.x, tiles_m, tiles_n, &tm, &tn);
  const uint32_t m0 = tm * TILE::bm, n0 = tn * TILE::bn, nb = (p.k + kBlk - 1) / kBlk;
  MmRegs<TILE, SCALE, EXACT> q;
  f32x4 acc[TILE::nt][TILE::mt];
#pragma unroll
  for (int i = 0; i < TILE::nt; i++)
#pragma unroll
    for (int j = 0; j < TILE::mt; j++) acc[i][j] = (f32x4){0, 0, 0, 0};
  if (nb) {
    q.load(p, m0, n0, 0);
    q.load_scales(p, m0, n0, 0, nb);
    q.put(s_code[0]);
    q.put_scales(s_scale[0]);
  }
  __syncthreads();
  constexpr uint32_t S = TILE::stages;
  for (uint32_t kb = 0; kb < nb; kb++) {
    if (kb + 1 < nb) q.load(p, m0, n0, kb + 1);
    if (kb % S == 0 && kb + S < nb) q.load_scales(p, m0, n0, kb + S, nb);
    mm_step<TILE, FA, FB, SCALE, EXACT>(s_code[kb & 1], s_scale[kb / S & 1], kb % S, wm, wn, lane, acc);
    if (kb + 1 < nb) q.put(s_code[(kb + 1) & 1]);
    // the set of scales that is replaced was last read before the last barrier
    if (kb % S == S - 1 && kb + 1 < nb) q.put_scales(s_scale[(kb + 1) / S & 1]);
    __syncthreads();
  }
  mm_store<TILE>(p, m0, n0, wm, wn, lane, acc);
}

#ifdef __HIP_DEVICE_COMPILE__
typedef __attribute__((address_space(3))) void LdsVoid;
// Rows of codes straight into LDS, 1 KB a wave and load (lane l: row l / 8 of the eight, place l % 8).  `at`: a lane's offsets
// in `src`.
template <int N, int WAVES>
__device__ __forceinline__ void mm_fetch(uint8_t *dst, __amdgpu_buffer_rsrc_t src, const uint32_t (&at)[N], uint32_t k, uint32_t wave) {
#pragma unroll
  for (int i = 0; i < N; i++) __builtin_amdgcn_raw_ptr_buffer_load_lds(src, (LdsVoid *)(dst + (i * WAVES + wave) * 1024), 16, at[i], k, 0, 0);
}
#endif

// Operands whose rows of codes start on 16 bytes: codes go to LDS directly.  A ring of stages;
// one barrier a block, behind which the block's codes are there and the stage before it is free for the block STAGES - 1
// ahead.  Each stage is an LDS variable of its own and the loop's fetches are unconditional (behind the last block they repeat
// it, into a stage that nobody reads): the compiler then sees which loads a read has to wait for, and waits for no others.
// The last block of a K that is no multiple of 128 goes through registers.
// 16384 x 12288 x 4096, powers of two: 720 us, 2.3 PFLOP/s (a loop of the same instructions on such data and nothing else 3.0, for
// the clock falls to 2.1 GHz); the matrix units are busy 52 % of the cycles, the rest goes to the barriers' rounds.  395 x 12288 x
// 4096: 35 us; the tiles are 1.5 for a compute unit, and a step of one waits for its fetch.  Widened, 4096 x 4096 x 11231: 383 us,
// 0.98 PFLOP/s: for each matrix instruction four vector ones widen and scale, most of whose time is not hidden behind it; 128 x 128 tiles use
// all 256 registers and spill five (powers of two seven).
template <typename TILE, int FA, int FB, int SCALE, bool EXACT>
__global__ __launch_bounds__(TILE::threads, 2) void k_block_matmul(MatmulArgs p, uint32_t tiles_m, uint32_t tiles_n) {
#ifdef __HIP_DEVICE_COMPILE__
  constexpr int BM = TILE::bm, BN = TILE::bn, NTH = TILE::threads, ROWS = TILE::rows, W = NTH / 64, S = TILE::stages;
  constexpr int LA = BM * 8 / NTH, LB = BN * 8 / NTH, SROWS = (ROWS + NTH - 1) / NTH;
  constexpr uint32_t SB = SCALE == MM_E8M0 ? 1 : 4;  // bytes of a scale
  static_assert(S == 2 || S == 4, "scales are loaded as two or four");
  if (p.part_blocks) mm_part<SCALE>(p);
  __shared__ __attribute__((aligned(1024))) uint8_t s_code0[ROWS * kBlk];
  __shared__ __attribute__((aligned(1024))) uint8_t s_code1[ROWS * kBlk];
  __shared__ __attribute__((aligned(1024))) uint8_t s_code2[S > 2 ? ROWS * kBlk : 16];
  __shared__ __attribute__((aligned(1024))) uint8_t s_code3[S > 2 ? ROWS * kBlk : 16];
  __shared__ __attribute__((aligned(16))) uint32_t s_scale[2][ROWS * (mm_bytes<SCALE, EXACT> ? 1 : S)];
  auto stage = [&](int i) { return i % S == 0 ? s_code0 : i % S == 1 ? s_code1 : i % S == 2 ? s_code2 : s_code3; };
  const uint32_t t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), wm = wave % TILE::wm, wn = wave / TILE::wm;
  uint32_t tm, tn;
  mm_tile_of(blockIdx.x, tiles_m, tiles_n, &tm, &tn);
  const uint32_t m0 = tm * BM, n0 = tn * BN, nb = (p.k + kBlk - 1) / kBlk, full = p.k / kBlk;
  // last row of the tile that exists; the ones behind it repeat it
  const uint32_t am = (p.m - m0 < BM ? p.m - m0 : BM) - 1, bn = (p.n - n0 < BN ? p.n - n0 : BN) - 1;
  const __amdgpu_buffer_rsrc_t a = __builtin_amdgcn_make_buffer_rsrc((void *)(p.a + m0 * p.lda), 0, am * (uint32_t)p.lda + p.k, 0x00027000);
  const __amdgpu_buffer_rsrc_t b = __builtin_amdgcn_make_buffer_rsrc((void *)(p.b + n0 * p.ldb), 0, bn * (uint32_t)p.ldb + p.k, 0x00027000);
  uint32_t va[LA], vb[LB];
  const uint32_t chunk = ((lane & 7) ^ (lane >> 3)) * 16;
#pragma unroll
  for (int i = 0; i < LA; i++) {
    const uint32_t r = (i * W + wave) * 8 + (lane >> 3);
    va[i] = (r < am ? r : am) * (uint32_t)p.lda + chunk;
  }
#pragma unroll
  for (int i = 0; i < LB; i++) {
    const uint32_t r = (i * W + wave) * 8 + (lane >> 3);
    vb[i] = (r < bn ? r : bn) * (uint32_t)p.ldb + chunk;
  }
  auto fetch = [&](uint8_t *dst, uint32_t kb) {
    mm_fetch<LA, W>(dst, a, va, kb * kBlk, wave);
    mm_fetch<LB, W>(dst + BM * kBlk, b, vb, kb * kBlk, wave);
  };
  // scales: a thread brings a row's of S blocks with one load, which near the row's end begins as many blocks earlier as it
  // would read past it (`back`)
  const uint8_t *sp[SROWS];
  u32x4 sc[SROWS];
#pragma unroll
  for (int i = 0; i < SROWS; i++) {
    const uint32_t r = i * NTH + t, n = n0 + (r - BM < bn ? r - BM : bn);
    const uint8_t *qa = (const uint8_t *)p.sa + (m0 + (r < am ? r : am)) * p.ldsa * SB;
    const uint8_t *qb = (const uint8_t *)p.sb + (p.b_tile ? n / kBlk : n) * p.ldsb * SB;
    sp[i] = r < (uint32_t)BM ? qa : qb;
  }
  auto load_scales = [&](uint32_t kb) {
    const uint32_t at = (kb + S <= nb ? kb : nb - S) * SB;
#pragma unroll
    for (int i = 0; i < SROWS; i++) __builtin_memcpy(&sc[i], sp[i] + at, S * SB);
  };
  auto put_scales = [&](uint32_t set) {
#pragma unroll
    for (int i = 0; i < SROWS; i++) {
      const uint32_t r = i * NTH + t;
      if (ROWS % NTH == 0 || r < (uint32_t)ROWS) mm_put_scale<TILE, SCALE, EXACT>(s_scale[set], r, sc[i]);
    }
  };
  auto sync = [&](auto outstanding) {  // loads end in order: all but the last `outstanding` have
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(decltype(outstanding)::value) : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  typedef std::integral_constant<int, 0> None;
  typedef std::integral_constant<int, (S - 2) * (LA + LB)> Ahead;
  f32x4 acc[TILE::nt][TILE::mt];
#pragma unroll
  for (int i = 0; i < TILE::nt; i++)
#pragma unroll
    for (int j = 0; j < TILE::mt; j++) acc[i][j] = (f32x4){0, 0, 0, 0};
  uint32_t kb = 0;
  if (nb >= S) {
    load_scales(0);
  } else {
#pragma unroll
    for (int i = 0; i < SROWS; i++)
      for (uint32_t j = 0; j < nb; j++) {
        if (SCALE == MM_E8M0) sc[i][0] = (j ? sc[i][0] : 0) | (uint32_t)sp[i][j] << (8 * j);
        else sc[i][j] = ((const uint32_t *)sp[i])[j];
      }
  }
  if (full) {
#pragma unroll
    for (int i = 0; i < S - 1; i++) fetch(stage(i), i < (int)full ? i : full - 1);
  }
  if (nb) put_scales(0);
  uint32_t set = 0;
  for (; kb + S <= full; kb += S, set ^= 1) {
#pragma unroll
    for (int s = 0; s < S; s++) {
      sync(Ahead{});
      if (s == 0) load_scales(kb + S);
      const uint32_t ahead = kb + s + S - 1;
      fetch(stage(s + S - 1), ahead < full ? ahead : full - 1);
      mm_step<TILE, FA, FB, SCALE, EXACT>(stage(s), s_scale[set], s, wm, wn, lane, acc);
      if (s == S - 1) put_scales(set ^ 1);  // last read in the round before this one
    }
  }
  // fewer whole blocks than a round, then what is left of a row
  const uint32_t back = nb >= S && kb + S > nb ? kb + S - nb : 0;
  MmRegs<TILE, SCALE, EXACT> q;
  if (full < nb) q.load(p, m0, n0, full);
#pragma unroll
  for (int s = 0; s < S - 1; s++)
    if (kb + s < full) {
      sync(None{});
      mm_step<TILE, FA, FB, SCALE, EXACT>(stage(s), s_scale[set], s + back, wm, wn, lane, acc);
    }
  sync(None{});
  if (full < nb) {
    q.put(s_code0);
    sync(None{});
    mm_step<TILE, FA, FB, SCALE, EXACT>(s_code0, s_scale[set], full % S + back, wm, wn, lane, acc);
  }
  mm_store<TILE>(p, m0, n0, wm, wn, lane, acc);
#endif
}

}  // namespace
