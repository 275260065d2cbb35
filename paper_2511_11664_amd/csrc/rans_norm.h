// rans_norm.h -- root-mean-square norm with the residual's addition and an output in 8 bits; its gradients
//
// Part of the translation unit rans_blocks.hip; not a stand-alone header.
//
// Forward, a row of K elements:  h = x + residual, rounded to the stream's type, because that is what the next residual
// addition and the backward pass read;  rstd = 1 / sqrt(sum h^2 / K + eps);  y = h * rstd * w, half a step of binary32 off
// and a little (rstd is kept in two parts);  codes and scales of y by the row blocks of rans_blocks.h, and / or y itself.
// Backward:  g = dy * w, xh = h * rstd;  dx = rstd * (g - xh * sum(g * xh) / K) + dsum;  dw = sum over rows of dy * xh.
// Squares of a row and their sum are binary64: no finite h overflows or vanishes there, and the sum's error does not show in
// rstd.  The backward's sums are binary32: a lane's own eight neighbours (and every further eight), then the lanes of a wave,
// then the waves.
//
// Bound by memory: each tensor is read once and written once, a row lives in registers between its sum and its output.
#pragma once

namespace {

// Sum over a work-group of NT threads, in every thread.  `s`: NT / 64 numbers.
template <int NT, typename N> __device__ inline N group_sum(N v, N *s) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d);
  if (NT == 64) return v;
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
  __syncthreads();
  N r = 0;
#pragma unroll
  for (int w = 0; w < NT / 64; w++) r += s[w];
  return r;
}

struct NormFwd {
  const void *x, *res, *weight;
  void *sum, *y;
  float *rstd;
  uint8_t *codes;
  void *scales;
  uint64_t ld_x, ld_res, ld_sum, ld_y, ld, ld_scale;
  uint32_t cols, e5m2;
  float eps;
  double inv_cols;
};

// 1 / sqrt(sum / cols + eps) as the nearest binary32 number and what it leaves: the approximate reciprocal root r of the mean m,
// whose own rounding errors are kept beside it, takes one step r + r / 2 (1 - m r^2).  Codes are a rounding of y to a few bits,
// and y is off by half a step of binary32 and not by one or two, so that fewer of them fall on the other side of a tie.
// Rows far from one, whose reciprocal root may pass binary32's range: h is multiplied by `pre`, a power of two, and r + low is
// the reciprocal root over it.  `out`: what the backward pass gets.
struct Rstd {
  float r, low, pre, out;
};
__device__ __forceinline__ Rstd rstd_of(double sum, const NormFwd &a) {
  const double mean = sum * a.inv_cols + (double)a.eps;
  const float m = (float)mean, m_low = (float)(mean - (double)m);
  if (!(m >= 0x1p-100f && m < 0x1p100f)) {
    if (!(mean > 0 && mean < (double)INFINITY)) {
      const float r = 1.0f / sqrtf(m);
      return Rstd{r, 0.0f, 1.0f, r};
    }
    // least mean 2^-328 (one subnormal number in 2^30): h * 2^64 is below 2^14 sqrt(K); largest 2^256
    const float pre = mean < 1 ? 0x1p64f : 0x1p-32f;
    const double d = 1.0 / sqrt(mean), q = d / (double)pre;
    const float r = (float)q;
    return Rstd{r, (float)(q - (double)r), pre, (float)d};
  }
  const float r = __builtin_amdgcn_rsqf(m), t = m * r, t_low = __builtin_fmaf(m_low, r, __builtin_fmaf(m, r, -t));
  const float step = 0.5f * r * __builtin_fmaf(-t_low, r, __builtin_fmaf(-t, r, 1.0f));
  const float high = r + step;
  return Rstd{high, (r - high) + step, 1.0f, high};
}

// A row per work-group of NT threads, NV times eight neighbouring elements a thread (NV = 0: any length, h read again).
// Everything a thread needs from memory is requested before the row's sum, the weight too.  16384 x 4096 fp16 with a residual,
// sums and codes written: 82 us, 5.8 TB/s; 8 rows 3.6 us, the launch and one trip to memory.  NV = 0, 4096 x 12288 bf16: 75 us,
// 4.7 TB/s, as h is read once more.
template <typename T, typename W, bool E8M0, int NT, int NV>
__global__ __launch_bounds__(NT) void k_norm_quant(NormFwd a, uint64_t row0) {
  typedef typename Vec8<T>::type V;
  __shared__ double s_sum[NT / 64];
  const uint64_t row = row0 + blockIdx.x;
  const uint32_t t = threadIdx.x, n = a.cols;
  const T *x = (const T *)a.x + row * a.ld_x;
  const T *res = a.res ? (const T *)a.res + row * a.ld_res : nullptr;
  T *sum = a.sum ? (T *)a.sum + row * a.ld_sum : nullptr;
  double acc = 0;
  Rstd rstd = {0, 0, 1, 0};
  auto add = [&](V v, V r) {
    f32x8 h = float8_of(v);
    if (res) {
#pragma unroll
      for (int i = 0; i < 8; i++) h[i] = (float)(T)(h[i] + (float)r[i]);
    }
    return h;
  };
  auto square = [&](f32x8 h) {
    double q[2] = {0, 0};  // two chains: a link waits for the one before
#pragma unroll
    for (int i = 0; i < 8; i++) q[i & 1] = __builtin_fma((double)h[i], (double)h[i], q[i & 1]);
    acc += q[0] + q[1];
  };
  auto weight8 = [&](uint32_t c) { return a.weight ? load8((const W *)a.weight, c, n) : (f32x8){1, 1, 1, 1, 1, 1, 1, 1}; };
  auto give = [&](uint32_t c, f32x8 h8, f32x8 w) {
    // 16 lanes hold a block; lanes behind the row's end hold zeros and take part in its maximum
    if (rstd.pre != 1) {
#pragma unroll
      for (int i = 0; i < 8; i++) h8[i] *= rstd.pre;
    }
    // h * rstd in two parts times w; an infinite w meets the lower part as a finite one
    auto lower = [&](int i, float x) { return __builtin_fmaf(h8[i], rstd.low, __builtin_fmaf(h8[i], rstd.r, -x)) * __builtin_amdgcn_fmed3f(w[i], -0x1.fffffep127f, 0x1.fffffep127f); };
    f32x8 v;
    // 0 where a y may lie on a border under powers of two, as far as its binary32 tells: halfway between two codes (normal ones
    // have one bit more than a code there, subnormal ones fewer) or at a scale's largest number
    uint32_t border = 1;
#pragma unroll
    for (int i = 0; i < 8; i++) {
      const float x = h8[i] * rstd.r;
      v[i] = __builtin_fmaf(x, w[i], lower(i, x));
      if (E8M0) {
        const uint32_t low = __float_as_uint(v[i]) << (a.e5m2 ? 12 : 13);
        border = low < border ? low : border;
      }
    }
    if (a.y && c < n) store8((T *)a.y + row * a.ld_y, c, n, v);
    if (a.codes) {
      if (E8M0 && border == 0 && c < n) {
        // powers of two leave a y on its side of a border: what binary32 dropped decides, as the next number on that side (a y
        // below some 2^-120 may have dropped what no binary32 number holds, and stays)
#pragma unroll
        for (int i = 0; i < 8; i++) {
          const uint32_t b = __float_as_uint(v[i]);
          const float x = h8[i] * rstd.r, rest = __builtin_fmaf(x, w[i], -v[i]) + lower(i, x);
          if (b << (a.e5m2 ? 12 : 13) == 0 && v[i] != 0 && (rest > 0 || rest < 0)) v[i] = __uint_as_float((rest > 0) == (v[i] > 0) ? b + 1 : b - 1);
        }
      }
      const BlockScale s = block_scale<E8M0>(max16(abs_max8(v)), a.e5m2);
      if (c < n) {
        store_codes8(a.codes + row * a.ld, c, n, codes8(v, s.factor, a.e5m2));
        if ((t & 15) == 0) store_scale<E8M0>(a.scales, row * a.ld_scale + c / kBlk, s);
      }
    }
  };
  if constexpr (NV > 0) {
    V vx[NV], vr[NV];
    typename Vec8<W>::type vw[NV];
    f32x8 h[NV];
#pragma unroll
    for (int k = 0; k < NV; k++) {
      const uint32_t c = (k * NT + t) * 8;
      vx[k] = load8_raw<true>(x, c, n);
      if (res) vr[k] = load8_raw<true>(res, c, n);
    }
#pragma unroll
    for (int k = 0; k < NV; k++)
      if (a.weight) vw[k] = load8_raw((const W *)a.weight, (k * NT + t) * 8, n);
#pragma unroll
    for (int k = 0; k < NV; k++) {
      const uint32_t c = (k * NT + t) * 8;
      h[k] = add(vx[k], vr[k]);
      if (sum && c < n) store8(sum, c, n, h[k]);
      square(h[k]);
    }
    rstd = rstd_of(group_sum<NT>(acc, s_sum), a);
#pragma unroll
    for (int k = 0; k < NV; k++) {
      const uint32_t c = (k * NT + t) * 8;
      if ((c & ~(kBlk - 1)) < n) give(c, h[k], a.weight ? float8_of(vw[k]) : (f32x8){1, 1, 1, 1, 1, 1, 1, 1});
    }
  } else {
    auto take = [&](uint32_t c) {
      const V v = load8_raw(x, c, n);
      return add(v, res ? load8_raw(res, c, n) : v);
    };
    for (uint32_t c = t * 8; c < n; c += NT * 8) {
      const f32x8 h = take(c);
      if (sum) store8(sum, c, n, h);
      square(h);
    }
    rstd = rstd_of(group_sum<NT>(acc, s_sum), a);
    for (uint32_t c = t * 8; (c & ~(kBlk - 1)) < n; c += NT * 8) {
      f32x8 h = {0, 0, 0, 0, 0, 0, 0, 0};
      if (c < n) h = sum ? load8((const T *)sum, c, n) : take(c);
      give(c, h, weight8(c));
    }
  }
  if (a.rstd && t == 0) a.rstd[row] = rstd.out;
}

struct NormBwd {
  const void *dy, *dsum, *h, *weight;
  const float *rstd;
  void *dx;
  float *part;  // [work-groups][cols] sums of dy * xh over a work-group's rows, or null
  uint64_t ld_dy, ld_dsum, ld_h, ld_dx;
  uint64_t rows;
  uint32_t cols;
  float inv_cols;
};

// Rows blockIdx.x, blockIdx.x + gridDim.x, ... ; the next row is requested before this one's sums, and the columns' sums stay
// in registers from row to row.  NV = 0: rows of any length, read twice, their sums added up in the partial row in memory,
// which each thread alone touches at its columns.  16384 x 4096 bf16: 83.5 us, 6.4 TB/s; 395 x 5120: 6.9 us, two rows and a trip to
// memory for each.  NV = 0, 4096 x 12288 bf16: 267 us, 1.5 TB/s, as the partial row is read and written for every row.
template <typename T, typename W, int NT, int NV> __device__ __forceinline__ void norm_bwd_rows(const NormBwd &a, const uint64_t first, const uint64_t step_rows) {
  typedef typename Vec8<T>::type V;
  __shared__ float s_sum[2][NT / 64];
  const uint32_t t = threadIdx.x, n = a.cols;
  float *part = a.part ? a.part + first * n : nullptr;
  float acc = 0, rstd = 0;
  // one vector: xh, g, their product's share of the row's sum, and the weight gradient's share
  auto step = [&](V vdy, V vh, f32x8 w, f32x8 &xh, f32x8 &g, f32x8 &dw) {
#pragma unroll
    for (int i = 0; i < 8; i++) {
      const float dy = (float)vdy[i];
      xh[i] = (float)vh[i] * rstd;
      g[i] = dy * w[i];
      dw[i] = __builtin_fmaf(dy, xh[i], dw[i]);
      acc = __builtin_fmaf(g[i], xh[i], acc);
    }
  };
  auto give = [&](uint64_t row, uint32_t c, f32x8 xh, f32x8 g, f32x8 d, float m) {
#pragma unroll
    for (int i = 0; i < 8; i++) d[i] = __builtin_fmaf(rstd, __builtin_fmaf(-xh[i], m, g[i]), d[i]);
    store8((T *)a.dx + row * a.ld_dx, c, n, d);
  };
  const f32x8 zero = {0, 0, 0, 0, 0, 0, 0, 0}, one = {1, 1, 1, 1, 1, 1, 1, 1};
  int turn = 0;  // two sets of partial sums in turn: a wave writes the next row's while another still reads this one's
  if constexpr (NV > 0) {
    V vdy[NV], vh[NV], vds[NV];
    typename Vec8<W>::type vw[NV];
    f32x8 dw[NV];
    auto request = [&](uint64_t row) {
#pragma unroll
      for (int k = 0; k < NV; k++) {
        const uint32_t c = (k * NT + t) * 8;
        vdy[k] = load8_raw<true>((const T *)a.dy + row * a.ld_dy, c, n);
        vh[k] = load8_raw<true>((const T *)a.h + row * a.ld_h, c, n);
        if (a.dsum) vds[k] = load8_raw<true>((const T *)a.dsum + row * a.ld_dsum, c, n);
      }
    };
#pragma unroll
    for (int k = 0; k < NV; k++) {
      dw[k] = zero;
      if (a.weight) vw[k] = load8_raw((const W *)a.weight, (k * NT + t) * 8, n);
    }
    request(first);
    float next_rstd = a.rstd[first];
    for (uint64_t row = first; row < a.rows; row += step_rows, turn ^= 1) {
      f32x8 xh[NV], g[NV], d[NV];
      acc = 0;
      rstd = next_rstd;
#pragma unroll
      for (int k = 0; k < NV; k++) {
        step(vdy[k], vh[k], a.weight ? float8_of(vw[k]) : one, xh[k], g[k], dw[k]);
        d[k] = a.dsum ? float8_of(vds[k]) : zero;
      }
      if (row + step_rows < a.rows) {
        request(row + step_rows);
        next_rstd = a.rstd[row + step_rows];
      }
      const float m = group_sum<NT>(acc, s_sum[turn]) * a.inv_cols;
#pragma unroll
      for (int k = 0; k < NV; k++) {
        const uint32_t c = (k * NT + t) * 8;
        if (c < n) give(row, c, xh[k], g[k], d[k], m);
      }
    }
    if (part) {
#pragma unroll
      for (int k = 0; k < NV; k++) {
        const uint32_t c = (k * NT + t) * 8;
        if (c < n) store8(part, c, n, dw[k]);
      }
    }
  } else {
    for (uint64_t row = first; row < a.rows; row += step_rows, turn ^= 1) {
      const T *pdy = (const T *)a.dy + row * a.ld_dy, *ph = (const T *)a.h + row * a.ld_h;
      f32x8 xh, g;
      acc = 0;
      rstd = a.rstd[row];
      for (uint32_t c = t * 8; c < n; c += NT * 8) {
        f32x8 d = zero;
        step(load8_raw(pdy, c, n), load8_raw(ph, c, n), a.weight ? load8((const W *)a.weight, c, n) : one, xh, g, d);
        if (part) {
#pragma unroll
          for (int i = 0; i < 8; i++)
            if (c + i < n) part[c + i] = (row == first ? 0.0f : part[c + i]) + d[i];
        }
      }
      const float m = group_sum<NT>(acc, s_sum[turn]) * a.inv_cols;
      for (uint32_t c = t * 8; c < n; c += NT * 8) {
        f32x8 unused = zero;
        step(load8_raw(pdy, c, n), load8_raw(ph, c, n), a.weight ? load8((const W *)a.weight, c, n) : one, xh, g, unused);
        give(row, c, xh, g, a.dsum ? load8((const T *)a.dsum + row * a.ld_dsum, c, n) : zero, m);
      }
    }
  }
}

template <typename T, typename W, int NT, int NV> __global__ __launch_bounds__(NT) void k_norm_bwd(NormBwd a) {
  norm_bwd_rows<T, W, NT, NV>(a, blockIdx.x, gridDim.x);
}

// Both gradients at once for a moderate number of rows: the first work-groups take 64 columns each and read dy and h down
// them, eight lanes a row, the others a row each.  dx must be none of the memory that the first ones read.  395 x 5120 bf16:
// 5.9 us, 2.8 TB/s by the bytes of one reading: a launch and two trips to memory.
template <typename T, typename W, int NT, int NV> __global__ __launch_bounds__(NT) void k_norm_bwd_both(NormBwd a, float *__restrict__ dw, uint32_t n_dw) {
  if (blockIdx.x >= n_dw) {
    norm_bwd_rows<T, W, NT, NV>(a, blockIdx.x - n_dw, a.rows);
    return;
  }
  constexpr int AT_ONCE = 4;
  constexpr uint32_t step = NT / 8;
  __shared__ float s[NT / 64][64];
  const uint32_t t = threadIdx.x, c = blockIdx.x * 64 + (t & 7) * 8, n = a.cols;
  f32x8 v = {0, 0, 0, 0, 0, 0, 0, 0};
  for (uint64_t row = t >> 3; c < n && row < a.rows; row += AT_ONCE * step) {
    typename Vec8<T>::type dy[AT_ONCE], h[AT_ONCE];
    float rstd[AT_ONCE];
#pragma unroll
    for (int u = 0; u < AT_ONCE; u++) {
      const uint64_t r = row + u * step < a.rows ? row + u * step : row;
      dy[u] = load8_raw((const T *)a.dy + r * a.ld_dy, c, n);
      h[u] = load8_raw((const T *)a.h + r * a.ld_h, c, n);
      rstd[u] = a.rstd[r];
    }
#pragma unroll
    for (int u = 0; u < AT_ONCE; u++) {
      if (row + u * step >= a.rows) break;
#pragma unroll
      for (int i = 0; i < 8; i++) v[i] = __builtin_fmaf((float)dy[u][i], (float)h[u][i] * rstd[u], v[i]);
    }
  }
#pragma unroll
  for (int i = 0; i < 8; i++) {
#pragma unroll
    for (int d = 8; d < 64; d *= 2) v[i] += __shfl_xor(v[i], d);
    if ((t & 63) < 8) s[t >> 6][(t & 7) * 8 + i] = v[i];
  }
  __syncthreads();
  if (t < 64 && blockIdx.x * 64 + t < n) {
    float r = s[0][t];
#pragma unroll
    for (int w = 1; w < NT / 64; w++) r += s[w][t];
    dw[blockIdx.x * 64 + t] = r;
  }
}

// dw[c] = sum of the partial rows, in a fixed order: 32 columns a work-group, every 32nd partial row a half wave, eight of
// them requested at a time.  256 x 4096: 4.9 us, most of it launch and trips to memory.
constexpr int kDwWG = 1024;
__global__ __launch_bounds__(kDwWG) void k_norm_dw(const float *__restrict__ part, uint32_t n_part, uint32_t col0, uint32_t cols, float *__restrict__ dw) {
  __shared__ float s[kDwWG];
  const uint32_t t = threadIdx.x, c = col0 + blockIdx.x * 32 + (t & 31), first = t >> 5;
  constexpr uint32_t step = kDwWG / 32;
  float v = 0;
  if (c < cols) {
    for (uint32_t p = first; p < n_part; p += 8 * step) {
      float q[8];
#pragma unroll
      for (int k = 0; k < 8; k++) q[k] = p + k * step < n_part ? part[(uint64_t)(p + k * step) * cols + c] : 0.0f;
#pragma unroll
      for (int k = 0; k < 8; k++) v += q[k];
    }
  }
  s[t] = v;
  __syncthreads();
  if (t < 32 && c < cols) {
    float r = 0;
#pragma unroll
    for (uint32_t k = 0; k < step; k++) r += s[k * 32 + t];
    dw[c] = r;
  }
}

}  // namespace
