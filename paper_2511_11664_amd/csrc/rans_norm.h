// rans_norm.h -- root-mean-square norm with the residual's addition and an output in 8 bits; its gradients
//
// Part of the translation unit rans_blocks.hip; not a stand-alone header.
//
// Forward, a row of K elements:  h = x + residual, rounded to the stream's type, because that is what the next residual
// addition and the backward pass read;  rstd = 1 / sqrt(sum h^2 / K + eps);  y = h * rstd * w in binary32;  codes and scales
// of y by the row blocks of rans_blocks.h, and / or y itself rounded once.
// Backward:  g = dy * w, xh = h * rstd;  dx = rstd * (g - xh * sum(g * xh) / K) + dsum;  dw = sum over rows of dy * xh.
// All sums are binary32: a lane's own eight neighbours (and every further eight), then the lanes of a wave, then the waves.
//
// Bound by memory: each tensor is read once and written once, a row lives in registers between its sum and its output.
#pragma once

namespace {

// Sum over a work-group of NT threads, in every thread.  `s`: NT / 64 floats per value; two values at most.
template <int NT> __device__ inline float wave_sum(float v) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d);
  return v;
}
template <int NT> __device__ inline float group_sum(float v, float *s) {
  v = wave_sum<NT>(v);
  if (NT == 64) return v;
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
  __syncthreads();
  float r = 0;
#pragma unroll
  for (int w = 0; w < NT / 64; w++) r += s[w];
  return r;
}

template <typename W> __device__ inline f32x8 load_weight8(const W *w, uint32_t c, uint32_t n, bool vec) {
  if (!w) return (f32x8){1, 1, 1, 1, 1, 1, 1, 1};
  return load8(w, c, n, vec);
}

struct NormFwd {
  const void *x, *res, *weight;
  void *sum, *y;
  float *rstd;
  uint8_t *codes;
  void *scales;
  uint64_t ld_x, ld_res, ld_sum, ld_y, ld, ld_scale;
  uint32_t cols, e5m2;
  float eps, inv_cols;
  int vec, vec_w, vec_c;  // every row of the streams / the weight / the codes may be taken 16 (codes: 8) bytes at a time
};

// A row per work-group of NT threads, NV times eight neighbouring elements a thread (NV = 0: any length, h read again).
template <typename T, typename W, bool E8M0, int NT, int NV>
__global__ __launch_bounds__(NT) void k_norm_quant(NormFwd a, uint64_t row0) {
  __shared__ float s_sum[NT / 64];
  const uint64_t row = row0 + blockIdx.x;
  const uint32_t t = threadIdx.x, n = a.cols;
  const T *x = (const T *)a.x + row * a.ld_x;
  const T *res = a.res ? (const T *)a.res + row * a.ld_res : nullptr;
  T *sum = a.sum ? (T *)a.sum + row * a.ld_sum : nullptr;
  constexpr int NR = NV ? NV : 1;
  f32x8 h[NR];
  float acc = 0;
  auto take = [&](uint32_t c) {
    f32x8 v = load8(x, c, n, a.vec);
    if (res) {
      const f32x8 r = load8(res, c, n, a.vec);
#pragma unroll
      for (int i = 0; i < 8; i++) v[i] = (float)(T)(v[i] + r[i]);
    }
    return v;
  };
  if (NV) {
#pragma unroll
    for (int k = 0; k < NR; k++) {
      const uint32_t c = (k * NT + t) * 8;
      h[k] = c < n ? take(c) : (f32x8){0, 0, 0, 0, 0, 0, 0, 0};
    }
#pragma unroll
    for (int k = 0; k < NR; k++) {
      const uint32_t c = (k * NT + t) * 8;
      if (sum && c < n) store8(sum, c, n, a.vec, h[k]);
#pragma unroll
      for (int i = 0; i < 8; i++) acc = __builtin_fmaf(h[k][i], h[k][i], acc);
    }
  } else {
    for (uint32_t c = t * 8; c < n; c += NT * 8) {
      const f32x8 v = take(c);
      if (sum) store8(sum, c, n, a.vec, v);
#pragma unroll
      for (int i = 0; i < 8; i++) acc = __builtin_fmaf(v[i], v[i], acc);
    }
  }
  const float rstd = 1.0f / sqrtf(group_sum<NT>(acc, s_sum) * a.inv_cols + a.eps);
  if (a.rstd && t == 0) a.rstd[row] = rstd;
  auto give = [&](uint32_t c, f32x8 v) {
    // 16 lanes hold a block; lanes behind the row's end hold zeros and take part in its maximum
    const f32x8 w = load_weight8((const W *)a.weight, c, n, a.vec_w);
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] = v[i] * rstd * w[i];
    if (a.y && c < n) store8((T *)a.y + row * a.ld_y, c, n, a.vec, v);
    if (a.codes) {
      const BlockScale s = block_scale<E8M0>(max16(abs_max8(v)), a.e5m2);
      if (c < n) {
        store_codes8(a.codes + row * a.ld, c, n, a.vec_c, codes8(v, s.factor, a.e5m2));
        if ((t & 15) == 0) store_scale<E8M0>(a.scales, row * a.ld_scale + c / kBlk, s);
      }
    }
  };
  if (NV) {
#pragma unroll
    for (int k = 0; k < NR; k++) {
      const uint32_t c = (k * NT + t) * 8;
      if ((c & ~(kBlk - 1)) < n) give(c, h[k]);
    }
  } else {
    for (uint32_t c = t * 8; (c & ~(kBlk - 1)) < n; c += NT * 8) {
      f32x8 v = {0, 0, 0, 0, 0, 0, 0, 0};
      if (c < n) v = sum ? load8((const T *)sum, c, n, a.vec) : take(c);
      give(c, v);
    }
  }
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
  int vec, vec_w;
};

// Rows blockIdx.x, blockIdx.x + gridDim.x, ... ; the columns' sums stay in registers from row to row.  NV = 0: rows of any
// length, read twice, their sums added up in the partial row in memory, which each thread alone touches at its columns.
template <typename T, typename W, int NT, int NV>
__global__ __launch_bounds__(NT) void k_norm_bwd(NormBwd a) {
  __shared__ float s_sum[2][NT / 64];
  const uint32_t t = threadIdx.x, n = a.cols;
  constexpr int NR = NV ? NV : 1;
  f32x8 dw[NR], w[NR];
#pragma unroll
  for (int k = 0; k < NR; k++) {
    dw[k] = (f32x8){0, 0, 0, 0, 0, 0, 0, 0};
    const uint32_t c = (k * NT + t) * 8;
    if (NV && c < n) w[k] = load_weight8((const W *)a.weight, c, n, a.vec_w);
  }
  float *part = a.part ? a.part + (uint64_t)blockIdx.x * n : nullptr;
  int turn = 0;
  for (uint64_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
    const T *pdy = (const T *)a.dy + row * a.ld_dy, *ph = (const T *)a.h + row * a.ld_h;
    const T *pds = a.dsum ? (const T *)a.dsum + row * a.ld_dsum : nullptr;
    T *pdx = (T *)a.dx + row * a.ld_dx;
    const float rstd = a.rstd[row];
    float acc = 0;
    f32x8 xh[NR], g[NR];
    auto step = [&](uint32_t c, f32x8 wv, f32x8 &xhv, f32x8 &gv, f32x8 &dwv) {
      const f32x8 dy = load8(pdy, c, n, a.vec), h = load8(ph, c, n, a.vec);
#pragma unroll
      for (int i = 0; i < 8; i++) {
        xhv[i] = h[i] * rstd;
        gv[i] = dy[i] * wv[i];
        dwv[i] = __builtin_fmaf(dy[i], xhv[i], dwv[i]);
        acc = __builtin_fmaf(gv[i], xhv[i], acc);
      }
    };
    auto give = [&](uint32_t c, f32x8 xhv, f32x8 gv, float m) {
      f32x8 d = {0, 0, 0, 0, 0, 0, 0, 0};
      if (pds) d = load8(pds, c, n, a.vec);
#pragma unroll
      for (int i = 0; i < 8; i++) d[i] = __builtin_fmaf(rstd, __builtin_fmaf(-xhv[i], m, gv[i]), d[i]);
      store8(pdx, c, n, a.vec, d);
    };
    if (NV) {
#pragma unroll
      for (int k = 0; k < NR; k++) {
        const uint32_t c = (k * NT + t) * 8;
        if (c < n) step(c, w[k], xh[k], g[k], dw[k]);
      }
    } else {
      for (uint32_t c = t * 8; c < n; c += NT * 8) {
        f32x8 d = {0, 0, 0, 0, 0, 0, 0, 0}, xv, gv;
        step(c, load_weight8((const W *)a.weight, c, n, a.vec_w), xv, gv, d);
        if (part) {
#pragma unroll
          for (int i = 0; i < 8; i++)
            if (c + i < n) part[c + i] = (row == blockIdx.x ? 0.0f : part[c + i]) + d[i];
        }
      }
    }
    // two sets of partial sums in turn: a wave writes the next row's while another still reads this one's
    const float m = group_sum<NT>(acc, s_sum[turn]) * a.inv_cols;
    if (NV) {
#pragma unroll
      for (int k = 0; k < NR; k++) {
        const uint32_t c = (k * NT + t) * 8;
        if (c < n) give(c, xh[k], g[k], m);
      }
    } else {
      for (uint32_t c = t * 8; c < n; c += NT * 8) {
        f32x8 xv, gv, d;
        const f32x8 wv = load_weight8((const W *)a.weight, c, n, a.vec_w), dy = load8(pdy, c, n, a.vec), h = load8(ph, c, n, a.vec);
        (void)d;
#pragma unroll
        for (int i = 0; i < 8; i++) xv[i] = h[i] * rstd, gv[i] = dy[i] * wv[i];
        give(c, xv, gv, m);
      }
    }
  }
  if (NV && part) {
#pragma unroll
    for (int k = 0; k < NR; k++) {
      const uint32_t c = (k * NT + t) * 8;
#pragma unroll
      for (int i = 0; i < 8; i++)
        if (c + i < n) part[c + i] = dw[k][i];
    }
  }
}

// dw[c] = sum of the partial rows, in a fixed order: 64 columns a work-group, a quarter of the rows a wave.
__global__ __launch_bounds__(kWG) void k_norm_dw(const float *__restrict__ part, uint32_t n_part, uint32_t cols, float *__restrict__ dw) {
  __shared__ float s[kWG];
  const uint32_t t = threadIdx.x, c = blockIdx.x * 64 + (t & 63);
  float v = 0;
  if (c < cols)
    for (uint32_t p = t >> 6; p < n_part; p += kWG / 64) v += part[(uint64_t)p * cols + c];
  s[t] = v;
  __syncthreads();
  if (t < 64 && c < cols) dw[c] = (s[t] + s[t + 64]) + (s[t + 128] + s[t + 192]);
}

}  // namespace
