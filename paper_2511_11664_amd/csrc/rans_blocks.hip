// rans_blocks.hip -- block codes, norm and matrix product: host side and extern "C" entry points
//
// A translation unit of its own beside the codec's (rans_if.hip); the kernels are in rans_blocks.h and
// rans_norm.h, the product's in rans_matmul.h, which rans_matmul_narrow.hip and rans_matmul_wide.hip compile.  The same flags:
// no contraction by the compiler, fused multiply-adds are written out.

#include <hip/hip_runtime.h>
#include <hip/hip_fp16.h>

#include <cmath>
#include <cstring>
#include <type_traits>

#include "rans_if.h"

#include "rans_host.h"
#include "rans_common.h"
#include "rans_blocks.h"
#include "rans_norm.h"
#include "rans_matmul_launch.h"

namespace {

// Work goes to the device that the stream belongs to; the caller's current device is put back.
struct StreamDevice {
  int before = -1;
  bool ok = true, moved = false;
  explicit StreamDevice(hipStream_t st) {
    if (!st) return;
    int dev = -1;
    if (hipStreamGetDevice(st, &dev) != hipSuccess || hipGetDevice(&before) != hipSuccess) {
      ok = false;
      return;
    }
    if (dev != before) {
      moved = hipSetDevice(dev) == hipSuccess;
      ok = moved;
    }
  }
  ~StreamDevice() {
    if (moved) (void)hipSetDevice(before);
  }
};

inline size_t elem_bytes(uint32_t dtype) { return dtype == RANS_F32 ? 4 : 2; }

int check_blocks(const rans_blocks *b) {
  if (!b) return RANS_ERR_ARG;
  if (b->format > RANS_E5M2 || b->scale_type > RANS_SCALE_E8M0 || b->block > RANS_BLOCK_TILE || b->reserved) return RANS_ERR_ARG;
  if (b->rows > kBlkMaxDim || b->cols > kBlkMaxDim || b->ld > kBlkMaxLd || b->ld_scale > kBlkMaxLd) return RANS_ERR_ARG;
  if (b->ld < b->cols || b->ld_scale < (b->cols + kBlk - 1) / kBlk) return RANS_ERR_SHAPE;
  return RANS_OK;
}
int check_blocks_data(const rans_blocks *b, const void *codes, const void *scales) {
  const int rc = check_blocks(b);
  if (rc) return rc;
  if (b->rows && b->cols && (!codes || !scales)) return RANS_ERR_ARG;
  if (b->scale_type == RANS_SCALE_F32 && !aligned_to(scales, 4)) return RANS_ERR_ARG;
  return RANS_OK;
}

// Calls f with an element of the type that `dtype` names.
template <typename F> int by_dtype(uint32_t dtype, F f) {
  if (dtype == RANS_F32) return f((float)0);
  if (dtype == RANS_F16) return f((_Float16)0);
  return f((__bf16)0);
}
template <typename F> int by_bool(bool v, F f) { return v ? f(std::true_type{}) : f(std::false_type{}); }

constexpr uint64_t kQuantSliceUnits = 1ull << 28;  // blocks of a launch
constexpr uint64_t kQuantSliceRows = 65535ull * kBlk;

}  // namespace

extern "C" {

int rans_block_quantize(const void *d_x, uint64_t ld_x, uint32_t in_dtype, int transpose, uint8_t *d_code, void *d_scale,
                        const rans_blocks *out, void *stream) {
  int rc = check_blocks_data(out, d_code, d_scale);
  if (rc) return rc;
  if (in_dtype > RANS_BF16 || ld_x > kBlkMaxLd) return RANS_ERR_ARG;
  const uint64_t x_rows = transpose ? out->cols : out->rows, x_cols = transpose ? out->rows : out->cols;
  if (ld_x < x_cols) return RANS_ERR_SHAPE;
  if (!x_rows || !x_cols) return RANS_OK;
  const size_t eb = elem_bytes(in_dtype);
  if (!d_x || !aligned_to(d_x, eb)) return RANS_ERR_ARG;
  hipStream_t st = (hipStream_t)stream;
  const StreamDevice on(st);
  if (!on.ok) return RANS_ERR_HIP;
  const bool tile = out->block == RANS_BLOCK_TILE;
  return by_dtype(in_dtype, [&](auto elem) {
    typedef decltype(elem) T;
    return by_bool(out->scale_type == RANS_SCALE_E8M0, [&](auto e8m0_tag) -> int {
      constexpr bool E8M0 = decltype(e8m0_tag)::value;
      const T *x = (const T *)d_x;
      if (!transpose && !tile) {
        const uint64_t nb = (x_cols + kBlk - 1) / kBlk;
        const FastDivU32 by_nb = FastDivU32::of((uint32_t)nb);
        const uint64_t step = kQuantSliceUnits / nb;
        for (uint64_t r = 0; r < x_rows; r += step) {
          const uint64_t rows = x_rows - r < step ? x_rows - r : step, units = rows * nb;
          const uint32_t g = (uint32_t)((units + kWG / 16 * kQuantUnits - 1) / (kWG / 16 * kQuantUnits));
          PROF_LAUNCH(KID_BLOCK_QUANT, (k_block_quant<T, E8M0>), dim3(g), dim3(kWG), 0, st, x + r * ld_x, ld_x, d_code + r * out->ld, out->ld,
                      (void *)((uint8_t *)d_scale + r * out->ld_scale * (E8M0 ? 1 : 4)), out->ld_scale, (uint32_t)units, (uint32_t)x_cols,
                      (uint32_t)nb, by_nb, out->format);
          LAUNCH_CHECK();
        }
        return RANS_OK;
      }
      for (uint64_t r = 0; r < x_rows; r += kQuantSliceRows) {
        const uint64_t rows = x_rows - r < kQuantSliceRows ? x_rows - r : kQuantSliceRows;
        const dim3 grid((uint32_t)((x_cols + kBlk - 1) / kBlk), (uint32_t)((rows + kBlk - 1) / kBlk));
        // a slice of x's rows is a slice of the result's columns where it is transposed
        uint8_t *codes = d_code + (transpose ? r : r * out->ld);
        uint8_t *scales = (uint8_t *)d_scale + (transpose ? r / kBlk : r / kBlk * out->ld_scale) * (E8M0 ? 1 : 4);
#define TILE_LAUNCH(TRANS, TILE)                                                                                                   \
  PROF_LAUNCH(KID_BLOCK_QUANT_TILE, (k_block_quant_tile<T, E8M0, TRANS, TILE>), grid, dim3(kWG), 0, st, x + r * ld_x, ld_x, (uint32_t)rows, \
              (uint32_t)x_cols, codes, out->ld, (void *)scales, out->ld_scale, out->format)
        if (!transpose) TILE_LAUNCH(false, true);
        else if (tile) TILE_LAUNCH(true, true);
        else TILE_LAUNCH(true, false);
#undef TILE_LAUNCH
        LAUNCH_CHECK();
      }
      return RANS_OK;
    });
  });
}

int rans_block_dequantize(const uint8_t *d_code, const void *d_scale, const rans_blocks *in, uint32_t out_dtype, void *d_x_out,
                          uint64_t ld_x, void *stream) {
  int rc = check_blocks_data(in, d_code, d_scale);
  if (rc) return rc;
  if (out_dtype > RANS_BF16 || ld_x > kBlkMaxLd) return RANS_ERR_ARG;
  if (ld_x < in->cols) return RANS_ERR_SHAPE;
  if (!in->rows || !in->cols) return RANS_OK;
  const size_t eb = elem_bytes(out_dtype);
  if (!d_x_out || !aligned_to(d_x_out, eb)) return RANS_ERR_ARG;
  hipStream_t st = (hipStream_t)stream;
  const StreamDevice on(st);
  if (!on.ok) return RANS_ERR_HIP;
  const uint32_t tile = in->block == RANS_BLOCK_TILE;
  return by_dtype(out_dtype, [&](auto elem) {
    typedef decltype(elem) T;
    return by_bool(in->scale_type == RANS_SCALE_E8M0, [&](auto e8m0_tag) -> int {
      constexpr bool E8M0 = decltype(e8m0_tag)::value;
      const uint64_t nb = (in->cols + kBlk - 1) / kBlk;
      const FastDivU32 by_nb = FastDivU32::of((uint32_t)nb);
      const uint64_t step = kQuantSliceUnits / nb;
      for (uint64_t r = 0; r < in->rows; r += step) {
        const uint64_t rows = in->rows - r < step ? in->rows - r : step, units = rows * nb;
        const uint32_t g = (uint32_t)((units + kWG / 16 * kQuantUnits - 1) / (kWG / 16 * kQuantUnits));
        const uint64_t srow = tile ? r / kBlk : r;
        PROF_LAUNCH(KID_BLOCK_DEQUANT, (k_block_dequant<T, E8M0>), dim3(g), dim3(kWG), 0, st, d_code + r * in->ld, in->ld,
                    (const void *)((const uint8_t *)d_scale + srow * in->ld_scale * (E8M0 ? 1 : 4)), in->ld_scale, (T *)d_x_out + r * ld_x, ld_x,
                    (uint32_t)units, (uint32_t)in->cols, (uint32_t)nb, by_nb, tile, (uint32_t)(r % kBlk), in->format);
        LAUNCH_CHECK();
      }
      return RANS_OK;
    });
  });
}

}  // extern "C"

// ------------------------------------------------------------------ norm

namespace {

int check_norm(const rans_norm_params *p) {
  if (!p) return RANS_ERR_ARG;
  if (p->dtype > RANS_BF16 || p->weight_dtype > RANS_BF16 || p->reserved) return RANS_ERR_ARG;
  if (p->rows > kBlkMaxDim || p->cols < 1 || p->cols > kBlkMaxDim || !(p->eps >= 0) || !std::isfinite(p->eps)) return RANS_ERR_ARG;
  const uint64_t lds[4] = {p->ld_x, p->ld_res, p->ld_sum, p->ld_y};
  for (uint64_t ld : lds) {
    if (ld > kBlkMaxLd) return RANS_ERR_ARG;
    if (ld < p->cols) return RANS_ERR_SHAPE;
  }
  return RANS_OK;
}

constexpr uint32_t kNormSliceRows = 1u << 21;  // rows of a launch, whose threads stay below 2^32
constexpr uint64_t kNormSliceCols = 1u << 26;  // columns of a launch of the weight gradient's sum

// The work-group that a row takes: f(threads, eights a thread); 0 eights: any length.
template <int NT, int NV, typename F> int with_row(F f) { return f(std::integral_constant<int, NT>{}, std::integral_constant<int, NV>{}); }

// Forward.  Few rows are quicker with more threads on each, many with more in flight for each thread.  Twice the threads / two
// vectors a thread, kernel us, bf16: 4096 columns 8 rows 4.4 / 4.8, 512 5.8 / 5.7, 1024 9.3 / 9.4, 2048 14.1 / 13.6, 4096 22.7 /
// 21.7, 16384 77 / 73; 5120 columns 128 rows 5.0 / 5.3, 1024 12.5 / 11.3, 2048 19.6 / 17.8, 16384 126 / 103.  binary32, 4096 columns:
// 512 rows 8.2 / 9.4, 2048 22.9 / 23.5, 16384 170 / 172; 2500 columns 1024 rows 11.0 / 11.6, 2048 19.0 / 17.9, 16384 137 / 122.
template <typename F> int by_row_forward(const rans_norm_params &p, F f) {
  const bool many = p.rows >= 2048;
  if (p.cols <= 64 * 8) return with_row<64, 1>(f);
  if (p.cols <= 256 * 8) return with_row<256, 1>(f);
  if (p.cols <= 512 * 8) return many ? with_row<256, 2>(f) : with_row<512, 1>(f);
  if (p.cols <= 1024 * 8) return many ? with_row<512, 2>(f) : with_row<1024, 1>(f);
  return with_row<512, 0>(f);
}

// Backward, and its work-groups, which are the rows of partial sums too: one or two on a compute unit, since the next row's
// loads are under way anyway and each partial row is written and read again; no more than take the same number of rows each.
// 16384 x 4096 with 256 / 512 of them 85.5 / 88.3 us; 16384 x 2048 (256 threads each) 59.7 / 45.6; 395 x 5120 with 198 /
// 256 / 395 of them 9.3 / 9.8 / 11.4, and with 1024 threads each instead of 640 10.1 / 10.5 / 13.6.
template <typename F> int by_row_backward(const rans_norm_params &p, F f) {
  if (p.cols <= 64 * 8) return with_row<64, 1>(f);
  if (p.cols <= 256 * 8) return with_row<256, 1>(f);
  if (p.cols <= 512 * 8) return with_row<512, 1>(f);
  if (p.cols <= 640 * 8) return with_row<640, 1>(f);
  if (p.cols <= 1024 * 8) return with_row<1024, 1>(f);
  return with_row<512, 0>(f);
}
uint32_t norm_parts(const rans_norm_params &p) {
  const uint32_t most = p.cols <= 64 * 8 ? 2048 : p.cols <= 256 * 8 ? 512 : 256;
  if (p.rows <= most) return (uint32_t)p.rows;
  const uint64_t each = (p.rows + most - 1) / most;
  return (uint32_t)((p.rows + each - 1) / each);
}

// Both gradients from one kernel, dy and h read twice, or partial rows and a second kernel to add them up: one for as many rows as
// stay in the caches and keep the columns' work-groups short.  One / two kernels, us: 8 x 4096 3.2 / 5.5, 395 x 1024 5.5 / 7.1, 395 x
// 5120 5.9 / 9.2, 1024 x 4096 9.8 / 11.7; 2048 x 4096 28.3 / 16.8, 1024 x 512 24.8 / 8.0.
bool norm_both(const rans_norm_params &p, uint32_t threads) { return p.rows <= 2 * threads && p.rows * p.cols <= 1u << 22; }

// Whether two matrices of the same shape have memory in common.
bool overlap(const void *a, uint64_t ld_a, const void *b, uint64_t ld_b, uint64_t rows, uint64_t cols, size_t eb) {
  const uintptr_t pa = (uintptr_t)a, pb = (uintptr_t)b;
  return pa < pb + ((rows - 1) * ld_b + cols) * eb && pb < pa + ((rows - 1) * ld_a + cols) * eb;
}

}  // namespace

extern "C" {

int rans_norm_quantize(const void *d_x, const void *d_res, const void *d_weight, const rans_norm_params *p, void *d_sum, float *d_rstd,
                       void *d_y, uint8_t *d_code, void *d_scale, const rans_blocks *out, void *stream) {
  int rc = check_norm(p);
  if (rc) return rc;
  if (d_code) {
    rc = check_blocks_data(out, d_code, d_scale);
    if (rc) return rc;
    if (out->block != RANS_BLOCK_ROW) return RANS_ERR_ARG;
    if (out->rows != p->rows || out->cols != p->cols) return RANS_ERR_SHAPE;
  }
  if (!p->rows) return RANS_OK;
  const size_t eb = elem_bytes(p->dtype), wb = elem_bytes(p->weight_dtype);
  if (!d_x || (!d_sum && !d_y && !d_code && !d_rstd)) return RANS_ERR_ARG;
  if (!aligned_to(d_x, eb) || !aligned_to(d_res, eb) || !aligned_to(d_sum, eb) || !aligned_to(d_y, eb) || !aligned_to(d_weight, wb) ||
      !aligned_to(d_rstd, 4))
    return RANS_ERR_ARG;
  hipStream_t st = (hipStream_t)stream;
  const StreamDevice on(st);
  if (!on.ok) return RANS_ERR_HIP;
  NormFwd a{};
  a.x = d_x, a.res = d_res, a.weight = d_weight, a.sum = d_sum, a.y = d_y, a.rstd = d_rstd, a.codes = d_code, a.scales = d_scale;
  a.ld_x = p->ld_x, a.ld_res = p->ld_res, a.ld_sum = p->ld_sum, a.ld_y = p->ld_y;
  a.cols = (uint32_t)p->cols, a.eps = p->eps, a.inv_cols = 1.0 / (double)p->cols;
  if (d_code) {
    a.ld = out->ld, a.ld_scale = out->ld_scale, a.e5m2 = out->format;
  }
  return by_dtype(p->dtype, [&](auto elem) {
    typedef decltype(elem) T;
    return by_bool(p->weight_dtype == p->dtype, [&](auto same_tag) {
      // a weight of another type than the stream's is binary32, or is refused below
      typedef typename std::conditional<decltype(same_tag)::value, T, float>::type W;
      if (!decltype(same_tag)::value && p->weight_dtype != RANS_F32) return (int)RANS_ERR_ARG;
      return by_bool(d_code && out->scale_type == RANS_SCALE_E8M0, [&](auto e8m0_tag) {
        constexpr bool E8M0 = decltype(e8m0_tag)::value;
        return by_row_forward(*p, [&](auto nt_tag, auto nv_tag) -> int {
          constexpr int NT = decltype(nt_tag)::value, NV = decltype(nv_tag)::value;
          for (uint64_t r = 0; r < p->rows; r += kNormSliceRows) {
            const uint32_t g = (uint32_t)(p->rows - r < kNormSliceRows ? p->rows - r : kNormSliceRows);
            PROF_LAUNCH(KID_NORM_QUANT, (k_norm_quant<T, W, E8M0, NT, NV>), dim3(g), dim3(NT), 0, st, a, r);
            LAUNCH_CHECK();
          }
          return RANS_OK;
        });
      });
    });
  });
}

int rans_norm_workspace_bytes(const rans_norm_params *p, size_t *ws_bytes) {
  const int rc = check_norm(p);
  if (rc) return rc;
  if (!ws_bytes) return RANS_ERR_ARG;
  *ws_bytes = align_up((size_t)norm_parts(*p) * p->cols * 4, 256);
  return RANS_OK;
}

int rans_norm_backward(const void *d_dy, const void *d_dsum, const void *d_sum, const void *d_weight, const float *d_rstd,
                       const rans_norm_params *p, void *d_dx, float *d_dweight, void *d_ws, size_t ws_bytes, void *stream) {
  int rc = check_norm(p);
  if (rc) return rc;
  const size_t eb = elem_bytes(p->dtype), wb = elem_bytes(p->weight_dtype);
  if (p->rows && (!d_dy || !d_sum || !d_rstd || !d_dx)) return RANS_ERR_ARG;
  if (!aligned_to(d_dy, eb) || !aligned_to(d_dsum, eb) || !aligned_to(d_sum, eb) || !aligned_to(d_dx, eb) || !aligned_to(d_weight, wb) ||
      !aligned_to(d_rstd, 4) || !aligned_to(d_dweight, 4))
    return RANS_ERR_ARG;
  if (p->weight_dtype != p->dtype && p->weight_dtype != RANS_F32) return RANS_ERR_ARG;
  if (d_dweight && p->rows) {
    if (!d_ws || !aligned_to(d_ws, 256)) return RANS_ERR_ARG;
    size_t need = 0;
    rans_norm_workspace_bytes(p, &need);
    if (ws_bytes < need) return RANS_ERR_WORKSPACE;
  }
  hipStream_t st = (hipStream_t)stream;
  const StreamDevice on(st);
  if (!on.ok) return RANS_ERR_HIP;
  NormBwd a{};
  a.dy = d_dy, a.dsum = d_dsum, a.h = d_sum, a.weight = d_weight, a.rstd = d_rstd, a.dx = d_dx;
  a.part = d_dweight ? (float *)d_ws : nullptr;
  a.ld_dy = p->ld_y, a.ld_dsum = p->ld_res, a.ld_h = p->ld_sum, a.ld_dx = p->ld_x;
  a.rows = p->rows, a.cols = (uint32_t)p->cols, a.inv_cols = 1.0f / (float)p->cols;
  const uint32_t g = norm_parts(*p);
  bool both = d_dweight && p->rows && !overlap(d_dx, p->ld_x, d_dy, p->ld_y, p->rows, p->cols, eb) &&
              !overlap(d_dx, p->ld_x, d_sum, p->ld_sum, p->rows, p->cols, eb);
  if (g) {
    rc = by_dtype(p->dtype, [&](auto elem) {
      typedef decltype(elem) T;
      return by_bool(p->weight_dtype == p->dtype, [&](auto same_tag) {
        typedef typename std::conditional<decltype(same_tag)::value, T, float>::type W;
        return by_row_backward(*p, [&](auto nt_tag, auto nv_tag) -> int {
          constexpr int NT = decltype(nt_tag)::value, NV = decltype(nv_tag)::value;
          both = both && norm_both(*p, NT);
          if (both) {
            const uint32_t n_dw = (uint32_t)((p->cols + 63) / 64);
            a.part = nullptr;
            PROF_LAUNCH(KID_NORM_BWD_BOTH, (k_norm_bwd_both<T, W, NT, NV>), dim3(n_dw + (uint32_t)p->rows), dim3(NT), 0, st, a, d_dweight, n_dw);
          } else {
            PROF_LAUNCH(KID_NORM_BWD, (k_norm_bwd<T, W, NT, NV>), dim3(g), dim3(NT), 0, st, a);
          }
          LAUNCH_CHECK();
          return RANS_OK;
        });
      });
    });
    if (rc) return rc;
  }
  for (uint64_t c = 0; d_dweight && !both && c < p->cols; c += kNormSliceCols) {
    const uint64_t n = p->cols - c < kNormSliceCols ? p->cols - c : kNormSliceCols;
    PROF_LAUNCH(KID_NORM_DW, k_norm_dw, dim3((uint32_t)((n + 31) / 32)), dim3(kDwWG), 0, st, (const float *)d_ws, g, (uint32_t)c, (uint32_t)p->cols,
                d_dweight);
    LAUNCH_CHECK();
  }
  return RANS_OK;
}

}  // extern "C"

// ------------------------------------------------------------------ matrix product

namespace {

int check_matmul(const rans_blocks *a, const rans_blocks *b) {
  int rc = check_blocks(a);
  if (rc) return rc;
  rc = check_blocks(b);
  if (rc) return rc;
  if (a->block != RANS_BLOCK_ROW || a->scale_type != b->scale_type) return RANS_ERR_ARG;
  if (a->cols != b->cols) return RANS_ERR_SHAPE;
  return RANS_OK;
}

constexpr uint64_t kMatmulSlice = 1u << 17;  // rows of A and of B in a launch: 2^22 of the smallest tiles; whole tiles of scales

// Enough for each of the launches, which follow one another: whether K goes in parts is decided for a launch's own rows, and
// the last rows of a long matrix may have few enough tiles where the ones before had not.
size_t matmul_ws_bytes(const rans_blocks *a, const rans_blocks *b, uint32_t units) {
  uint64_t need = 0;
  for (uint64_t m : {a->rows < kMatmulSlice ? a->rows : kMatmulSlice, a->rows % kMatmulSlice})
    for (uint64_t n : {b->rows < kMatmulSlice ? b->rows : kMatmulSlice, b->rows % kMatmulSlice}) {
      const uint64_t bytes = matmul_part_bytes(matmul_parts(m, n, a->cols, units), m, n);
      need = bytes > need ? bytes : need;
    }
  return align_up((size_t)need, 256);
}
inline uint32_t matmul_units() {
  const uint32_t units = compute_units();
  return units ? units : 256;
}

}  // namespace

extern "C" {

int rans_matmul_workspace_bytes(const rans_blocks *a, const rans_blocks *b, size_t *ws_bytes) {
  const int rc = check_matmul(a, b);
  if (rc) return rc;
  if (!ws_bytes) return RANS_ERR_ARG;
  *ws_bytes = matmul_ws_bytes(a, b, matmul_units());
  return RANS_OK;
}

int rans_block_matmul(const uint8_t *d_a, const void *d_a_scale, const rans_blocks *a, const uint8_t *d_b, const void *d_b_scale,
                      const rans_blocks *b, uint32_t out_dtype, void *d_c, uint64_t ld_c, void *d_ws, size_t ws_bytes, void *stream) {
  int rc = check_matmul(a, b);
  if (rc) return rc;
  rc = check_blocks_data(a, d_a, d_a_scale);
  if (rc) return rc;
  rc = check_blocks_data(b, d_b, d_b_scale);
  if (rc) return rc;
  if (out_dtype > RANS_BF16 || ld_c > kBlkMaxLd) return RANS_ERR_ARG;
  if (ld_c < b->rows) return RANS_ERR_SHAPE;
  if (!a->rows || !b->rows) return RANS_OK;
  const size_t eb = elem_bytes(out_dtype);
  if (!d_c || !aligned_to(d_c, eb)) return RANS_ERR_ARG;
  hipStream_t st = (hipStream_t)stream;
  const StreamDevice on(st);
  if (!on.ok) return RANS_ERR_HIP;
  const uint32_t units = matmul_units();
  const size_t need = matmul_ws_bytes(a, b, units);
  if (need && (!d_ws || !aligned_to(d_ws, 256))) return RANS_ERR_ARG;
  if (ws_bytes < need) return RANS_ERR_WORKSPACE;
  const int fmt = (a->format == RANS_E5M2 ? 2 : 0) + (b->format == RANS_E5M2 ? 1 : 0);
  const uint64_t sb = a->scale_type == RANS_SCALE_E8M0 ? 1 : 4;
  for (uint64_t m = 0; m < a->rows; m += kMatmulSlice)
    for (uint64_t n = 0; n < b->rows; n += kMatmulSlice) {
      const uint64_t nm = a->rows - m < kMatmulSlice ? a->rows - m : kMatmulSlice, nn = b->rows - n < kMatmulSlice ? b->rows - n : kMatmulSlice;
      MatmulArgs p{};
      p.a = d_a + m * a->ld, p.lda = a->ld, p.sa = (const uint8_t *)d_a_scale + m * a->ld_scale * sb, p.ldsa = a->ld_scale;
      p.b = d_b + n * b->ld, p.ldb = b->ld, p.ldsb = b->ld_scale;
      p.sb = (const uint8_t *)d_b_scale + (b->block == RANS_BLOCK_TILE ? n / kBlk : n) * b->ld_scale * sb;
      p.c = (uint8_t *)d_c + (m * ld_c + n) * eb, p.ldc = ld_c;
      p.m = (uint32_t)nm, p.n = (uint32_t)nn, p.k = (uint32_t)a->cols;
      p.e8m0 = a->scale_type == RANS_SCALE_E8M0, p.b_tile = b->block == RANS_BLOCK_TILE, p.out = out_dtype;
      const MatmulParts parts = matmul_parts(nm, nn, a->cols, units);
      rc = out_dtype == RANS_F32 ? launch_matmul_wide(p, fmt, parts, d_ws, st) : launch_matmul_narrow(p, fmt, parts, d_ws, st);
      if (rc) return rc;
    }
  return RANS_OK;
}

}  // extern "C"
