// rans_host.h -- what the host sides of all translation units share: the per-kernel timing aid and launch checks
#pragma once

#include <hip/hip_runtime.h>
#include <hip/hip_ext.h>

#include <cstddef>
#include <cstdint>
#include <atomic>
#include <mutex>
#include <vector>

#include "rans_if.h"

#pragma GCC visibility push(hidden)

// ------------------------------------------------------------------ instrumentation

// Optional per-kernel timing for benchmarks: when a kernel's bit is set in the
// mask, each of its launches is bracketed by a pair of HIP events recorded on the
// launch stream.  Off by default; the normal path records nothing.
enum KernelId {
  KID_MINMAX = 0, KID_QINFO, KID_QUANT_HIST, KID_SCAN, KID_CSR_COMPACT, KID_CSR_ROWS,
  KID_NORMALIZE, KID_ENCODE, KID_CHUNK_SCAN, KID_GATHER, KID_DEC_PREPARE, KID_DECODE, KID_ROW_SCAN,
  KID_CSR_EXPAND, KID_DEQUANT, KID_RS_MASK, KID_RS_COUNT, KID_RS_COST,
  KID_ENCODE_FEED, KID_DECODE_LEAN, KID_BLOCK_QUANT, KID_BLOCK_QUANT_TILE, KID_BLOCK_DEQUANT, KID_NORM_QUANT, KID_NORM_BWD,
  KID_NORM_DW, KID_BLOCK_MATMUL, KID_BLOCK_MATMUL_FEW, KID_BLOCK_MATMUL_ANY,
  KID_BLOCK_MATMUL_SUM, KID_NORM_BWD_BOTH,
  KID_BLOCK_MATMUL_128, KID_BLOCK_MATMUL_DEEP, KID_BLOCK_MATMUL_256, KID_BLOCK_MATMUL_ANY_128,  // larger tiles than the name alone: 64 x 64
  KID_COUNT
};
inline const char *const kKernelNames[KID_COUNT] = {
    "k_minmax", "k_qinfo", "k_quant_hist", "k_scan_u32", "k_csr_compact", "k_csr_rows",
    "k_normalize", "k_encode", "k_chunk_scan", "k_gather", "k_dec_prepare", "k_decode", "k_row_part",
    "k_csr_to_dense", "k_dequant", "k_rs_mask", "k_rs_count", "k_rs_cost",
    "k_encode_feed", "k_decode_lean", "k_block_quant", "k_block_quant_tile", "k_block_dequant", "k_norm_quant", "k_norm_bwd",
    "k_norm_dw", "k_block_matmul", "k_block_matmul_few", "k_block_matmul_any",
    "k_block_matmul_sum", "k_norm_bwd_both",
    "k_block_matmul_128", "k_block_matmul_deep", "k_block_matmul_256", "k_block_matmul_any_128"};

struct ProfRecord {
  int kid;
  hipEvent_t a, b;
};
struct Profiler {
  uint64_t mask = 0;
  uint32_t every = 1;                 // bracket every n-th launch of an enabled kernel
  uint32_t seen[KID_COUNT] = {0};     // launches seen per kernel id since the last enable
  std::vector<ProfRecord> recs;   // records in use
  std::vector<ProfRecord> pool;   // event pairs ready for reuse
  std::mutex mu;
};
inline Profiler g_prof;  // one for the library

// Takes an event pair for launch `kid` if that launch is to be timed.
inline bool prof_take(int kid, ProfRecord *r) {
  if (!((g_prof.mask >> kid) & 1)) return false;
  std::lock_guard<std::mutex> lk(g_prof.mu);
  if (g_prof.seen[kid]++ % g_prof.every != 0) return false;
  if (!g_prof.pool.empty()) {
    *r = g_prof.pool.back();
    g_prof.pool.pop_back();
  } else if (hipEventCreate(&r->a) != hipSuccess || hipEventCreate(&r->b) != hipSuccess) {
    return false;
  }
  r->kid = kid;
  return true;
}
inline void prof_keep(const ProfRecord &r) {
  std::lock_guard<std::mutex> lk(g_prof.mu);
  g_prof.recs.push_back(r);
}

// Kernel launch; a timed launch hands its event pair to the runtime, which stamps
// them with the begin and end of the kernel's execution on the device (the same
// interval a kernel trace reports), the stream is always the 5th macro argument.
#define PROF_LAUNCH(KID, KERNEL, GRID, BLOCK, LDS, STREAM, ...)                                \
  do {                                                                                         \
    ProfRecord prof_rec_{-1, nullptr, nullptr};                                                \
    if (prof_take(KID, &prof_rec_)) {                                                          \
      hipExtLaunchKernelGGL(KERNEL, GRID, BLOCK, LDS, STREAM, prof_rec_.a, prof_rec_.b, 0,     \
                            __VA_ARGS__);                                                      \
      prof_keep(prof_rec_);                                                                    \
    } else {                                                                                   \
      hipLaunchKernelGGL(KERNEL, GRID, BLOCK, LDS, STREAM, __VA_ARGS__);                       \
    }                                                                                          \
  } while (0)

#define LAUNCH_CHECK()                                  \
  do {                                                  \
    if (hipGetLastError() != hipSuccess) return RANS_ERR_HIP; \
  } while (0)

inline bool aligned_to(const void *p, size_t a) { return ((uintptr_t)p % a) == 0; }

// Compute units of the current device (0 if the query fails); asked once per device.
inline uint32_t compute_units() {
  static std::atomic<int> cached[64];
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return 0;
  int v = cached[dev].load(std::memory_order_relaxed);
  if (v == 0) {
    if (hipDeviceGetAttribute(&v, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || v <= 0) return 0;
    cached[dev].store(v, std::memory_order_relaxed);
  }
  return (uint32_t)v;
}

#pragma GCC visibility pop
