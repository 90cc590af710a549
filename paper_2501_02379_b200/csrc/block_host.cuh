// Host-side helpers of the operators of a trained block: types, rows, packed matrices.
#pragma once
#include <cmath>
#include <cstring>

#include "../../include/tgrad.h"
#include "launch.cuh"
#include "packed.cuh"

namespace tg {

#define TG_TRY(expr) do { tgrad_status s_ = (expr); if (s_ != TGRAD_OK) return s_; } while (0)

inline int sm_count() {
  int dev = 0, sm = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sm, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || sm < 1) return 148;
  return sm;
}
inline bool misaligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }
inline size_t align_up(size_t x) { return (x + 255) / 256 * 256; }
template <typename F>
tgrad_status allow_shared(F kern, size_t bytes, std::atomic<uint64_t>& done) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return TGRAD_ERR_CUDA;
  const uint64_t bit = 1ull << (dev & 63);
  if (dev < 64 && (done.load(std::memory_order_acquire) & bit)) return TGRAD_OK;
  if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) != cudaSuccess) return TGRAD_ERR_CUDA;
  if (dev < 64) done.fetch_or(bit, std::memory_order_release);
  return TGRAD_OK;
}

inline int kind_of(int32_t dtype) { return dtype == TGRAD_R32 ? LS_F32 : dtype == TGRAD_R16H ? LS_F16 : dtype == TGRAD_R16B ? LS_BF16 : -1; }
inline int bytes_of(int kind) { return kind == LS_F32 ? 4 : 2; }

// Rows as the kernels take them; al: what divides the address of every row's first entry.
inline RowsOf rows_of(const tgrad_rows& r, int64_t rows, int kind) {
  const int b = bytes_of(kind);
  RowsOf t;
  t.p = static_cast<char*>(r.d_data); t.ld = rows > 1 ? r.row_stride : 0;
  uint64_t bits = reinterpret_cast<uintptr_t>(t.p) | (uint64_t)(t.ld * b);
  t.al = bits & 1 ? 1 : bits & 2 ? 2 : bits & 4 ? 4 : bits & 8 ? 8 : 16;
  return t;
}
inline RowsOf vector_of(const void* p, int kind) { tgrad_rows r; r.d_data = const_cast<void*>(p); r.row_stride = 0; return rows_of(r, 1, kind); }
// Whether a matrix's address and stride are none that can be used.  `wanted`: it has to be there.
inline bool bad_rows(const tgrad_rows& r, int64_t rows, int64_t width, int kind, bool wanted) {
  if (rows == 0) return false;
  if (!r.d_data) return wanted;
  return misaligned(r.d_data, bytes_of(kind)) || (rows > 1 && (r.row_stride < width || r.row_stride >= ((int64_t)1 << 40)));
}

// ---- packed ----
inline int64_t blocks_of(int64_t width) { return (width + 31) / 32; }
inline int64_t exp_stride(int64_t width) { return (blocks_of(width) + 3) / 4 * 4; }
inline tgrad_status check_shape(int64_t rows, int64_t width) {
  if (rows < 0 || width < 1 || width > ((int64_t)1 << 30) || rows >= ((int64_t)1 << 40)) return TGRAD_ERR_INVALID_ARG;
  if (rows > (((int64_t)1 << 48) - 1) / blocks_of(width)) return TGRAD_ERR_INVALID_ARG;
  return TGRAD_OK;
}
inline bool bad_packed(const void* p, int64_t rows, bool wanted) { return rows > 0 && (p ? misaligned(p, 16) : wanted); }
inline PackedRows packed_of(const void* p, int64_t rows, int64_t width) {
  PackedRows t;
  t.blocks = (int)blocks_of(width); t.exp_stride = (int)exp_stride(width);
  t.codes = static_cast<unsigned char*>(const_cast<void*>(p)); t.exps = p ? t.codes + rows * 32 * t.blocks : nullptr;
  return t;
}
}  // namespace tg
