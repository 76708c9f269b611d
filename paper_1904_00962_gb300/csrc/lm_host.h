// Host helpers of the language-model operators: errors, the device guard, and
// tensor maps.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdarg.h>
#include <stdint.h>
#include <stdio.h>

#include "lamb.h"
#include "lamb_internal.h"

namespace lamb {

inline lamb_status_t lm_fail(lamb_status_t st, const char* fmt, ...) {
  char msg[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(msg, sizeof(msg), fmt, ap);
  va_end(ap);
  set_last_error(msg);
  return st;
}

// The runtime's record of the error is taken back: it is reported here, once, and
// would be the next launch's otherwise.
inline lamb_status_t lm_cuda_fail(cudaError_t e, const char* what) {
  (void)cudaGetLastError();
  return lm_fail(e == cudaErrorMemoryAllocation ? LAMB_ERR_OOM : LAMB_ERR_CUDA,
                 "%s: %s (%d)", what, cudaGetErrorString(e), (int)e);
}

// Makes a device current for a scope.
struct LmDevice {
  int prev = -1;
  cudaError_t err;
  explicit LmDevice(int dev) {
    err = cudaGetDevice(&prev);
    if (err == cudaSuccess && prev != dev) {
      err = cudaSetDevice(dev);
    } else {
      prev = -1;
    }
  }
  ~LmDevice() {
    if (prev >= 0) cudaSetDevice(prev);
  }
};

constexpr int64_t lm_round_up(int64_t x, int64_t a) { return (x + a - 1) / a * a; }
constexpr int64_t lm_ceil_div(int64_t x, int64_t a) { return (x + a - 1) / a; }

// Pieces of one device allocation, each on a 1024-byte boundary.
struct LmArena {
  char* base = nullptr;
  size_t used = 0;
  template <class T>
  void take(T** p, int64_t n) {
    *p = base ? reinterpret_cast<T*>(base + used) : nullptr;
    used += (size_t)lm_round_up(n * (int64_t)sizeof(T), 1024);
  }
};

inline int lm_elem_size(int dtype) { return dtype == LAMB_F32 ? 4 : 2; }

// Launches a kernel; its own error, whatever an earlier call left.  after_prior: it may start while the launch in front of it in
// the stream still runs, and waits for that one itself (after_prior_launch).
template <class... P, class... A>
cudaError_t lm_launch(void (*kernel)(P...), unsigned grid, unsigned block,
                      size_t smem, cudaStream_t stream, bool after_prior,
                      A&&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(block);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = after_prior ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...);
}

typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t,
                                void*, const cuuint64_t*, const cuuint64_t*,
                                const cuuint32_t*, const cuuint32_t*,
                                CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion,
                                CUtensorMapFloatOOBfill);

// The driver's encoder; NULL if the driver has none.
inline EncodeTiled lm_encoder() {
  void* fn = nullptr;
  cudaDriverEntryPointQueryResult found;
  if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000,
                                       cudaEnableDefault, &found) !=
          cudaSuccess ||
      found != cudaDriverEntryPointSuccess) {
    (void)cudaGetLastError();
    return nullptr;
  }
  return reinterpret_cast<EncodeTiled>(fn);
}

// A 16-bit matrix of `rows` lines of `cols` elements, row_stride elements apart
// (a multiple of 8, the base on 16 bytes), copied in boxes of 64 columns (128-byte
// swizzle) or 32 (64-byte swizzle) by box_rows lines.
inline bool lm_map(EncodeTiled encode, CUtensorMap* map, bool bf16,
                   const void* base, int64_t rows, int64_t cols,
                   int64_t row_stride, int box_rows, int box_cols = 64) {
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)row_stride * 2};
  const cuuint32_t box[2] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows};
  const cuuint32_t step[2] = {1, 1};
  return encode(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
                          : CU_TENSOR_MAP_DATA_TYPE_FLOAT16,
                2, const_cast<void*>(base), dims, strides, box, step,
                CU_TENSOR_MAP_INTERLEAVE_NONE,
                box_cols == 64 ? CU_TENSOR_MAP_SWIZZLE_128B
                               : CU_TENSOR_MAP_SWIZZLE_64B,
                CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// An fp32 matrix in boxes of 32 columns (128-byte swizzle) by box_rows lines; the
// row stride a multiple of 4.
inline bool lm_map_f32(EncodeTiled encode, CUtensorMap* map, const void* base,
                       int64_t rows, int64_t cols, int64_t row_stride,
                       int box_rows) {
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)row_stride * 4};
  const cuuint32_t box[2] = {32, (cuuint32_t)box_rows};
  const cuuint32_t step[2] = {1, 1};
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 2,
                const_cast<void*>(base), dims, strides, box, step,
                CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// A matrix of `blocks` times 64 columns in boxes of 64 lines by box_blocks blocks,
// which arrive block after block (an MN-major operand).  Whole blocks are copied:
// the rows have to have that many elements, whatever the last ones are.
inline bool lm_map_blocks(EncodeTiled encode, CUtensorMap* map, bool bf16,
                          const void* base, int64_t rows, int64_t row_stride,
                          int64_t blocks, int box_blocks) {
  const cuuint64_t dims[3] = {64, (cuuint64_t)rows, (cuuint64_t)blocks};
  const cuuint64_t strides[2] = {(cuuint64_t)row_stride * 2, 128};
  const cuuint32_t box[3] = {64, 64, (cuuint32_t)box_blocks};
  const cuuint32_t step[3] = {1, 1, 1};
  return encode(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
                          : CU_TENSOR_MAP_DATA_TYPE_FLOAT16,
                3, const_cast<void*>(base), dims, strides, box, step,
                CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Whether a 16-bit matrix can be copied by a tensor map where it lies.
inline bool lm_mappable(const void* p, int64_t row_stride) {
  return ((uintptr_t)p & 15) == 0 && row_stride % 8 == 0;
}

}  // namespace lamb
