// Root-mean-square norm of rows, with the residual's addition.
//
//   h = x + residual, rounded to the residual's type and stored;  h = x without
//   r = 1 / sqrt(mean of h^2 + eps)
//   y = h r w, in fp32 or bf16, or in e4m3 with a scale for each block of columns:
//       s = max(largest |y| of the block, 2^-100) / 448,  q = e4m3(y (1 / s))
//
// The norm is that of h as it is stored, so that the gradient (lm_norm_grad.cu),
// which reads h, is the gradient of this function.  Sums of squares are fp32.
//
// Bound by memory: each row is read once, kept in registers while its sum goes over
// the lanes, and written.  A row of up to 1,024 columns is a warp's (or a part of one),
// so that no barrier is needed; one of up to 16,384 is a CTA's.  65,536 x 1,024 in bf16
// 81 us, 6.6 TB/s; 8,191 x 4,096 from an fp32 stream to e4m3 60, 6.1 (64 registers a
// thread, so that eight CTAs of 128 fit an SM, spill some: 64).  Rows that are taken
// column by column are slower: 30,000 x 757 in bf16 50 us, 27 at memory's rate.
#include <algorithm>
#include <new>

#include "lamb_sync.cuh"
#include "lm_norm.h"
#include "lm_rows.cuh"

namespace lamb {
namespace {

constexpr float kE4m3Max = 448.f;
constexpr float kLeast = 7.8886090522101181e-31f;      // 2^-100

struct NormArgs {
  const void* x;
  const void* residual;       // NULL: h = x
  void* total;                // h, where there is a residual
  const void* weight;         // NULL: ones
  void* out;
  float* scales;              // [rows][blocks]
  int64_t x_stride, residual_stride, total_stride, out_stride;
  int64_t rows;
  int width, weight_bf16;
  int block, blocks;          // columns of a scale: 32, 128, or the width
  int block_log2;             // (where it is 32 or 128)
  int lanes;                  // of a row, in a warp
  float eps, inv_width;
};

__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi) {
  return __nv_cvt_float2_to_fp8x2(make_float2(lo, hi), __NV_SATFINITE,
                                  __NV_E4M3);
}
__device__ __forceinline__ float scale_of(float largest) {
  return max_nan(largest, kLeast) / kE4m3Max;
}

// The largest size over a warp: NaN, whose bits are above all numbers', if one is.
__device__ __forceinline__ float warp_largest(float x) {
  return __uint_as_float(
      __reduce_max_sync(0xffffffffu, __float_as_uint(x) & 0x7fffffffu));
}

// The sum or the largest over a row's threads.
template <bool kMax>
__device__ __forceinline__ float over_row(float v, int lanes, bool wide,
                                          float* shared) {
  v = kMax ? lanes_max(v, lanes) : lanes_sum(v, lanes);
  if (wide) {
    const int warps = blockDim.x >> 5;
    if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = v;
    __syncthreads();
    v = shared[0];
    for (int w = 1; w < warps; ++w)
      v = kMax ? max_nan(v, shared[w]) : v + shared[w];
  }
  return v;
}

// Eight values in e4m3.
template <bool kVec>
__device__ __forceinline__ void put_e4m3(uint8_t* row, const Place& p, int i,
                                         const float (&y)[8], float inv) {
  if (kVec) {
    if (!has<kVec>(p, i, 0)) return;
    uint2 q;
    q.x = e4m3x2(y[0] * inv, y[1] * inv) | e4m3x2(y[2] * inv, y[3] * inv) << 16;
    q.y = e4m3x2(y[4] * inv, y[5] * inv) | e4m3x2(y[6] * inv, y[7] * inv) << 16;
    *reinterpret_cast<uint2*>(row + column<kVec>(p, i, 0)) = q;
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (has<kVec>(p, i, j))
        row[column<kVec>(p, i, j)] = (uint8_t)(e4m3x2(y[j] * inv, 0.f) & 255u);
  }
}

template <class TX, class TH, int kOut, int kN, bool kWide, bool kVec>
__global__ void __launch_bounds__(kWide ? 32 * kNormMostWarps : kNormThreads)
norm_rows_kernel(const NormArgs a) {
  __shared__ float shared[2][kNormMostWarps];
  // (more than one group a lane: a whole warp has the row)
  const int lanes = kWide || kN > 1 ? 32 : a.lanes;
  const int64_t row =
      kWide ? blockIdx.x
            : ((int64_t)blockIdx.x * kNormThreads + threadIdx.x) / lanes;
  const Place p = place<kVec, kWide, kN>(lanes, a.width, kWide || row < a.rows);
  const bool add = a.residual != nullptr;
  Group<TX, kVec> ex[kN];
  Group<TH, kVec> er[kN];
#pragma unroll
  for (int i = 0; i < kN; ++i)
    ex[i].load(static_cast<const TX*>(a.x) + row * a.x_stride, p, i);
  if (add) {
#pragma unroll
    for (int i = 0; i < kN; ++i)
      er[i].load(static_cast<const TH*>(a.residual) + row * a.residual_stride, p,
                 i);
  }
  float h[kN][8];
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < kN; ++i) {
    ex[i].get(h[i]);
    if (add) {
      float y[8];
      er[i].get(y);
#pragma unroll
      for (int j = 0; j < 8; ++j) y[j] += h[i][j];
      er[i].set(y);
      er[i].get(h[i]);
      er[i].store(static_cast<TH*>(a.total) + row * a.total_stride, p, i);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) sum = fmaf(h[i][j], h[i][j], sum);
  }
  sum = over_row<false>(sum, lanes, kWide, shared[0]);
  const float r = rsqrtf(fmaf(sum, a.inv_width, a.eps));
  uint8_t* out8 = static_cast<uint8_t*>(a.out) + row * a.out_stride;
  float most = 0.f;
#pragma unroll
  for (int i = 0; i < kN; ++i) {
    float w[8];
    weight8<kVec>(a.weight, a.weight_bf16, p, i, w);
#pragma unroll
    for (int j = 0; j < 8; ++j) h[i][j] = h[i][j] * r * w[j];
    if (kOut == 0) {
      Group<float, kVec> o;
      o.set(h[i]);
      o.store(static_cast<float*>(a.out) + row * a.out_stride, p, i);
    }
    if (kOut == 1) {
      Group<__nv_bfloat16, kVec> o;
      o.set(h[i]);
      o.store(static_cast<__nv_bfloat16*>(a.out) + row * a.out_stride, p, i);
    }
    if (kOut == 2 && a.block == a.width) {
#pragma unroll
      for (int j = 0; j < 8; ++j) most = max_nan(most, fabsf(h[i][j]));
    }
    if (kOut == 2 && a.block != a.width && kVec) {
      // the threads of a block of columns are neighbours
      float m = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) m = max_nan(m, fabsf(h[i][j]));
      const float s = scale_of(lanes_max(m, a.block / 8));
      put_e4m3<kVec>(out8, p, i, h[i], 1.f / s);
      const int c = column<kVec>(p, i, 0);
      if (has<kVec>(p, i, 0) && (c & (a.block - 1)) == 0)
        a.scales[row * a.blocks + (c >> a.block_log2)] = s;
    }
    if (kOut == 2 && a.block != a.width && !kVec) {
      // 32 neighbouring columns are a warp's, four such a block of 128
      float m[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) m[j] = warp_largest(h[i][j]);
      if (a.block == 128) {
#pragma unroll
        for (int j = 0; j < 8; j += 4)
          m[j] = m[j + 1] = m[j + 2] = m[j + 3] =
              max_nan(max_nan(m[j], m[j + 1]), max_nan(m[j + 2], m[j + 3]));
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float s = scale_of(m[j]);
        const int c = column<kVec>(p, i, j);
        if (!has<kVec>(p, i, j)) continue;
        out8[c] = (uint8_t)(e4m3x2(h[i][j] * (1.f / s), 0.f) & 255u);
        if ((c & (a.block - 1)) == 0)
          a.scales[row * a.blocks + (c >> a.block_log2)] = s;
      }
    }
  }
  if (kOut == 2 && a.block == a.width) {
    const float s = scale_of(over_row<true>(most, lanes, kWide, shared[1]));
    if (p.in && p.mine == 0) a.scales[row] = s;
#pragma unroll
    for (int i = 0; i < kN; ++i) put_e4m3<kVec>(out8, p, i, h[i], 1.f / s);
  }
}

// Rows that do not fit a CTA's registers, of any alignment: a warp has 128 columns at
// a time, and the second look at h comes from memory (its own stores, in the same
// thread).  4,096 x 20,480 in bf16 257 us, 2.6 TB/s of bytes that it cannot do without.
template <class TX, class TH, int kOut>
__global__ void __launch_bounds__(kNormWalk) norm_walk_kernel(const NormArgs a) {
  __shared__ float shared[2][kNormWalk / 32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t row = blockIdx.x;
  const TX* x = static_cast<const TX*>(a.x) + row * a.x_stride;
  const TH* res = static_cast<const TH*>(a.residual) + row * a.residual_stride;
  TH* total = static_cast<TH*>(a.total) + row * a.total_stride;
  const bool add = a.residual != nullptr;
  float sum = 0.f;
  for (int c0 = warp * 128; c0 < a.width; c0 += kNormWalk / 32 * 128)
    for (int c = c0 + lane; c < min(c0 + 128, a.width); c += 32) {
      float h = get1(x + c);
      if (add) {
        h = as_held<TH>(h + get1(res + c));
        put1(total + c, h);
      }
      sum = fmaf(h, h, sum);
    }
  sum = over_row<false>(sum, 32, true, shared[0]);
  const float r = rsqrtf(fmaf(sum, a.inv_width, a.eps));
  const auto value = [&](int c) {
    const float h = add ? get1(total + c) : get1(x + c);
    return h * r * weight1(a.weight, a.weight_bf16, c);
  };
  if (kOut != 2) {
    for (int c0 = warp * 128; c0 < a.width; c0 += kNormWalk / 32 * 128)
      for (int c = c0 + lane; c < min(c0 + 128, a.width); c += 32) {
        if (kOut == 0)
          static_cast<float*>(a.out)[row * a.out_stride + c] = value(c);
        else
          put1(static_cast<__nv_bfloat16*>(a.out) + row * a.out_stride + c,
               value(c));
      }
    return;
  }
  uint8_t* out = static_cast<uint8_t*>(a.out) + row * a.out_stride;
  float s = 0.f;
  if (a.block == a.width) {
    float most = 0.f;
    for (int c0 = warp * 128; c0 < a.width; c0 += kNormWalk / 32 * 128)
      for (int c = c0 + lane; c < min(c0 + 128, a.width); c += 32)
        most = max_nan(most, fabsf(value(c)));
    s = scale_of(over_row<true>(most, 32, true, shared[1]));
    if (threadIdx.x == 0) a.scales[row] = s;
  }
  for (int c0 = warp * 128; c0 < a.width; c0 += kNormWalk / 32 * 128) {
    float y[4], most[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = c0 + i * 32 + lane;
      y[i] = c < a.width ? value(c) : 0.f;
      if (a.block != a.width) most[i] = warp_largest(y[i]);
    }
    if (a.block == 128) {
      const float m =
          max_nan(max_nan(most[0], most[1]), max_nan(most[2], most[3]));
      most[0] = most[1] = most[2] = most[3] = m;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = c0 + i * 32 + lane;
      if (a.block != a.width) s = scale_of(most[i]);
      if (c >= a.width) continue;
      if (a.block != a.width && (c & (a.block - 1)) == 0)
        a.scales[row * a.blocks + (c >> a.block_log2)] = s;
      out[c] = (uint8_t)(e4m3x2(y[i] * (1.f / s), 0.f) & 255u);
    }
  }
}

template <class TX, class TH, int kOut, bool kVec>
cudaError_t launch_norm(const NormArgs& a, const NormLayout& l,
                        cudaStream_t stream) {
  void (*k)(NormArgs) = norm_walk_kernel<TX, TH, kOut>;
  if (l.wide) k = norm_rows_kernel<TX, TH, kOut, kNormEights, true, kVec>;
  else if (!l.walk && l.eights == 1)
    k = norm_rows_kernel<TX, TH, kOut, 1, false, kVec>;
  else if (!l.walk && l.eights == 2)
    k = norm_rows_kernel<TX, TH, kOut, 2, false, kVec>;
  else if (!l.walk)
    k = norm_rows_kernel<TX, TH, kOut, 4, false, kVec>;
  return lm_launch(k, (unsigned)lm_ceil_div(a.rows, l.rows), l.threads, 0,
                   stream, false, a);
}
template <class TX, class TH>
cudaError_t launch_out(const NormArgs& a, const NormLayout& l, int out_dtype,
                       cudaStream_t stream) {
  if (out_dtype == LAMB_F32)
    return l.vec ? launch_norm<TX, TH, 0, true>(a, l, stream)
                 : launch_norm<TX, TH, 0, false>(a, l, stream);
  if (out_dtype == LAMB_BF16)
    return l.vec ? launch_norm<TX, TH, 1, true>(a, l, stream)
                 : launch_norm<TX, TH, 1, false>(a, l, stream);
  return l.vec ? launch_norm<TX, TH, 2, true>(a, l, stream)
               : launch_norm<TX, TH, 2, false>(a, l, stream);
}

}  // namespace

lamb_status_t norm_check(const lamb_norm* v, int64_t n) {
  if (!v) return lm_fail(LAMB_ERR_INVALID_ARG, "plan is NULL");
  if (n < 0 || n > v->max_rows)
    return lm_fail(LAMB_ERR_INVALID_ARG,
                   "n_rows %lld is not in [0, max_rows = %lld]", (long long)n,
                   (long long)v->max_rows);
  return LAMB_OK;
}
lamb_status_t norm_check_rows(const lamb_norm* v, const LmRows& m, bool e4m3) {
  const bool known = m.dtype == LAMB_F32 || m.dtype == LAMB_BF16 ||
                     (e4m3 && m.dtype == LAMB_E4M3);
  if (!known)
    return lm_fail(LAMB_ERR_UNSUPPORTED_DTYPE, "%s: dtype %d unsupported",
                   m.name, m.dtype);
  if (!m.p) return lm_fail(LAMB_ERR_INVALID_ARG, "%s is NULL", m.name);
  if (m.stride < v->width)
    return lm_fail(LAMB_ERR_INVALID_ARG, "%s: row stride below the width %d",
                   m.name, v->width);
  if (m.dtype != LAMB_E4M3 && (uintptr_t)m.p % lm_elem_size(m.dtype))
    return lm_fail(LAMB_ERR_INVALID_ARG, "%s: pointer not aligned", m.name);
  return LAMB_OK;
}
lamb_status_t norm_check_vector(const char* name, const void* p, int dtype) {
  if (dtype != LAMB_F32 && dtype != LAMB_BF16)
    return lm_fail(LAMB_ERR_UNSUPPORTED_DTYPE, "%s: dtype %d unsupported", name,
                   dtype);
  if ((uintptr_t)p % lm_elem_size(dtype))
    return lm_fail(LAMB_ERR_INVALID_ARG, "%s: pointer not aligned", name);
  return LAMB_OK;
}

}  // namespace lamb

using namespace lamb;

extern "C" lamb_status_t lamb_norm_create(int32_t width, int64_t max_rows,
                                          double eps, int32_t device,
                                          struct lamb_norm** out) {
  if (!out) return lm_fail(LAMB_ERR_INVALID_ARG, "out is NULL");
  *out = nullptr;
  if (width < 1 || width > (1 << 20))
    return lm_fail(LAMB_ERR_INVALID_ARG, "width is not in [1, 2^20]");
  if (max_rows < 1 || max_rows > (1ll << 24))
    return lm_fail(LAMB_ERR_INVALID_ARG, "max_rows is not in [1, 2^24]");
  if (!(eps >= 1e-20) || !(eps <= 1.))
    return lm_fail(LAMB_ERR_INVALID_ARG, "eps is not in [1e-20, 1]");
  if (device < 0) return lm_fail(LAMB_ERR_INVALID_ARG, "device < 0");
  LmDevice dev(device);
  if (dev.err != cudaSuccess) return lm_cuda_fail(dev.err, "cudaSetDevice");
  lamb_norm* v = new (std::nothrow) lamb_norm;
  if (!v) return lm_fail(LAMB_ERR_OOM, "host allocation failed");
  v->device = device;
  v->width = width;
  v->max_rows = max_rows;
  v->eps = (float)eps;
  cudaError_t e =
      cudaDeviceGetAttribute(&v->sms, cudaDevAttrMultiProcessorCount, device);
  if (e == cudaSuccess) {
    v->max_parts = (int)std::min<int64_t>(max_rows, norm_most_parts(v->sms, width));
    e = cudaMalloc((void**)&v->part,
                   (size_t)v->max_parts * width * sizeof(float));
  }
  if (e == cudaSuccess) {
    e = norm_grad_setup(width);
    if (e != cudaSuccess) cudaFree(v->part);
  }
  if (e != cudaSuccess) {
    delete v;
    return lm_cuda_fail(e, "norm plan");
  }
  *out = v;
  return LAMB_OK;
}

extern "C" lamb_status_t lamb_norm_destroy(struct lamb_norm* v) {
  if (!v) return LAMB_OK;
  LmDevice dev(v->device);
  cudaError_t e = dev.err;
  if (e == cudaSuccess) e = cudaFree(v->part);
  delete v;
  return e == cudaSuccess ? LAMB_OK : lm_cuda_fail(e, "cudaFree(plan)");
}

extern "C" lamb_status_t lamb_norm_forward(
    struct lamb_norm* v, const void* x, int32_t x_dtype, int64_t x_stride,
    const void* residual, int64_t residual_stride, void* total,
    int64_t total_stride, int32_t total_dtype, const void* weight,
    int32_t weight_dtype, int64_t n_rows, void* out, int32_t out_dtype,
    int64_t out_stride, float* scales, int32_t block, cudaStream_t stream) {
  lamb_status_t st = norm_check(v, n_rows);
  if (st != LAMB_OK) return st;
  if ((residual != nullptr) != (total != nullptr))
    return lm_fail(LAMB_ERR_INVALID_ARG, "total: needed iff there is a residual");
  if (weight)
    if ((st = norm_check_vector("weight", weight, weight_dtype)) != LAMB_OK)
      return st;
  const bool e4m3 = out_dtype == LAMB_E4M3;
  if (e4m3 && block != 0 && block != 32 && block != 128)
    return lm_fail(LAMB_ERR_INVALID_ARG, "block is not 0, 32 or 128");
  if (!n_rows) return LAMB_OK;
  if (e4m3 && (!scales || (uintptr_t)scales % 4))
    return lm_fail(LAMB_ERR_INVALID_ARG, "scales is NULL or not aligned");
  const LmRows in = {"x", x, x_dtype, x_stride},
               to = {"out", out, out_dtype, out_stride};
  if ((st = norm_check_rows(v, in, false)) != LAMB_OK ||
      (st = norm_check_rows(v, to, true)) != LAMB_OK)
    return st;
  if (residual) {
    const LmRows r = {"residual", residual, total_dtype, residual_stride},
                 t = {"total", total, total_dtype, total_stride};
    if ((st = norm_check_rows(v, r, false)) != LAMB_OK ||
        (st = norm_check_rows(v, t, false)) != LAMB_OK)
      return st;
  }
  LmDevice dev(v->device);
  if (dev.err != cudaSuccess) return lm_cuda_fail(dev.err, "cudaSetDevice");
  NormArgs a = {};
  a.x = x;
  a.residual = residual;
  a.total = total;
  a.weight = weight;
  a.out = out;
  a.scales = scales;
  a.x_stride = x_stride;
  a.residual_stride = residual_stride;
  a.total_stride = total_stride;
  a.out_stride = out_stride;
  a.rows = n_rows;
  a.width = v->width;
  a.weight_bf16 = weight_dtype == LAMB_BF16;
  a.block = block && block < v->width ? block : v->width;
  a.blocks = (int)lm_ceil_div(v->width, a.block);
  a.block_log2 = a.block == 128 ? 7 : 5;
  a.eps = v->eps;
  a.inv_width = (float)(1. / v->width);
  const bool vec =
      v->width % 8 == 0 && norm_vec(x, x_dtype, x_stride) &&
      norm_vec(out, out_dtype, out_stride) && ((uintptr_t)weight & 15) == 0 &&
      (!residual || (norm_vec(residual, total_dtype, residual_stride) &&
                     norm_vec(total, total_dtype, total_stride)));
  // (threads that form a scale together share the row)
  const bool scaled = e4m3 && a.block != a.width;
  const NormLayout l = norm_layout(
      v->width, vec, !scaled ? 1 : vec ? a.block / 8 : 32, kNormEights,
      kNormEights);
  a.lanes = l.lanes;
  typedef __nv_bfloat16 bf;
  const bool th_f32 = !residual || total_dtype == LAMB_F32;
  cudaError_t e;
  if (x_dtype == LAMB_F32 && th_f32)
    e = launch_out<float, float>(a, l, out_dtype, stream);
  else if (x_dtype == LAMB_F32)
    e = launch_out<float, bf>(a, l, out_dtype, stream);
  else if (th_f32)
    e = launch_out<bf, float>(a, l, out_dtype, stream);
  else
    e = launch_out<bf, bf>(a, l, out_dtype, stream);
  return e == cudaSuccess ? LAMB_OK : lm_cuda_fail(e, "norm launch");
}
