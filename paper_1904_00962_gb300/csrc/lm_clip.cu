// Global norm of a list of gradients, and their scaling so that it stays in bounds.
//
//   N = |s| sqrt(sum over all tensors of g^2),  f = s min(1, max_norm / N),  out = f g
//
// Where f is 1 and the gradients are clipped in place, nothing is written.  An f below
// fp32's normal numbers (of gradients near 1e38) is kept as f 2^126 and 2^-126, which g is
// multiplied by one after the other: so it has its digits.  (336e6 gradients: no slower.)
//
// Sums of squares are fp32 for the 64 or so elements of a thread's part of a chunk,
// and 64-bit beyond.  Such a part whose fp32 sum leaves [2^-100, 2^128) is summed
// again with its elements times 2^100 or 2^-100, so that neither gradients of 1e-30
// nor of 1e30 lose their norm.  CTAs have their chunks by number and their sums are
// added in order: the same bits in every run.
//
// Bound by memory: the gradients are read twice, once for N.  The second time goes
// backwards, so that what the first left in L2 is met there.  336e6 fp32 gradients to
// bf16 494 us, 6.6 and 6.9 TB/s (1,570 element by element, where tensors are off their
// boundary); 109e6 of bf16 within the bound 41, 5.6.  Other numbers
// of groups of a thread and of CTAs an SM are slower: (8, 4) 579 us, (4, 6) 538, (16, 2)
// 531 and (2, 8) 522 of the first, against 503 of (8, 3) then.
#include <math.h>

#include <algorithm>
#include <new>
#include <vector>

#include "lamb_sync.cuh"
#include "lm_host.h"
#include "lm_ranges.h"
#include "lm_rows.cuh"

namespace lamb {
namespace {

constexpr int kClipThreads = 256;
constexpr int kClipEights = 8;                 // groups of eight of a thread
constexpr int kClipChunk = kClipThreads * kClipEights * 8;
constexpr int kClipPerSm = 3;

struct ClipChunk {
  const void* g;
  void* out;
  int len, vec;               // vec: both addresses are on eight elements
};

struct ClipArgs {
  const ClipChunk* chunks;
  int n_chunks;
  const float* d_scale;       // NULL: 1
  double max_norm;
  double* part;               // of each CTA
  uint32_t* ticket;
  float2* own_factor;         // f, as a product
  float* norm;                // NULL, or for the caller
  float* factor;
  uint32_t* status;
};

// Sum of the squares of (g times) of a thread's part of a chunk.
template <class T>
__device__ __forceinline__ float squares(const ClipChunk& c, float times) {
  const T* g = static_cast<const T*>(c.g);
  float s = 0.f;
  if (c.vec) {
    const int eights = c.len / 8;
    Eight<T> e[kClipEights];
#pragma unroll
    for (int i = 0; i < kClipEights; ++i) {
      const int at = threadIdx.x + i * kClipThreads;
      if (at < eights) e[i].load_global(g + at * 8);
      else e[i].clear();
    }
#pragma unroll
    for (int i = 0; i < kClipEights; ++i) {
      float x[8];
      e[i].get(x);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        x[j] *= times;
        s = fmaf(x[j], x[j], s);
      }
    }
    const int at = eights * 8 + threadIdx.x;
    if (at < c.len) {
      const float x = get1(g + at) * times;
      s = fmaf(x, x, s);
    }
  } else {
    for (int at = threadIdx.x; at < c.len; at += kClipThreads) {
      const float x = get1(g + at) * times;
      s = fmaf(x, x, s);
    }
  }
  return s;
}

__device__ __forceinline__ double lanes_sum64(double x) {
#pragma unroll
  for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}
// Over the CTA, in every thread.
__device__ __forceinline__ double cta_sum64(double x, double* shared) {
  x = lanes_sum64(x);
  if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = x;
  __syncthreads();
  x = 0.;
#pragma unroll
  for (int w = 0; w < kClipThreads / 32; ++w) x += shared[w];
  __syncthreads();
  return x;
}

template <class T>
__global__ void __launch_bounds__(kClipThreads, kClipPerSm)
clip_norm_kernel(const ClipArgs a) {
  __shared__ double shared[kClipThreads / 32];
  __shared__ uint32_t last;
  double sum = 0.;
  for (int k = blockIdx.x; k < a.n_chunks; k += gridDim.x) {
    const ClipChunk c = a.chunks[k];
    const float s = squares<T>(c, 1.f);
    if (s >= 0x1p-100f && s < INFINITY) {
      sum += (double)s;
    } else if (s < 1.f) {
      sum += (double)squares<T>(c, 0x1p100f) * 0x1p-200;
    } else {
      sum += (double)squares<T>(c, 0x1p-100f) * 0x1p200;     // (or NaN)
    }
  }
  sum = cta_sum64(sum, shared);
  if (threadIdx.x == 0) {
    a.part[blockIdx.x] = sum;
    __threadfence();
    last = atomicInc(a.ticket, gridDim.x - 1) == gridDim.x - 1;
  }
  __syncthreads();
  if (!last) return;
  __threadfence();
  sum = 0.;
  for (int k = threadIdx.x; k < gridDim.x; k += kClipThreads) sum += a.part[k];
  sum = cta_sum64(sum, shared);
  if (threadIdx.x) return;
  const double s = a.d_scale ? (double)*a.d_scale : 1.;
  const double norm = fabs(s) * sqrt(sum);
  double f = s;
  if (isfinite(norm)) {
    if (norm > a.max_norm) f = s * (a.max_norm / norm);
  } else {
    atomicOr(a.status, LAMB_STATUS_GRAD_NONFINITE);
  }
  *a.own_factor = fabs(f) < 0x1p-126
                      ? make_float2((float)(f * 0x1p126), 0x1p-126f)
                      : make_float2((float)f, 1.f);
  if (a.norm) *a.norm = (float)norm;
  if (a.factor) *a.factor = (float)f;
}

template <class T, class TO>
__global__ void __launch_bounds__(kClipThreads, kClipPerSm)
clip_apply_kernel(const ClipArgs a, bool in_place) {
  after_prior_launch();
  const float2 f = *a.own_factor;
  if (in_place && f.x == 1.f && f.y == 1.f) return;
  for (int k = a.n_chunks - 1 - blockIdx.x; k >= 0; k -= gridDim.x) {
    const ClipChunk c = a.chunks[k];
    const T* g = static_cast<const T*>(c.g);
    TO* out = static_cast<TO*>(c.out);
    if (c.vec) {
      const int eights = c.len / 8;
      Eight<T> e[kClipEights];
#pragma unroll
      for (int i = 0; i < kClipEights; ++i) {
        const int at = threadIdx.x + i * kClipThreads;
        if (at < eights) e[i].load_global(g + at * 8);
      }
#pragma unroll
      for (int i = 0; i < kClipEights; ++i) {
        const int at = threadIdx.x + i * kClipThreads;
        if (at >= eights) continue;
        float x[8];
        e[i].get(x);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = x[j] * f.x * f.y;
        Eight<TO> o;
        o.set(x);
        o.store_global(out + at * 8);
      }
      const int at = eights * 8 + threadIdx.x;
      if (at < c.len) put1(out + at, get1(g + at) * f.x * f.y);
    } else {
      for (int at = threadIdx.x; at < c.len; at += kClipThreads)
        put1(out + at, get1(g + at) * f.x * f.y);
    }
  }
}

}  // namespace
}  // namespace lamb

using namespace lamb;

struct lamb_clip {
  int device = 0, sms = 0;
  std::vector<int64_t> sizes;
  int grad_dtype = 0, out_dtype = LAMB_DTYPE_NONE;
  int n_chunks = 0;
  bool bound = false;
  void* arena = nullptr;
  ClipChunk* chunks = nullptr;
  double* part = nullptr;
  uint32_t* ticket = nullptr;
  float2* factor = nullptr;
  uint32_t* status = nullptr;
};

extern "C" lamb_status_t lamb_clip_create(const int64_t* sizes, int32_t n_tensors,
                                          int32_t grad_dtype, int32_t out_dtype,
                                          int32_t device, struct lamb_clip** out) {
  if (!out) return lm_fail(LAMB_ERR_INVALID_ARG, "out is NULL");
  *out = nullptr;
  if (!sizes || n_tensors < 1)
    return lm_fail(LAMB_ERR_INVALID_ARG, "need n_tensors >= 1 and sizes");
  if (grad_dtype != LAMB_F32 && grad_dtype != LAMB_BF16)
    return lm_fail(LAMB_ERR_UNSUPPORTED_DTYPE, "grad_dtype %d unsupported",
                   grad_dtype);
  if (out_dtype != LAMB_DTYPE_NONE && out_dtype != LAMB_F32 &&
      out_dtype != LAMB_BF16)
    return lm_fail(LAMB_ERR_UNSUPPORTED_DTYPE, "out_dtype %d unsupported",
                   out_dtype);
  if (device < 0) return lm_fail(LAMB_ERR_INVALID_ARG, "device < 0");
  int64_t total = 0, chunks = 0;
  for (int k = 0; k < n_tensors; ++k) {
    if (sizes[k] < 0 || sizes[k] > (1ll << 40))
      return lm_fail(LAMB_ERR_INVALID_ARG, "sizes[%d] is not in [0, 2^40]", k);
    total += sizes[k];
    chunks += lm_ceil_div(sizes[k], kClipChunk);
    if (total > (1ll << 40))
      return lm_fail(LAMB_ERR_INVALID_ARG, "more than 2^40 elements");
  }
  LmDevice dev(device);
  if (dev.err != cudaSuccess) return lm_cuda_fail(dev.err, "cudaSetDevice");
  lamb_clip* p = nullptr;
  try {
    p = new lamb_clip;
    p->sizes.assign(sizes, sizes + n_tensors);
  } catch (const std::bad_alloc&) {
    delete p;
    return lm_fail(LAMB_ERR_OOM, "host allocation failed");
  }
  p->device = device;
  p->grad_dtype = grad_dtype;
  p->out_dtype = out_dtype;
  p->n_chunks = (int)chunks;
  cudaError_t e =
      cudaDeviceGetAttribute(&p->sms, cudaDevAttrMultiProcessorCount, device);
  LmArena a;
  for (int pass = 0; e == cudaSuccess && pass < 2; ++pass) {
    a.used = 0;
    a.take(&p->chunks, std::max<int64_t>(chunks, 1));
    a.take(&p->part, p->sms * kClipPerSm);
    a.take(&p->ticket, 1);
    a.take(&p->factor, 1);
    a.take(&p->status, 1);
    if (pass) break;
    e = cudaMalloc(&p->arena, a.used);
    a.base = static_cast<char*>(p->arena);
  }
  if (e == cudaSuccess) e = cudaMemset(p->arena, 0, a.used);
  if (e == cudaSuccess) e = cudaDeviceSynchronize();
  if (e != cudaSuccess) {
    cudaFree(p->arena);
    delete p;
    return lm_cuda_fail(e, "clipping plan");
  }
  *out = p;
  return LAMB_OK;
}

extern "C" lamb_status_t lamb_clip_destroy(struct lamb_clip* p) {
  if (!p) return LAMB_OK;
  LmDevice dev(p->device);
  cudaError_t e = dev.err;
  if (e == cudaSuccess) e = cudaFree(p->arena);
  delete p;
  return e == cudaSuccess ? LAMB_OK : lm_cuda_fail(e, "cudaFree(plan)");
}

extern "C" lamb_status_t lamb_clip_bind(struct lamb_clip* p, void* const* g,
                                        void* const* out, cudaStream_t stream) {
  if (!p) return lm_fail(LAMB_ERR_INVALID_ARG, "plan is NULL");
  if (!g) return lm_fail(LAMB_ERR_INVALID_ARG, "g is required");
  if ((out != nullptr) != (p->out_dtype != LAMB_DTYPE_NONE))
    return lm_fail(LAMB_ERR_INVALID_ARG,
                   "out is required iff the plan has an out_dtype");
  const int in_size = lm_elem_size(p->grad_dtype);
  const int out_size = out ? lm_elem_size(p->out_dtype) : in_size;
  try {
    std::vector<ClipChunk> h;
    std::vector<MemoryRange> ranges;
    h.reserve(p->n_chunks);
    ranges.reserve(2 * p->sizes.size());
    for (size_t k = 0; k < p->sizes.size(); ++k) {
      if (!p->sizes[k]) continue;
      const char* from = static_cast<const char*>(g[k]);
      char* to = static_cast<char*>(out ? out[k] : g[k]);
      if (!from || !to)
        return lm_fail(LAMB_ERR_INVALID_ARG, "tensor %d: a pointer is NULL",
                       (int)k);
      if ((uintptr_t)from % in_size || (uintptr_t)to % out_size)
        return lm_fail(LAMB_ERR_INVALID_ARG, "tensor %d: a pointer is not aligned",
                       (int)k);
      const uintptr_t reads = (uintptr_t)from, writes = (uintptr_t)to;
      if (reads != writes || in_size != out_size)
        ranges.push_back({reads, reads + p->sizes[k] * in_size, (int)k, false});
      ranges.push_back({writes, writes + p->sizes[k] * out_size, (int)k, true});
      const int vec = (uintptr_t)from % (8 * in_size) == 0 &&
                      (uintptr_t)to % (8 * out_size) == 0;
      for (int64_t at = 0; at < p->sizes[k]; at += kClipChunk)
        h.push_back({from + at * in_size, to + at * out_size,
                     (int)std::min<int64_t>(kClipChunk, p->sizes[k] - at), vec});
    }
    const int bad = overlapping_range(ranges);
    if (bad >= 0)
      return lm_fail(LAMB_ERR_INVALID_ARG,
                     "tensor %d overlaps another one that is written", bad);
    LmDevice dev(p->device);
    cudaError_t e = dev.err;
    if (e == cudaSuccess && !h.empty())
      e = cudaMemcpyAsync(p->chunks, h.data(), h.size() * sizeof(ClipChunk),
                          cudaMemcpyHostToDevice, stream);
    if (e == cudaSuccess) e = cudaStreamSynchronize(stream);
    if (e != cudaSuccess) return lm_cuda_fail(e, "clipping bind");
  } catch (const std::bad_alloc&) {
    return lm_fail(LAMB_ERR_OOM, "host allocation failed");
  }
  p->bound = true;
  return LAMB_OK;
}

extern "C" lamb_status_t lamb_clip_grads(struct lamb_clip* p, double max_norm,
                                         const float* d_scale, float* norm,
                                         float* factor, cudaStream_t stream) {
  if (!p) return lm_fail(LAMB_ERR_INVALID_ARG, "plan is NULL");
  if (!(max_norm >= 0.))
    return lm_fail(LAMB_ERR_INVALID_ARG, "max_norm is not >= 0");
  if ((uintptr_t)d_scale % 4 || (uintptr_t)norm % 4 || (uintptr_t)factor % 4)
    return lm_fail(LAMB_ERR_INVALID_ARG,
                   "scale, norm or factor: pointer not aligned");
  if (!p->bound)
    return lm_fail(LAMB_ERR_NOT_BOUND, "lamb_clip_grads before lamb_clip_bind");
  LmDevice dev(p->device);
  if (dev.err != cudaSuccess) return lm_cuda_fail(dev.err, "cudaSetDevice");
  ClipArgs a = {};
  a.chunks = p->chunks;
  a.n_chunks = p->n_chunks;
  a.d_scale = d_scale;
  a.max_norm = max_norm;
  a.part = p->part;
  a.ticket = p->ticket;
  a.own_factor = p->factor;
  a.norm = norm;
  a.factor = factor;
  a.status = p->status;
  const unsigned grid =
      std::max(1, std::min(p->n_chunks, p->sms * kClipPerSm));
  typedef __nv_bfloat16 bf;
  const bool g16 = p->grad_dtype == LAMB_BF16;
  const bool in_place = p->out_dtype == LAMB_DTYPE_NONE;
  const bool o16 = in_place ? g16 : p->out_dtype == LAMB_BF16;
  cudaError_t e = lm_launch(g16 ? clip_norm_kernel<bf> : clip_norm_kernel<float>,
                            grid, kClipThreads, 0, stream, false, a);
  if (e == cudaSuccess)
    e = lm_launch(g16 ? (o16 ? clip_apply_kernel<bf, bf>
                             : clip_apply_kernel<bf, float>)
                      : (o16 ? clip_apply_kernel<float, bf>
                             : clip_apply_kernel<float, float>),
                  grid, kClipThreads, 0, stream, true, a, in_place);
  return e == cudaSuccess ? LAMB_OK : lm_cuda_fail(e, "clipping launch");
}

extern "C" lamb_status_t lamb_clip_query(struct lamb_clip* p,
                                         uint32_t* status_bits, int32_t clear,
                                         cudaStream_t stream) {
  if (!p) return lm_fail(LAMB_ERR_INVALID_ARG, "plan is NULL");
  if (!status_bits)
    return lm_fail(LAMB_ERR_INVALID_ARG, "status_bits is NULL");
  LmDevice dev(p->device);
  cudaError_t e = dev.err;
  if (e == cudaSuccess)
    e = cudaMemcpyAsync(status_bits, p->status, sizeof(uint32_t),
                        cudaMemcpyDeviceToHost, stream);
  if (e == cudaSuccess && clear)
    e = cudaMemsetAsync(p->status, 0, sizeof(uint32_t), stream);
  if (e == cudaSuccess) e = cudaStreamSynchronize(stream);
  return e == cudaSuccess ? LAMB_OK : lm_cuda_fail(e, "status query");
}
