// Gradient of the root-mean-square norm (lm_norm.cu).  With h the normalised rows'
// input, y = h r w and r = 1 / sqrt(mean of h^2 + eps):
//
//   g = dy w,  c = r^2 mean(g h),  dh = r (g - c h) + dh_in
//   dw_j (+)= sum over the rows of dy_j h_j r
//
// r is formed again from h, which is read anyway; h r comes before dy's factor, as dy h
// may leave fp32's range where dy h r is in it.  A row's two sums go over the
// threads that hold it; a CTA keeps dw's terms of its rows in registers, leaves one
// fp32 row of sums, and a second launch adds those in order: the same bits in every
// run, whatever the order in which CTAs finish.
#include <algorithm>

#include "lamb_sync.cuh"
#include "lm_norm.h"
#include "lm_rows.cuh"

namespace lamb {
namespace {

constexpr int kWideEights = 2;         // of a thread, where a CTA has the row
constexpr int kJoinColumns = 32;       // of a CTA that adds the parts
constexpr int kJoinThreads = 1024;

struct NormGradArgs {
  const void* dy;
  const void* h;
  const void* weight;         // NULL: ones
  const void* dh_in;          // NULL: zeros
  void* dh;
  float* part;                // [CTAs][width]; NULL: no dw
  int64_t dy_stride, h_stride, dh_in_stride, dh_stride;
  int64_t rows;
  int width, weight_bf16;
  int lanes;
  float eps, inv_width;
};

// c of a row; 0 where r is 0, because the squares' sum is beyond fp32, whatever gh is.
__device__ __forceinline__ float correction(float gh, float r, float inv_width) {
  return r > 0.f ? gh * inv_width * r * r : 0.f;
}

// Both sums over a row's threads.  `turn` alternates from row to row, so that one
// barrier a row is enough.
template <bool kWide>
__device__ __forceinline__ void over_row2(float& x, float& y, int lanes,
                                          float2 (*shared)[kNormMostWarps],
                                          int turn) {
  x = lanes_sum(x, lanes);
  y = lanes_sum(y, lanes);
  if (kWide) {
    const int warps = blockDim.x >> 5;
    if ((threadIdx.x & 31) == 0) shared[turn][threadIdx.x >> 5] = make_float2(x, y);
    __syncthreads();
    x = y = 0.f;
    for (int w = 0; w < warps; ++w) {
      x += shared[turn][w].x;
      y += shared[turn][w].y;
    }
  }
}

// 16 bytes from memory to shared memory, past the registers; kHalf: half of a 32-byte
// sector, of which the other half is taken next (from L1 then).
template <bool kHalf>
__device__ __forceinline__ void copy16(void* to, const void* from) {
  if (kHalf)
    asm volatile("cp.async.ca.shared.global [%0], [%1], 16;"
                 :: "r"(smem_u32(to)), "l"(from) : "memory");
  else
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;"
                 :: "r"(smem_u32(to)), "l"(from) : "memory");
}
__device__ __forceinline__ void copies_end() {
  asm volatile("cp.async.commit_group;" ::: "memory");
}
// All of the thread's copies but those of the last `kLeft` groups have arrived.
template <int kLeft>
__device__ __forceinline__ void copies_wait() {
  asm volatile("cp.async.wait_group %0;" :: "n"(kLeft) : "memory");
}

// A thread's part of the rows on their way: pieces of 16 bytes, a thread's next to its
// neighbours'.  Each thread reads what it copied itself, so that nothing waits for
// other threads.
template <class TG, class TH, int kN>
struct RowRing {
  static constexpr int kG = kN * (int)sizeof(TG) / 2, kH = kN * (int)sizeof(TH) / 2;
  static constexpr int kPieces = kG + 2 * kH;          // grad_out, h, grad_in
  uint4* at;                  // of the thread, in the first stage
  int threads;

  __device__ __forceinline__ uint4* piece(int stage, int k) const {
    return at + (stage * kPieces + k) * threads;
  }
  template <class T>
  __device__ __forceinline__ void fetch(int stage, int first, const T* row,
                                        const Place& p) const {
    constexpr int kEach = sizeof(T) / 2;
#pragma unroll
    for (int i = 0; i < kN; ++i)
      if (has<true>(p, i, 0)) {
        const T* from = row + column<true>(p, i, 0);
#pragma unroll
        for (int e = 0; e < kEach; ++e)
          copy16<kEach == 2>(piece(stage, first + i * kEach + e),
                             from + e * (8 / kEach));
      }
  }
  template <class T>
  __device__ __forceinline__ void get(int stage, int first, int i, bool present,
                                      Two (&x)[4]) const {
    constexpr int kEach = sizeof(T) / 2;
    Eight<T> e;
    e.clear();
    if (present) {
      uint4 v[kEach];
#pragma unroll
      for (int k = 0; k < kEach; ++k) v[k] = *piece(stage, first + i * kEach + k);
      e.load(reinterpret_cast<const T*>(v));
    }
    e.get(x);
  }
};

constexpr int ctas_by_registers(int eights, bool vec) {  // of 128 threads, on an SM
  return !vec ? (eights == 1 ? 5 : 3) : eights == 1 ? 8 : eights == 2 ? 5 : 4;
}

// A CTA's sums of dw's terms, each thread's in dw, into its row of the parts; shared:
// eight floats for each of a thread's groups.
template <int kN, bool kWide, bool kVec>
__device__ __forceinline__ void leave_part(const NormGradArgs& a,
                                           const float (&dw)[kN][8], int lanes,
                                           float* shared) {
  float* part = a.part + (int64_t)blockIdx.x * a.width;
  const Place p = place<kVec, kWide, kN>(lanes, a.width, true);
  if (kWide) {
#pragma unroll
    for (int i = 0; i < kN; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (has<kVec>(p, i, j)) part[column<kVec>(p, i, j)] = dw[i][j];
    return;
  }
  // the groups of lanes one after another
  const int each = lanes * 8 * kN, group = threadIdx.x / lanes;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kN; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j)
      shared[group * each + column<kVec>(p, i, j)] = dw[i][j];
  __syncthreads();
  for (int c = threadIdx.x; c < a.width; c += kNormThreads) {
    float s = shared[c];
    for (int k = 1; k < kNormThreads / lanes; ++k) s += shared[k * each + c];
    part[c] = s;
  }
}

// Rows that can be taken 16 bytes at a time.  They pass through a ring of two in shared
// memory, so that a row is on its way while the one in front is worked on, and are
// worked on two numbers at a time.  Bound by memory: 65,536 x 1,024 in bf16 in 85 us, 6.3
// TB/s (119 with rows loaded into registers when they are wanted, 100 one number at a
// time, 112 so with a ring of three).
template <class TG, class TH, int kN, bool kWide>
__global__ void __launch_bounds__(kWide ? 32 * kNormMostWarps : kNormThreads,
                                  kWide ? 1 : ctas_by_registers(kN, true))
norm_grad_ring_kernel(const NormGradArgs a) {
  __shared__ float2 sums[2][kNormMostWarps];
  // weights that registers have no room for
  constexpr bool kKept = kN <= 2;
  __shared__ float4 weights[kKept ? 1 : 32 * kN * 2];
  extern __shared__ uint4 ring_memory[];
  // (more than one group a lane: a whole warp has the row)
  const int lanes = kWide || kN > 1 ? 32 : a.lanes;
  const int rows = kWide ? 1 : kNormThreads / lanes;      // of the CTA
  const int64_t step = (int64_t)gridDim.x * rows;
  typedef RowRing<TG, TH, kN> Ring;
  const Ring ring = {ring_memory + threadIdx.x, (int)blockDim.x};
  const auto fetch = [&](int stage, int64_t row) {
    const Place p = place<true, kWide, kN>(lanes, a.width, row < a.rows);
    ring.fetch(stage, 0, static_cast<const TG*>(a.dy) + row * a.dy_stride, p);
    ring.fetch(stage, Ring::kG, static_cast<const TH*>(a.h) + row * a.h_stride, p);
    if (a.dh_in)
      ring.fetch(stage, Ring::kG + Ring::kH,
                 static_cast<const TH*>(a.dh_in) + row * a.dh_in_stride, p);
    copies_end();
  };
  int64_t row = (int64_t)blockIdx.x * rows + (kWide ? 0 : threadIdx.x / lanes);
  fetch(0, row);
  Two kept[kKept ? kN : 1][4];
  const Place all = place<true, kWide, kN>(lanes, a.width, true);
  if (kKept) {
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      float w[8];
      weight8<true>(a.weight, a.weight_bf16, all, i, w);
#pragma unroll
      for (int j = 0; j < 4; ++j) kept[kKept ? i : 0][j] = two(w[2 * j], w[2 * j + 1]);
    }
  } else {
    // [group][half][lane]
    if (threadIdx.x < 32) {
#pragma unroll
      for (int i = 0; i < kN; ++i) {
        float w[8];
        weight8<true>(a.weight, a.weight_bf16, all, i, w);
        weights[(2 * i) * 32 + threadIdx.x] = make_float4(w[0], w[1], w[2], w[3]);
        weights[(2 * i + 1) * 32 + threadIdx.x] = make_float4(w[4], w[5], w[6], w[7]);
      }
    }
    __syncthreads();
  }
  const auto weight = [&](int i, Two (&w)[4]) {
    if (kKept) {
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = kept[kKept ? i : 0][j];
    } else {
      Eight<float> e;
      e.a = weights[(2 * i) * 32 + (threadIdx.x & 31)];
      e.b = weights[(2 * i + 1) * 32 + (threadIdx.x & 31)];
      e.get(w);
    }
  };
  const Two zero = two(0.f, 0.f);
  Two dw[kN][4];
#pragma unroll
  for (int i = 0; i < kN; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) dw[i][j] = zero;
  int stage = 0;
  for (int64_t row0 = (int64_t)blockIdx.x * rows; row0 < a.rows;
       row0 += step, row += step, stage ^= 1) {
    const Place p = place<true, kWide, kN>(lanes, a.width, row < a.rows);
    fetch(stage ^ 1, row + step);
    copies_wait<1>();
    Two hh2 = zero, gh2 = zero;
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      Two w[4], h[4], g[4];
      const bool present = has<true>(p, i, 0);
      weight(i, w);
      ring.template get<TH>(stage, Ring::kG, i, present, h);
      ring.template get<TG>(stage, 0, i, present, g);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        hh2 = fma2(h[j], h[j], hh2);
        gh2 = fma2(mul2(g[j], w[j]), h[j], gh2);
      }
    }
    float hh, gh, more;
    apart(hh2, hh, more);
    hh += more;
    apart(gh2, gh, more);
    gh += more;
    over_row2<kWide>(hh, gh, lanes, sums, stage);
    const float r = rsqrtf(fmaf(hh, a.inv_width, a.eps));
    const float c = correction(gh, r, a.inv_width);
    const Two r2 = two(r, r), minus_rc2 = two(-r * c, -r * c);
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      Two w[4], h[4], g[4], in[4];
      const bool present = has<true>(p, i, 0);
      weight(i, w);
      ring.template get<TH>(stage, Ring::kG, i, present, h);
      ring.template get<TG>(stage, 0, i, present, g);
      if (a.dh_in) {
        ring.template get<TH>(stage, Ring::kG + Ring::kH, i, present, in);
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) in[j] = zero;
      }
      float out[8];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        // (zeros where there is no such column or row)
        dw[i][j] = fma2(g[j], mul2(h[j], r2), dw[i][j]);
        apart(fma2(h[j], minus_rc2, fma2(mul2(g[j], w[j]), r2, in[j])), out[2 * j],
              out[2 * j + 1]);
      }
      Group<TH, true> e;
      e.set(out);
      e.store(static_cast<TH*>(a.dh) + row * a.dh_stride, p, i);
    }
  }
  copies_wait<0>();
  if (!a.part) return;
  float sum[kN][8];
#pragma unroll
  for (int i = 0; i < kN; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) apart(dw[i][j], sum[i][2 * j], sum[i][2 * j + 1]);
  // (the ring has the room)
  leave_part<kN, kWide, true>(a, sum, lanes, reinterpret_cast<float*>(ring_memory));
}

// Other rows are loaded into registers, column by column, when they are wanted: 30,000 x
// 757 in bf16 66 us, 2.7 TB/s.
template <class TG, class TH, int kN, bool kWide>
__global__ void __launch_bounds__(kWide ? 32 * kNormMostWarps : kNormThreads,
                                  kWide ? 1 : ctas_by_registers(kN, false))
norm_grad_rows_kernel(const NormGradArgs a) {
  __shared__ float2 sums[2][kNormMostWarps];
  __shared__ float joined[kWide ? 1 : kNormThreads * 8 * kN];
  // (more than one group a lane: a whole warp has the row)
  const int lanes = kWide || kN > 1 ? 32 : a.lanes;
  const int rows = kWide ? 1 : kNormThreads / lanes;      // of the CTA
  const int64_t step = (int64_t)gridDim.x * rows;
  float dw[kN][8];
#pragma unroll
  for (int i = 0; i < kN; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) dw[i][j] = 0.f;
  int turn = 0;
  for (int64_t row0 = (int64_t)blockIdx.x * rows; row0 < a.rows; row0 += step) {
    const int64_t row = row0 + (kWide ? 0 : threadIdx.x / lanes);
    const Place p = place<false, kWide, kN>(lanes, a.width, row < a.rows);
    Group<TG, false> eg[kN];
    Group<TH, false> eh[kN], ei[kN];
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      eh[i].load(static_cast<const TH*>(a.h) + row * a.h_stride, p, i);
      eg[i].load(static_cast<const TG*>(a.dy) + row * a.dy_stride, p, i);
    }
    if (a.dh_in) {
#pragma unroll
      for (int i = 0; i < kN; ++i)
        ei[i].load(static_cast<const TH*>(a.dh_in) + row * a.dh_in_stride, p, i);
    }
    float hh = 0.f, gh = 0.f;
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      float w[8], h[8], g[8];
      weight8<false>(a.weight, a.weight_bf16, p, i, w);
      eh[i].get(h);
      eg[i].get(g);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        hh = fmaf(h[j], h[j], hh);
        gh = fmaf(g[j] * w[j], h[j], gh);
      }
    }
    over_row2<kWide>(hh, gh, lanes, sums, turn);
    turn ^= 1;
    const float r = rsqrtf(fmaf(hh, a.inv_width, a.eps));
    const float c = correction(gh, r, a.inv_width);
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      float w[8], h[8], g[8], in[8];
      weight8<false>(a.weight, a.weight_bf16, p, i, w);
      eh[i].get(h);
      eg[i].get(g);
      if (a.dh_in) ei[i].get(in);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        // (zeros where there is no such column or row)
        dw[i][j] = fmaf(g[j], h[j] * r, dw[i][j]);
        h[j] = fmaf(h[j], -r * c, fmaf(g[j] * w[j], r, a.dh_in ? in[j] : 0.f));
      }
      eh[i].set(h);
      eh[i].store(static_cast<TH*>(a.dh) + row * a.dh_stride, p, i);
    }
  }
  if (a.part) leave_part<kN, kWide, false>(a, dw, lanes, joined);
}

// Rows that do not fit a CTA's registers: two looks at memory a row, and dw's sums in
// the CTA's row of parts.  4,096 x 16,384 in bf16 671 us, 0.8 TB/s of bytes that it cannot
// do without.
template <class TG, class TH>
__global__ void __launch_bounds__(kNormWalk) norm_grad_walk_kernel(
    const NormGradArgs a) {
  __shared__ float2 sums[2][kNormMostWarps];
  float* part = a.part ? a.part + (int64_t)blockIdx.x * a.width : nullptr;
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const TG* dy = static_cast<const TG*>(a.dy) + row * a.dy_stride;
    const TH* h = static_cast<const TH*>(a.h) + row * a.h_stride;
    const TH* in = static_cast<const TH*>(a.dh_in) + row * a.dh_in_stride;
    TH* dh = static_cast<TH*>(a.dh) + row * a.dh_stride;
    float hh = 0.f, gh = 0.f;
    for (int c = threadIdx.x; c < a.width; c += kNormWalk) {
      const float x = get1(h + c);
      const float w = weight1(a.weight, a.weight_bf16, c);
      hh = fmaf(x, x, hh);
      gh = fmaf(get1(dy + c) * w, x, gh);
    }
    over_row2<true>(hh, gh, 32, sums, turn);
    turn ^= 1;
    const float r = rsqrtf(fmaf(hh, a.inv_width, a.eps));
    const float k = correction(gh, r, a.inv_width);
    for (int c = threadIdx.x; c < a.width; c += kNormWalk) {
      const float x = get1(h + c), g = get1(dy + c);
      const float w = weight1(a.weight, a.weight_bf16, c);
      float d = r * (g * w - k * x);
      if (a.dh_in) d += get1(in + c);
      if (part) {
        const float before = row == blockIdx.x ? 0.f : part[c];
        part[c] = fmaf(g, x * r, before);
      }
      put1(dh + c, d);
    }
  }
}

// dw (+)= the parts, a warp every 32nd of them, then the warps in order.
template <class TW>
__global__ void __launch_bounds__(kJoinThreads) norm_grad_join_kernel(
    const float* part, int parts, int width, TW* dw, int accumulate) {
  __shared__ float shared[kJoinThreads / 32][kJoinColumns];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int c = blockIdx.x * kJoinColumns + lane;
  after_prior_launch();
  float s = 0.f;
  if (c < width) {
    constexpr int kAhead = 10;          // loads of a thread in flight
    for (int k0 = warp; k0 < parts; k0 += kAhead * (kJoinThreads / 32)) {
      float v[kAhead];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const int k = k0 + i * (kJoinThreads / 32);
        v[i] = k < parts ? part[(int64_t)k * width + c] : 0.f;
      }
#pragma unroll
      for (int i = 0; i < kAhead; ++i) s += v[i];
    }
  }
  shared[warp][lane] = s;
  __syncthreads();
  if (warp || c >= width) return;
  s = accumulate ? get1(dw + c) : 0.f;
  float t = 0.f;
#pragma unroll
  for (int k = 0; k < kJoinThreads / 32; ++k) t += shared[k][lane];
  put1(dw + c, s + t);
}

struct GradKernel {
  void (*run)(NormGradArgs);
  int smem;                   // dynamic, of a thread
  int registers;              // CTAs of 128 threads that an SM has registers for
};
template <class TG, class TH, int kN, bool kWide>
GradKernel grad_ring() {
  return {norm_grad_ring_kernel<TG, TH, kN, kWide>,
          2 * RowRing<TG, TH, kN>::kPieces * 16,
          kWide ? 4 : ctas_by_registers(kN, true)};
}
template <class TG, class TH, int kN, bool kWide>
GradKernel grad_rows() {
  return {norm_grad_rows_kernel<TG, TH, kN, kWide>, 0,
          kWide ? 4 : ctas_by_registers(kN, false)};
}
template <class TG, class TH>
GradKernel grad_kernel(const NormLayout& l) {
  if (l.walk) return {norm_grad_walk_kernel<TG, TH>, 0, 8};
  if (!l.vec)
    return l.wide          ? grad_rows<TG, TH, kWideEights, true>()
           : l.eights == 1 ? grad_rows<TG, TH, 1, false>()
                           : grad_rows<TG, TH, 2, false>();
  return l.wide          ? grad_ring<TG, TH, kWideEights, true>()
         : l.eights == 1 ? grad_ring<TG, TH, 1, false>()
         : l.eights == 2 ? grad_ring<TG, TH, 2, false>()
                         : grad_ring<TG, TH, 4, false>();
}
GradKernel grad_kernel_of(const NormLayout& l, bool g16, bool h16) {
  typedef __nv_bfloat16 bf;
  return g16 ? (h16 ? grad_kernel<bf, bf>(l) : grad_kernel<bf, float>(l))
             : (h16 ? grad_kernel<float, bf>(l)
                    : grad_kernel<float, float>(l));
}

// A warp's row has four groups a lane where all of it is bf16; two where fp32 rows take
// twice the ring (65,536 x 768 in fp32: 159 us with four), or columns one by one more
// registers.
NormLayout grad_layout(int width, bool vec, bool bf16) {
  return norm_layout(width, vec, 1, vec && bf16 ? kNormEights : 2, kWideEights);
}

}  // namespace

// Shared-memory limits on the current device of the kernels for a width.  A limit is
// its kernel's, and one for all plans: a CTA's rows are of many widths, so that theirs is
// what the widest ones need (fp32: 196,608 bytes).
cudaError_t norm_grad_setup(int width) {
  cudaError_t e = cudaSuccess;
  for (int t = 0; t < 4 && e == cudaSuccess; ++t) {
    const NormLayout l = grad_layout(width, true, t == 3);
    const GradKernel k = grad_kernel_of(l, t & 1, t & 2);
    const int most_threads = l.wide ? 32 * kNormMostWarps : kNormThreads;
    if (k.smem)
      e = cudaFuncSetAttribute(k.run, cudaFuncAttributeMaxDynamicSharedMemorySize,
                               k.smem * most_threads);
  }
  return e;
}

}  // namespace lamb

using namespace lamb;

extern "C" lamb_status_t lamb_norm_grad(
    struct lamb_norm* v, const void* grad_out, int32_t grad_dtype,
    int64_t grad_stride, const void* total, int64_t total_stride,
    const void* grad_in, int64_t grad_in_stride, void* grad_total,
    int64_t grad_total_stride, int32_t total_dtype, const void* weight,
    int32_t weight_dtype, int64_t n_rows, void* weight_grad,
    int32_t weight_grad_dtype, int32_t accumulate, cudaStream_t stream) {
  lamb_status_t st = norm_check(v, n_rows);
  if (st != LAMB_OK) return st;
  if (weight)
    if ((st = norm_check_vector("weight", weight, weight_dtype)) != LAMB_OK)
      return st;
  if (weight_grad)
    if ((st = norm_check_vector("weight_grad", weight_grad,
                                weight_grad_dtype)) != LAMB_OK)
      return st;
  const LmRows dy = {"grad_out", grad_out, grad_dtype, grad_stride},
               h = {"total", total, total_dtype, total_stride},
               in = {"grad_in", grad_in, total_dtype, grad_in_stride},
               dh = {"grad_total", grad_total, total_dtype, grad_total_stride};
  if (n_rows) {
    if ((st = norm_check_rows(v, dy, false)) != LAMB_OK ||
        (st = norm_check_rows(v, h, false)) != LAMB_OK ||
        (grad_in && (st = norm_check_rows(v, in, false)) != LAMB_OK) ||
        (st = norm_check_rows(v, dh, false)) != LAMB_OK)
      return st;
  }
  LmDevice dev(v->device);
  if (dev.err != cudaSuccess) return lm_cuda_fail(dev.err, "cudaSetDevice");
  int parts = 0;
  if (n_rows) {
    NormGradArgs a = {};
    a.dy = grad_out;
    a.h = total;
    a.weight = weight;
    a.dh_in = grad_in;
    a.dh = grad_total;
    a.part = weight_grad ? v->part : nullptr;
    a.dy_stride = grad_stride;
    a.h_stride = total_stride;
    a.dh_in_stride = grad_in_stride;
    a.dh_stride = grad_total_stride;
    a.rows = n_rows;
    a.width = v->width;
    a.weight_bf16 = weight_dtype == LAMB_BF16;
    a.eps = v->eps;
    a.inv_width = (float)(1. / v->width);
    const bool vec = v->width % 8 == 0 && ((uintptr_t)weight & 15) == 0 &&
                     norm_vec(grad_out, grad_dtype, grad_stride) &&
                     norm_vec(total, total_dtype, total_stride) &&
                     norm_vec(grad_total, total_dtype, grad_total_stride) &&
                     (!grad_in || norm_vec(grad_in, total_dtype, grad_in_stride));
    const bool g16 = grad_dtype == LAMB_BF16, h16 = total_dtype == LAMB_BF16;
    const NormLayout l = grad_layout(v->width, vec, g16 && h16);
    a.lanes = l.lanes;
    const GradKernel k = grad_kernel_of(l, g16, h16);
    const int smem = k.smem * l.threads;
    // as many CTAs as are resident at a time
    int per_sm = k.registers * kNormThreads / l.threads;
    if (smem) per_sm = std::min(per_sm, 226 * 1024 / (smem + 1024));
    per_sm = std::max(per_sm, 1);
    parts = (int)std::min<int64_t>(lm_ceil_div(n_rows, l.rows),
                                   std::min(per_sm * v->sms, v->max_parts));
    const cudaError_t e =
        lm_launch(k.run, parts, l.threads, smem, stream, false, a);
    if (e != cudaSuccess) return lm_cuda_fail(e, "norm gradient launch");
  }
  if (!weight_grad || (!parts && accumulate)) return LAMB_OK;
  const unsigned grid = (unsigned)lm_ceil_div(v->width, kJoinColumns);
  const cudaError_t e =
      weight_grad_dtype == LAMB_F32
          ? lm_launch(norm_grad_join_kernel<float>, grid, kJoinThreads, 0, stream,
                      true, v->part, parts, v->width, (float*)weight_grad,
                      accumulate)
          : lm_launch(norm_grad_join_kernel<__nv_bfloat16>, grid, kJoinThreads, 0,
                      stream, true, v->part, parts, v->width,
                      (__nv_bfloat16*)weight_grad, accumulate);
  return e == cudaSuccess ? LAMB_OK : lm_cuda_fail(e, "norm gradient join");
}
