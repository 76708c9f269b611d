// Orthogonalised (Muon) update of matrices.
//
//   m <- beta m + (1 - beta) g,  u = (1 - beta) g + beta m  (Nesterov) or m
//   X = u / (|u|_F + eps); `steps` times, with G the Gram matrix of X's shorter
//   side:  X <- a X + (b G + c G G) X      (X (b G + c G G) for a tall X)
//   w <- (1 - eta lambda) w - eta s X
//
// Three products a step on the tensor cores (lm_gemm.cuh), in fp16 with fp32
// accumulators.  Eleven significant bits are enough only where the large terms
// stay out of the rounding, so
//   X is a pair of halves hi + lo (22 bits; the products read hi),
//   G is kept as its diagonal in fp32 and the rest D in fp16, and so is
//   b G + c G G = diag(beta) + E:  with G = diag(l) + D,
//     E_ij = b D_ij + c ((l_i + l_j) D_ij + (D D)_ij),   i != j
//     beta_i = b l_i + c (l_i^2 + (D D)_ii)
//   and X <- (a + beta_i) X + E X takes X whole from the pair.
// The direction is then within 3e-4 .. 1e-3 of the exact one (Gaussian, low-rank
// and power-law spectra, 10 x 10 to 1536 x 1600; up to 4.4e-3 where all entries are
// equal or the rank is one, at short sides of 100 to 300): half a bf16 rounding; with G
// rounded as it is, 1.7e-3 .. 1.2e-2, in bf16 1.3e-2 .. 1e-1.  Scales that are
// powers of two keep the entries inside fp16's range.
//
// lm_muon_steps.cu multiplies; here are the momentum and the norm in front of it,
// small matrices, and the plan.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>
#include <vector>

#include "lm_muon.h"

namespace lamb {
namespace {

constexpr int kMuonThreads = 256;
constexpr int kMuonChunk = 8192;             // elements of a chunk
// ---- momentum and norm --------------------------------------------------------
template <class TG>
__device__ __forceinline__ float load_grad(const void* p, int64_t i);
template <>
__device__ __forceinline__ float load_grad<float>(const void* p, int64_t i) {
  return reinterpret_cast<const float*>(p)[i];
}
template <>
__device__ __forceinline__ float load_grad<__nv_bfloat16>(const void* p,
                                                          int64_t i) {
  return __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(p)[i]);
}

__device__ __forceinline__ float update_of(const MuonConsts& k, float g,
                                           float m) {
  return k.nesterov ? fmaf(k.beta, m, k.omb * g) : m;
}

// Sum over a CTA, in thread 0: each warp's in fp32, the warps' in fp64.
template <int kThreads>
__device__ __forceinline__ double block_sum(float s, float* sh) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = s;
  __syncthreads();
  double d = 0.0;
  if (threadIdx.x == 0)
    for (int i = 0; i < kThreads / 32; ++i) d += (double)sh[i];
  return d;
}

// Four consecutive values (kVec: by one access; else n of them).
template <class TG, bool kVec>
__device__ __forceinline__ void load_grads(const void* p, int64_t i, int n,
                                           float (&x)[4]) {
  if (kVec && sizeof(TG) == 4) {
    const float4 v = *reinterpret_cast<const float4*>(
        reinterpret_cast<const float*>(p) + i);
    x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
  } else if (kVec) {
    const uint2 v = *reinterpret_cast<const uint2*>(
        reinterpret_cast<const __nv_bfloat16*>(p) + i);
    x[0] = __uint_as_float(v.x << 16);
    x[1] = __uint_as_float(v.x & 0xffff0000u);
    x[2] = __uint_as_float(v.y << 16);
    x[3] = __uint_as_float(v.y & 0xffff0000u);
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = k < n ? load_grad<TG>(p, i + k) : 0.f;
  }
}

// What a vector access needs of a chunk (chunks start at multiples of 4).
template <class TG, bool kStep>
__device__ __forceinline__ bool chunk_vec(const MuonPtrs& p, int len) {
  return len % 4 == 0 && (uintptr_t)p.g % (4 * sizeof(TG)) == 0 &&
         (!kStep || (uintptr_t)p.m % 16 == 0);
}

template <class TG, bool kStep, bool kVec>
__device__ __forceinline__ float norm_chunk(const MuonPtrs& p,
                                            const MuonChunk& c,
                                            const MuonConsts& k) {
  float s = 0.f;
#pragma unroll 4
  for (int i = threadIdx.x * 4; i < c.len; i += kMuonThreads * 4) {
    const int64_t at = c.offset + i;
    const int n = min(4, c.len - i);
    float u[4];
    load_grads<TG, kVec>(p.g, at, n, u);
    if (kStep) {
      float m[4];
      load_grads<float, kVec>(p.m, at, n, m);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        m[q] = fmaf(k.beta, m[q], k.omb * u[q]);
        u[q] = update_of(k, u[q], m[q]);
      }
      if (kVec) {
        *reinterpret_cast<float4*>(p.m + at) =
            make_float4(m[0], m[1], m[2], m[3]);
      } else {
#pragma unroll
        for (int q = 0; q < 4; ++q)
          if (q < n) p.m[at + q] = m[q];
      }
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) s = fmaf(u[q], u[q], s);
  }
  return s;
}

// New momentum (kStep) and the sum of squares of a chunk's u.
template <class TG, bool kStep>
__global__ void __launch_bounds__(kMuonThreads)
muon_norm_kernel(const MuonPtrs* ptrs, const MuonChunk* chunks, MuonConsts k,
                 double* part) {
  __shared__ float sh[kMuonThreads / 32];
  const MuonChunk c = chunks[blockIdx.x];
  const MuonPtrs p = ptrs[c.matrix];
  const float s = chunk_vec<TG, kStep>(p, c.len)
                      ? norm_chunk<TG, kStep, true>(p, c, k)
                      : norm_chunk<TG, kStep, false>(p, c, k);
  const double sum = block_sum<kMuonThreads>(s, sh);
  if (threadIdx.x == 0) part[blockIdx.x] = sum;
}

template <class TG, bool kStep, bool kVec>
__device__ __forceinline__ void start_chunk(const MuonMatrix& x,
                                            const MuonPtrs& p,
                                            const MuonChunk& c,
                                            const MuonConsts& k, float f) {
  __half* const hi = x.hi[0];
  __half* const lo = x.lo;
  const int cols = x.cols, pitch = x.pitch;
#pragma unroll 4
  for (int i = threadIdx.x * 4; i < c.len; i += kMuonThreads * 4) {
    const int64_t at = c.offset + i;
    const int n = min(4, c.len - i);
    float u[4];
    load_grads<TG, kVec>(p.g, at, n, u);
    if (kStep) {
      float m[4];
      load_grads<float, kVec>(p.m, at, n, m);
#pragma unroll
      for (int q = 0; q < 4; ++q) u[q] = update_of(k, u[q], m[q]);
    }
    uint32_t h[2], l[2];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const float a = u[2 * q] * f, b = u[2 * q + 1] * f;
      h[q] = pack_half2(a, b);
      const float2 r = half2_at(h[q]);
      l[q] = pack_half2((a - r.x) * kScaleLo, (b - r.y) * kScaleLo);
    }
    if (kVec && pitch == cols) {
      *reinterpret_cast<uint2*>(hi + at) = make_uint2(h[0], h[1]);
      *reinterpret_cast<uint2*>(lo + at) = make_uint2(l[0], l[1]);
    } else {
      int64_t r = at / cols;
      int col = (int)(at - r * cols);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if (q >= n) break;
        const int64_t to = r * pitch + col;
        hi[to] = __ushort_as_half(half_bits(h[q >> 1], q & 1));
        lo[to] = __ushort_as_half(half_bits(l[q >> 1], q & 1));
        if (++col == cols) {
          col = 0;
          ++r;
        }
      }
    }
  }
}

// X = u / (|u| + eps) as a pair of halves.
template <class TG, bool kStep>
__global__ void __launch_bounds__(kMuonThreads)
muon_start_kernel(const MuonMatrix* mats, const MuonPtrs* ptrs,
                  const MuonChunk* chunks, MuonConsts k, const double* part,
                  uint32_t* done, uint32_t* status) {
  __shared__ float sh_norm;
  const MuonChunk c = chunks[blockIdx.x];
  const MuonMatrix& x = mats[c.matrix];
  const MuonPtrs p = ptrs[c.matrix];
  if (threadIdx.x < 32) {       // the chunks' sums, in a fixed order
    double s = 0.0;
    for (int i = threadIdx.x; i < x.n_chunks; i += 32)
      s += part[x.first_chunk + i];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (threadIdx.x == 0) {
      const float n = sqrtf((float)s);
      sh_norm = n;
      if (!isfinite(n)) atomicOr(status, LAMB_STATUS_NONFINITE);
      if (c.offset == 0) done[c.matrix] = 0;       // of the products to come
    }
  }
  __syncthreads();
  const float norm = sh_norm;
  const float f = x.scale / (norm + k.eps);
  if (chunk_vec<TG, kStep>(p, c.len))
    start_chunk<TG, kStep, true>(x, p, c, k, f);
  else
    start_chunk<TG, kStep, false>(x, p, c, k, f);
}

// ---- small matrices ------------------------------------------------------------
// A matrix whose X fits in shared memory twice goes through all of its steps in
// one CTA, in fp32 on the CUDA cores: momentum, norm, products, update.  A chain
// of launches on the tensor cores costs some 15 launches' latency, and an entry of
// a tiny matrix is too few terms for its 11-bit roundings to average out.
constexpr int kSmallThreads = 512;
constexpr int kSmallSide = 64;               // m up to
constexpr int64_t kSmallElems = 20480;       // m n up to
constexpr int64_t kSmallProduct = 1 << 19;   // m m n up to

bool muon_is_small(int64_t m, int64_t n) {
  return m <= kSmallSide && m * n <= kSmallElems && m * m * n <= kSmallProduct;
}
// Rows of X: on 16 bytes, and four rows on at other banks.
__host__ __device__ constexpr int64_t small_pitch(int64_t n) {
  return (n + 3) / 4 * 4 + ((n + 3) / 4 % 2 ? 0 : 4);
}
int64_t small_smem(int64_t m, int64_t n) {
  return (m * lm_round_up(m, 4) + m * lm_round_up(m | 1, 4) +
          2 * m * small_pitch(n)) * 4;
}
// What no such matrix passes (a row's pitch is at most seven elements above it).
// The kernel's limit belongs to the device, not to a plan: it is always this.
constexpr int kSmallSmem =
    (kSmallSide * kSmallSide + kSmallSide * (kSmallSide + 4) +
     2 * ((int)kSmallElems + 7 * kSmallSide)) * 4;
static_assert(kSmallSmem <= 227 * 1024 - 2048, "a CTA's shared memory");

// out = b in + c (in in^T), or in in^T (kPlain), both symmetric: blocks of 4 x 4
// (the task's places are in `where`), each by 16 neighbouring lanes that take
// every 16th k.  Their sums are exchanged so that each lane ends with one entry.
template <bool kPlain>
__device__ __forceinline__ void small_gram(const float* in, int pitch, int m,
                                           int n, float b, float c, float* out,
                                           int out_pitch, const uint16_t* where,
                                           int tasks) {
  const int s = threadIdx.x & 15;
  for (int base = 0; base < tasks; base += kSmallThreads / 16) {
    const int task = base + (threadIdx.x >> 4);
    const int w = where[min(task, tasks - 1)];
    const int i0 = 4 * (w >> 8), j0 = 4 * (w & 255);
    const float *ri[4], *rj[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      ri[q] = in + min(i0 + q, m - 1) * pitch;
      rj[q] = in + min(j0 + q, m - 1) * pitch;
    }
    float acc[16] = {};
#pragma unroll 4
    for (int k = s; k < n; k += 16) {
      float x[4], y[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        x[q] = ri[q][k];
        y[q] = rj[q][k];
      }
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int v = 0; v < 4; ++v)
          acc[4 * u + v] = fmaf(x[u], y[v], acc[4 * u + v]);
    }
#pragma unroll
    for (int h = 8; h > 0; h >>= 1) {
      const bool up = s & h;
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        if (q >= h) break;
        const float send = up ? acc[q] : acc[q + h];
        const float keep = up ? acc[q + h] : acc[q];
        acc[q] = keep + __shfl_xor_sync(0xffffffffu, send, h);
      }
    }
    const int i = i0 + (s >> 2), j = j0 + (s & 3);
    if (task < tasks && i < m && j < m) {
      const float r =
          kPlain ? acc[0] : fmaf(b, in[i * pitch + j], c * acc[0]);
      out[i * out_pitch + j] = r;
      out[j * out_pitch + i] = r;
    }
  }
}

template <class TG, bool kStep>
__global__ void __launch_bounds__(kSmallThreads)
muon_small_kernel(const MuonMatrix* mats, const MuonPtrs* ptrs,
                  const int* which, MuonConsts k, int steps, const float* d_lr,
                  uint32_t* status) {
  extern __shared__ float sm[];
  __shared__ float sh[kSmallThreads / 32], sh_norm;
  __shared__ uint16_t where[kSmallSide / 4 * (kSmallSide / 4 + 1) / 2];
  const MuonMatrix& x = mats[which[blockIdx.x]];
  const MuonPtrs p = ptrs[which[blockIdx.x]];
  const int m = x.m, n = x.n, cols = x.cols, total = m * n;
  // (a warp's lanes are at several rows of X and G at a time)
  const int np = (int)small_pitch(n), gp = m | 1, mp = (m + 3) & ~3;
  const bool tall = x.tall;
  float *H = sm, *G = H + m * mp, *X = G + m * ((gp + 3) & ~3), *Y = X + m * np;
  for (int i = threadIdx.x; i < m * mp; i += kSmallThreads) H[i] = 0.f;
  const int nb = (m + 3) >> 2, blocks = nb * (nb + 1) / 2;
  if (threadIdx.x < nb)       // the blocks on and above the diagonal
    for (int j = threadIdx.x, t = threadIdx.x * nb -
                                  threadIdx.x * ((int)threadIdx.x - 1) / 2;
         j < nb; ++j, ++t)
      where[t] = (uint16_t)(threadIdx.x << 8 | j);

  float s = 0.f;
  for (int i = threadIdx.x; i < total; i += kSmallThreads) {
    float u = load_grad<TG>(p.g, i);
    if (kStep) {
      const float mm = fmaf(k.beta, p.m[i], k.omb * u);
      p.m[i] = mm;
      u = update_of(k, u, mm);
    }
    s = fmaf(u, u, s);
    const int r = i / cols, c = i - r * cols;
    X[tall ? c * np + r : r * np + c] = u;
  }
  const double d = block_sum<kSmallThreads>(s, sh);
  if (threadIdx.x == 0) {
    sh_norm = sqrtf((float)d);
    if (!isfinite(sh_norm)) atomicOr(status, LAMB_STATUS_NONFINITE);
  }
  __syncthreads();
  const float norm = sh_norm;
  const float f = 1.f / (norm + k.eps);
  for (int i = threadIdx.x; i < total; i += kSmallThreads) {
    const int r = i / n;
    X[r * np + (i - r * n)] *= f;
  }
  __syncthreads();

  for (int it = 0; it < steps; ++it) {
    small_gram<true>(X, np, m, n, 0.f, 0.f, G, gp, where, blocks);
    __syncthreads();
    small_gram<false>(G, gp, m, m, k.b, k.c, H, mp, where, blocks);
    __syncthreads();
    // Y = a X + H X, 4 x 4 entries a thread: two 16-byte loads for 16 products
    // (four rows of one column were bound by shared memory)
    const int nc = (n + 3) >> 2, tasks = nb * nc;
    for (int t = threadIdx.x; t < tasks; t += kSmallThreads) {
      const int i0 = t / nc * 4, j0 = t % nc * 4;
      float acc[4][4] = {};
#pragma unroll 4
      for (int q = 0; q < m; ++q) {
        const float4 x = *reinterpret_cast<const float4*>(X + q * np + j0);
        const float4 h = *reinterpret_cast<const float4*>(H + q * mp + i0);
        const float hv[4] = {h.x, h.y, h.z, h.w};
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          acc[u][0] = fmaf(hv[u], x.x, acc[u][0]);
          acc[u][1] = fmaf(hv[u], x.y, acc[u][1]);
          acc[u][2] = fmaf(hv[u], x.z, acc[u][2]);
          acc[u][3] = fmaf(hv[u], x.w, acc[u][3]);
        }
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (i0 + u >= m) break;
        const int at = (i0 + u) * np + j0;
        const float4 x = *reinterpret_cast<const float4*>(X + at);
        *reinterpret_cast<float4*>(Y + at) =
            make_float4(fmaf(k.a, x.x, acc[u][0]), fmaf(k.a, x.y, acc[u][1]),
                        fmaf(k.a, x.z, acc[u][2]), fmaf(k.a, x.w, acc[u][3]));
      }
    }
    __syncthreads();
    float* z = X;
    X = Y;
    Y = z;
  }

  const float lr = kStep ? *d_lr : 0.f;
  const float size = muon_size(k, x.rows, x.cols);
  const float keep = 1.f - lr * k.wd * x.decay, move = lr * size;
  for (int i = threadIdx.x; i < total; i += kSmallThreads) {
    const int r = i / cols, c = i - r * cols;
    float v = X[tall ? c * np + r : r * np + c];
    if (kStep) {
      v = keep * p.w[i] - move * v;
      p.w[i] = v;
    }
    if (p.out) p.out[i] = __float2bfloat16_rn(v);
  }
}

template <class TG, bool kStep>
cudaError_t allow_small_smem() {
  return cudaFuncSetAttribute(muon_small_kernel<TG, kStep>,
                              cudaFuncAttributeMaxDynamicSharedMemorySize,
                              kSmallSmem);
}

}  // namespace

}  // namespace lamb

using namespace lamb;

struct lamb_muon {
  int device = 0, units = 0, n = 0;
  bool pair = false;                   // tiles by pairs of CTAs
  bool grad_bf16 = false, copy = false;
  bool bound = false, bound_direction = false;
  void* arena = nullptr;
  void* work = nullptr;
  MuonMatrix* mats = nullptr;
  MuonPtrs* ptrs = nullptr;            // of the step
  MuonPtrs* dir_ptrs = nullptr;        // of the direction
  MuonChunk* chunks = nullptr;
  MuonTile* tiles = nullptr;
  uint32_t* done = nullptr;
  double* part = nullptr;
  int* small = nullptr;                // matrices of the small kernel
  int n_small = 0;
  int64_t small_bytes = 0;             // shared memory of the largest
  uint32_t* status = nullptr;
  std::vector<int64_t> numel;
  int n_chunks = 0;
  int64_t step_tiles = 0;              // tiles of one step of all matrices
};

namespace {

// Up to so many tiles of 256 x 256 for a pair of CTAs, the smaller ones are taken.
// Measured (us, the whole call; tiles of 128 | of 256), by tiles for a pair of 76:
//   512 x 512            0.05    115 | 146
//   1024 x 1024          0.2     139 | 184
//   1024 x 4096          0.8     221 | 258
//   9 of 1000 x 500      0.9     184 | 212
//   1536 x 4096          1.3     285 | 330
//   8 of 1024 x 1024     1.7     240 | 239
//   a BERT-large layer   2.5     350 | 353
//   16 of 1024 x 1024    3.4     488 | 373
//   BERT-base            18     2021 | 1690 (the whole step)
constexpr int64_t kSingleTiles = 2;

struct MuonLayout {
  std::vector<MuonMatrix> mats;
  std::vector<MuonChunk> chunks;
  std::vector<MuonTile> tiles;
  std::vector<int> small;
  std::vector<int64_t> at[7];     // byte offsets in the workspace, per matrix
  int64_t work_bytes = 0;
  bool pair = false;
};

int64_t take(int64_t* used, int64_t bytes) {
  const int64_t at = *used;
  *used = lm_round_up(at + bytes, 1024);
  return at;
}

// Workspace offsets, chunks and tiles of the matrices (host only).
void muon_layout(const int64_t* rows, const int64_t* cols, int n,
                 const uint8_t* mask, int pairs, MuonLayout* L) {
  L->mats.resize(n);
  for (auto& v : L->at) v.assign(n, 0);
  std::vector<int> large;
  int64_t used = 0;
  for (int k = 0; k < n; ++k) {
    MuonMatrix& x = L->mats[k];
    memset(&x, 0, sizeof(x));
    x.rows = (int)rows[k];
    x.cols = (int)cols[k];
    x.m = std::min(x.rows, x.cols);
    x.n = std::max(x.rows, x.cols);
    x.tall = x.rows > x.cols;
    x.pitch = (int)lm_round_up(x.cols, 64);   // whole blocks
    x.pitch_m = (int)lm_round_up(x.m, 8);
    x.scale = (float)std::exp2(std::round(0.5 * std::log2((double)std::max(
        1, x.n))));
    x.decay = mask ? (mask[k] ? 1.f : 0.f) : 1.f;
    if (!x.m) continue;
    if (muon_is_small(x.m, x.n)) {
      L->small.push_back(k);
      continue;
    }
    const int64_t sx = (int64_t)x.rows * x.pitch * 2;
    const int64_t sm = (int64_t)x.m * x.pitch_m * 2;
    for (int i = 0; i < 3; ++i) L->at[i][k] = take(&used, sx);
    for (int i = 3; i < 5; ++i) L->at[i][k] = take(&used, sm);
    for (int i = 5; i < 7; ++i) L->at[i][k] = take(&used, x.m * 4ll);
    large.push_back(k);
    x.first_chunk = (int)L->chunks.size();
    const int64_t total = (int64_t)x.rows * x.cols;
    for (int64_t o = 0; o < total; o += kMuonChunk)
      L->chunks.push_back(
          {k, (int)std::min<int64_t>(kMuonChunk, total - o), o});
    x.n_chunks = (int)L->chunks.size() - x.first_chunk;
  }
  L->work_bytes = used;
  if (large.empty()) return;

  // Tiles of 256 x 256 by pairs of CTAs copy half the operands for a product, tiles
  // of 128 x 128 by single ones end sooner and are more: those where the others
  // would be too few.
  int64_t tiles = 0;
  for (int k : large)
    tiles += lm_ceil_div(L->mats[k].rows, 256) *
             lm_ceil_div(L->mats[k].cols, 256);
  L->pair = tiles > kSingleTiles * pairs;
  const int tile = L->pair ? 2 * kMuonRows : kMuonRows;
  for (int k : large) {
    MuonMatrix& x = L->mats[k];
    // a CTA that has no rows of a tile does not count it
    for (int i = 0; i * kMuonRows < x.m; ++i)
      x.sym += (int)lm_ceil_div(x.m, tile) - i * kMuonRows / tile;
    x.app = (int)(lm_ceil_div(x.rows, kMuonRows) * lm_ceil_div(x.cols, tile));
  }

  // two sets of about equal work, the largest matrices first, each to the set that
  // has less so far
  auto work = [&](int k) {
    const MuonMatrix& x = L->mats[k];
    return (double)x.m * x.m * x.n;
  };
  std::stable_sort(large.begin(), large.end(),
                   [&](int p, int q) { return work(p) > work(q); });
  std::vector<int> set[2];
  double load[2] = {0.0, 0.0};
  for (int k : large) {
    const int to = load[1] < load[0];
    set[to].push_back(k);
    load[to] += work(k);
  }
  // the tiles of one step: product by product, the sets in turn, long products
  // first
  for (int phase = kGram; phase <= kApply; ++phase)
    for (std::vector<int>& of : set) {
      std::stable_sort(of.begin(), of.end(), [&](int p, int q) {
        const MuonMatrix &x = L->mats[p], &y = L->mats[q];
        return phase == kGram ? x.n > y.n : x.m > y.m;
      });
      for (int k : of) {
        const MuonMatrix& x = L->mats[k];
        const int r = phase == kApply ? x.rows : x.m;
        const int c = phase == kApply ? x.cols : x.m;
        for (int i = 0; i * tile < r; ++i)
          for (int j = phase == kApply ? 0 : i; j * tile < c; ++j) {
            MuonTile t = {};
            t.matrix = k;
            t.i = i;
            t.j = j;
            t.phase = phase;
            L->tiles.push_back(t);
          }
      }
    }
}

lamb_status_t muon_check(const lamb_muon* p, const lamb_muon_hyper_t* h) {
  if (!p) return lm_fail(LAMB_ERR_INVALID_ARG, "plan is NULL");
  if (!h) return lm_fail(LAMB_ERR_INVALID_ARG, "hyper is NULL");
  const double v[] = {h->momentum, h->weight_decay, h->eps, h->a, h->b, h->c,
                      h->update_scale};
  for (double x : v)
    if (!std::isfinite(x))
      return lm_fail(LAMB_ERR_INVALID_ARG, "hyper: a value is not finite");
  if (h->momentum < 0 || h->momentum >= 1 || h->eps < 0 || h->weight_decay < 0)
    return lm_fail(LAMB_ERR_INVALID_ARG,
                   "hyper: need 0 <= momentum < 1, eps >= 0, weight_decay >= 0");
  if (h->steps < 1 || h->steps > 64)
    return lm_fail(LAMB_ERR_INVALID_ARG, "hyper: steps is not in [1, 64]");
  if (std::fabs(h->a) > 16 || std::fabs(h->b) > 16 || std::fabs(h->c) > 16)
    return lm_fail(LAMB_ERR_INVALID_ARG,
                   "hyper: coefficients beyond 16 leave fp16's range");
  if (h->scale_kind < LAMB_MUON_SCALE_ONE || h->scale_kind > LAMB_MUON_SCALE_RMS)
    return lm_fail(LAMB_ERR_INVALID_ARG, "hyper: unknown scale_kind %d",
                   h->scale_kind);
  return LAMB_OK;
}

// The small matrices, and what comes in front of the others' products.  A launch that
// is refused is the last of the call.
template <class TG, bool kStep>
cudaError_t muon_front(const lamb_muon* p, const MuonPtrs* ptrs,
                       const MuonConsts& k, int steps, const float* d_lr,
                       cudaStream_t stream) {
  cudaError_t e = cudaSuccess;
  if (p->n_small)
    e = lm_launch(muon_small_kernel<TG, kStep>, (unsigned)p->n_small,
                  kSmallThreads, (size_t)p->small_bytes, stream, false, p->mats,
                  ptrs, p->small, k, steps, d_lr, p->status);
  if (e != cudaSuccess || !p->n_chunks) return e;
  e = lm_launch(muon_norm_kernel<TG, kStep>, (unsigned)p->n_chunks, kMuonThreads,
                0, stream, false, ptrs, p->chunks, k, p->part);
  if (e != cudaSuccess) return e;
  return lm_launch(muon_start_kernel<TG, kStep>, (unsigned)p->n_chunks,
                   kMuonThreads, 0, stream, false, p->mats, ptrs, p->chunks, k,
                   p->part, p->done, p->status);
}

lamb_status_t muon_run(lamb_muon* p, const lamb_muon_hyper_t* h,
                       const float* d_lr, cudaStream_t stream) {
  LmDevice dev(p->device);
  if (dev.err != cudaSuccess) return lm_cuda_fail(dev.err, "cudaSetDevice");
  MuonParams q;
  q.mats = p->mats;
  q.ptrs = d_lr ? p->ptrs : p->dir_ptrs;
  q.d_lr = d_lr;
  q.status = p->status;
  q.k.a = (float)h->a;
  q.k.b = (float)h->b;
  q.k.c = (float)h->c;
  q.k.beta = (float)h->momentum;
  q.k.omb = (float)(1.0 - h->momentum);
  q.k.eps = (float)h->eps;
  q.k.wd = (float)h->weight_decay;
  q.k.size = (float)h->update_scale;
  q.k.nesterov = (h->flags & LAMB_MUON_FLAG_NESTEROV) != 0;
  q.k.scale_kind = h->scale_kind;
  typedef __nv_bfloat16 bf;
  cudaError_t e;
  if (d_lr && p->grad_bf16)
    e = muon_front<bf, true>(p, q.ptrs, q.k, h->steps, d_lr, stream);
  else if (d_lr)
    e = muon_front<float, true>(p, q.ptrs, q.k, h->steps, d_lr, stream);
  else if (p->grad_bf16)
    e = muon_front<bf, false>(p, q.ptrs, q.k, h->steps, nullptr, stream);
  else
    e = muon_front<float, false>(p, q.ptrs, q.k, h->steps, nullptr, stream);
  if (e == cudaSuccess && p->step_tiles) {
    q.tiles = p->tiles;
    q.done = p->done;
    q.steps = h->steps;
    q.n_mats = p->n;
    q.step_tiles = (int)p->step_tiles;
    q.total = (int)(p->step_tiles * h->steps);
    e = muon_launch_steps(q, p->pair, p->units, stream);
  }
  return e == cudaSuccess ? LAMB_OK : lm_cuda_fail(e, "muon launch");
}

lamb_status_t upload_ptrs(lamb_muon* p, MuonPtrs* to,
                          const std::vector<MuonPtrs>& h, cudaStream_t stream) {
  LmDevice dev(p->device);
  cudaError_t e = dev.err;
  if (e == cudaSuccess)
    e = cudaMemcpyAsync(to, h.data(), h.size() * sizeof(MuonPtrs),
                        cudaMemcpyHostToDevice, stream);
  if (e == cudaSuccess) e = cudaStreamSynchronize(stream);
  return e == cudaSuccess ? LAMB_OK : lm_cuda_fail(e, "muon bind");
}

}  // namespace

extern "C" lamb_status_t lamb_muon_create(
    const int64_t* rows, const int64_t* cols, int32_t n_matrices,
    const uint8_t* decay_mask, int32_t grad_dtype, int32_t copy_dtype,
    int32_t device, struct lamb_muon** out) {
  if (!out) return lm_fail(LAMB_ERR_INVALID_ARG, "out is NULL");
  *out = nullptr;
  if (!rows || !cols || n_matrices < 1)
    return lm_fail(LAMB_ERR_INVALID_ARG, "need n_matrices >= 1, rows and cols");
  if (grad_dtype != LAMB_F32 && grad_dtype != LAMB_BF16)
    return lm_fail(LAMB_ERR_UNSUPPORTED_DTYPE, "grad_dtype %d unsupported",
                   grad_dtype);
  if (copy_dtype != LAMB_DTYPE_NONE && copy_dtype != LAMB_BF16)
    return lm_fail(LAMB_ERR_UNSUPPORTED_DTYPE, "copy_dtype %d unsupported",
                   copy_dtype);
  if (device < 0) return lm_fail(LAMB_ERR_INVALID_ARG, "device < 0");
  int64_t total = 0;
  for (int k = 0; k < n_matrices; ++k) {
    if (rows[k] < 0 || cols[k] < 0 || rows[k] > (1 << 20) ||
        cols[k] > (1 << 20))
      return lm_fail(LAMB_ERR_INVALID_ARG,
                     "matrix %d: sides are not in [0, 2^20]", k);
    if (std::min(rows[k], cols[k]) > (1 << 15))
      return lm_fail(LAMB_ERR_INVALID_ARG,
                     "matrix %d: the shorter side is above 2^15", k);
    total += rows[k] * cols[k];
    if (total > (1ll << 36))
      return lm_fail(LAMB_ERR_INVALID_ARG, "more than 2^36 elements");
  }
  LmDevice dev(device);
  if (dev.err != cudaSuccess) return lm_cuda_fail(dev.err, "cudaSetDevice");
  lamb_muon* p = nullptr;
  cudaError_t e = cudaSuccess;
  const char* what = "muon plan";
  try {
    p = new lamb_muon;
    p->device = device;
    p->n = n_matrices;
    p->grad_bf16 = grad_dtype == LAMB_BF16;
    p->copy = copy_dtype == LAMB_BF16;
    for (int k = 0; k < n_matrices; ++k) p->numel.push_back(rows[k] * cols[k]);
    MuonLayout L;
    int sms = 0, ctas = 0, pairs = 0;
    e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device);
    if (e == cudaSuccess) e = muon_steps_setup(sms, &ctas, &pairs);
    if (e != cudaSuccess) {
      lamb_muon_destroy(p);
      return lm_cuda_fail(e, what);
    }
    muon_layout(rows, cols, n_matrices, decay_mask, pairs, &L);
    p->pair = L.pair;
    p->units = L.pair ? pairs : ctas;
    p->n_chunks = (int)L.chunks.size();
    p->step_tiles = (int64_t)L.tiles.size();
    if (p->step_tiles * 64 > INT32_MAX || L.chunks.size() > INT32_MAX) {
      lamb_muon_destroy(p);
      return lm_fail(LAMB_ERR_INVALID_ARG, "the matrices have too many tiles");
    }
    const EncodeTiled encode = lm_encoder();
    LmArena a;
    for (int pass = 0; e == cudaSuccess && pass < 2; ++pass) {
      a.used = 0;
      a.take(&p->status, 1);
      a.take(&p->mats, n_matrices);
      a.take(&p->ptrs, n_matrices);
      a.take(&p->dir_ptrs, n_matrices);
      a.take(&p->chunks, (int64_t)L.chunks.size());
      a.take(&p->tiles, (int64_t)L.tiles.size());
      a.take(&p->done, n_matrices);
      a.take(&p->part, (int64_t)L.chunks.size());
      a.take(&p->small, (int64_t)L.small.size());
      if (pass == 0) {
        e = cudaMalloc(&p->arena, a.used);
        a.base = (char*)p->arena;
      }
    }
    if (e == cudaSuccess && L.work_bytes)
      e = cudaMalloc(&p->work, (size_t)L.work_bytes);
    bool ok = encode != nullptr;
    char* base = (char*)p->work;
    for (int k = 0; e == cudaSuccess && ok && k < n_matrices; ++k) {
      MuonMatrix& x = L.mats[k];
      if (!x.sym) continue;          // empty or small
      bool m = true;
      auto map = [&](CUtensorMap* t, const __half* at, int rows_, int cols_,
                     int pitch, int box_rows, int box_cols) {
        m = m && lm_map(encode, t, false, at, rows_, cols_, pitch, box_rows,
                        box_cols);
      };
      for (int i = 0; i < 2; ++i) {
        x.hi[i] = (__half*)(base + L.at[i][k]);
        map(&x.x_k[i], x.hi[i], x.rows, x.cols, x.pitch, kMuonRows, 64);
        m = m && lm_map_blocks(encode, &x.x_mn[i], false, x.hi[i], x.rows,
                               x.pitch, x.pitch / 64, kMuonRows / 64);
        map(&x.x_c[i], x.hi[i], x.rows, x.cols, x.pitch, kMuonRows, kMuonCols);
      }
      x.lo = (__half*)(base + L.at[2][k]);
      x.D = (__half*)(base + L.at[3][k]);
      x.E = (__half*)(base + L.at[4][k]);
      x.diag = (float*)(base + L.at[5][k]);
      x.beta = (float*)(base + L.at[6][k]);
      map(&x.lo_c, x.lo, x.rows, x.cols, x.pitch, kMuonRows, kMuonCols);
      map(&x.d, x.D, x.m, x.m, x.pitch_m, kMuonRows, 64);
      map(&x.e, x.E, x.m, x.m, x.pitch_m, kMuonRows, 64);
      map(&x.d_c, x.D, x.m, x.m, x.pitch_m, kMuonRows, kMuonCols);
      map(&x.e_c, x.E, x.m, x.m, x.pitch_m, kMuonRows, kMuonCols);
      map(&x.d_t, x.D, x.m, x.m, x.pitch_m, kMuonCols, 64);
      map(&x.e_t, x.E, x.m, x.m, x.pitch_m, kMuonCols, 64);
      ok = m;
    }
    for (MuonTile& t : L.tiles) {
      const MuonMatrix& x = L.mats[t.matrix];
      t.height = t.phase == kApply ? x.rows : x.m;
      t.width = t.phase == kApply ? x.cols : x.m;
      t.kn = (int)lm_ceil_div(t.phase == kGram ? x.n : x.m, 64);
      t.tall = x.tall;
      t.sym = x.sym;
      t.app = x.app;
      t.scale = x.scale;
      t.decay = x.decay;
      t.x = p->mats + t.matrix;
      t.diag = x.diag;
      t.beta = x.beta;
      t.rows = x.rows;
      t.cols = x.cols;
    }
    if (e == cudaSuccess && !ok) {
      e = cudaErrorNotSupported;
      what = "cuTensorMapEncodeTiled";
    }
    p->n_small = (int)L.small.size();
    for (int k : L.small)
      p->small_bytes = std::max(p->small_bytes,
                                small_smem(L.mats[k].m, L.mats[k].n));
    if (e == cudaSuccess) e = allow_small_smem<__nv_bfloat16, true>();
    if (e == cudaSuccess) e = allow_small_smem<__nv_bfloat16, false>();
    if (e == cudaSuccess) e = allow_small_smem<float, true>();
    if (e == cudaSuccess) e = allow_small_smem<float, false>();
    if (e == cudaSuccess && p->n_small)
      e = cudaMemcpy(p->small, L.small.data(), L.small.size() * sizeof(int),
                     cudaMemcpyHostToDevice);
    if (e == cudaSuccess) e = cudaMemset(p->status, 0, sizeof(uint32_t));
    if (e == cudaSuccess)
      e = cudaMemcpy(p->mats, L.mats.data(), L.mats.size() * sizeof(MuonMatrix),
                     cudaMemcpyHostToDevice);
    if (e == cudaSuccess && !L.chunks.empty())
      e = cudaMemcpy(p->chunks, L.chunks.data(),
                     L.chunks.size() * sizeof(MuonChunk),
                     cudaMemcpyHostToDevice);
    if (e == cudaSuccess && !L.tiles.empty())
      e = cudaMemcpy(p->tiles, L.tiles.data(),
                     L.tiles.size() * sizeof(MuonTile), cudaMemcpyHostToDevice);
    if (e == cudaSuccess) e = cudaDeviceSynchronize();
  } catch (const std::bad_alloc&) {
    lamb_muon_destroy(p);
    return lm_fail(LAMB_ERR_OOM, "host allocation failed");
  }
  if (e != cudaSuccess) {
    lamb_muon_destroy(p);
    return lm_cuda_fail(e, what);
  }
  *out = p;
  return LAMB_OK;
}

extern "C" lamb_status_t lamb_muon_bind(struct lamb_muon* p, void* const* w,
                                        const void* const* g, void* const* m,
                                        void* const* w_copy,
                                        cudaStream_t stream) {
  if (!p) return lm_fail(LAMB_ERR_INVALID_ARG, "plan is NULL");
  if (!w || !g || !m)
    return lm_fail(LAMB_ERR_INVALID_ARG, "w, g and m are required");
  if (p->copy != (w_copy != nullptr))
    return lm_fail(LAMB_ERR_INVALID_ARG,
                   "w_copy is required iff the plan has a bf16 copy");
  try {
    std::vector<MuonPtrs> h(p->n);
    for (int k = 0; k < p->n; ++k) {
      h[k] = {(float*)w[k], g[k], (float*)m[k],
              w_copy ? (__nv_bfloat16*)w_copy[k] : nullptr};
      if (!p->numel[k]) continue;
      if (!w[k] || !g[k] || !m[k] || (w_copy && !w_copy[k]))
        return lm_fail(LAMB_ERR_INVALID_ARG, "matrix %d: a pointer is NULL", k);
      if ((uintptr_t)w[k] % 4 || (uintptr_t)m[k] % 4 ||
          (uintptr_t)g[k] % (p->grad_bf16 ? 2 : 4) ||
          (w_copy && (uintptr_t)w_copy[k] % 2))
        return lm_fail(LAMB_ERR_INVALID_ARG,
                       "matrix %d: a pointer is not aligned", k);
    }
    const lamb_status_t st = upload_ptrs(p, p->ptrs, h, stream);
    if (st == LAMB_OK) p->bound = true;
    return st;
  } catch (const std::bad_alloc&) {
    return lm_fail(LAMB_ERR_OOM, "host allocation failed");
  }
}

extern "C" lamb_status_t lamb_muon_bind_direction(struct lamb_muon* p,
                                                  const void* const* u,
                                                  void* const* o,
                                                  cudaStream_t stream) {
  if (!p) return lm_fail(LAMB_ERR_INVALID_ARG, "plan is NULL");
  if (!u || !o) return lm_fail(LAMB_ERR_INVALID_ARG, "u and o are required");
  try {
    std::vector<MuonPtrs> h(p->n);
    for (int k = 0; k < p->n; ++k) {
      h[k] = {nullptr, u[k], nullptr, (__nv_bfloat16*)o[k]};
      if (!p->numel[k]) continue;
      if (!u[k] || !o[k])
        return lm_fail(LAMB_ERR_INVALID_ARG, "matrix %d: a pointer is NULL", k);
      if ((uintptr_t)u[k] % (p->grad_bf16 ? 2 : 4) || (uintptr_t)o[k] % 2)
        return lm_fail(LAMB_ERR_INVALID_ARG,
                       "matrix %d: a pointer is not aligned", k);
    }
    const lamb_status_t st = upload_ptrs(p, p->dir_ptrs, h, stream);
    if (st == LAMB_OK) p->bound_direction = true;
    return st;
  } catch (const std::bad_alloc&) {
    return lm_fail(LAMB_ERR_OOM, "host allocation failed");
  }
}

extern "C" lamb_status_t lamb_muon_step(struct lamb_muon* p,
                                        const lamb_muon_hyper_t* hyper,
                                        const float* d_lr,
                                        cudaStream_t stream) {
  lamb_status_t st = muon_check(p, hyper);
  if (st != LAMB_OK) return st;
  if (!d_lr || (uintptr_t)d_lr % 4)
    return lm_fail(LAMB_ERR_INVALID_ARG, "d_lr is NULL or not aligned");
  if (!p->bound)
    return lm_fail(LAMB_ERR_NOT_BOUND, "lamb_muon_step before lamb_muon_bind");
  return muon_run(p, hyper, d_lr, stream);
}

extern "C" lamb_status_t lamb_muon_direction(struct lamb_muon* p,
                                             const lamb_muon_hyper_t* hyper,
                                             cudaStream_t stream) {
  lamb_status_t st = muon_check(p, hyper);
  if (st != LAMB_OK) return st;
  if (!p->bound_direction)
    return lm_fail(LAMB_ERR_NOT_BOUND,
                   "lamb_muon_direction before lamb_muon_bind_direction");
  return muon_run(p, hyper, nullptr, stream);
}

extern "C" lamb_status_t lamb_muon_query(struct lamb_muon* p,
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

extern "C" lamb_status_t lamb_muon_destroy(struct lamb_muon* p) {
  if (!p) return LAMB_OK;
  LmDevice dev(p->device);
  cudaError_t e = dev.err;
  if (e == cudaSuccess) e = cudaFree(p->arena);
  if (e == cudaSuccess) e = cudaFree(p->work);
  delete p;
  return e == cudaSuccess ? LAMB_OK : lm_cuda_fail(e, "cudaFree(plan)");
}
