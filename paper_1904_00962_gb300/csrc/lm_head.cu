// Vocabulary head: softmax cross entropy of hidden rows against the word table,
// with both gradients, without keeping the logits.
//
//   l = h W^T,  lse_t = log sum_v exp l_tv,  loss_t = lse_t - l_t,y
//   dl = (exp(l - lse) - onehot) * scale / n,  dh = dl W,  dW = dl^T h
//
// n counts the labels that are present.  A row without one has no loss and no
// gradient, so it is left out before the first product: the rows that have a
// label are gathered, and all sizes below come from their number on the device.
// (Whatever an absent row holds, an Inf or NaN too, then reaches nothing.)
// Exponentials are taken in base 2: x' = x log2 e.  Beyond kFarLogit the rounding
// of x' is no longer small beside one (at -1e10 it makes an exponent of 328), so
// there the difference of the logits is taken first.
//
// The loss is one product on the tensor cores (lm_gemm.cuh) whose epilogue
// leaves, of each 256 columns of a row, the maximum and the sum of exponentials
// (fp32); a small kernel joins them in a fixed order.  The label's own column is
// left out of those: with R the sum of exp(l_v - l_y) over the others, the loss is
// log1p(R), which keeps its digits where the label is nearly sure.  So does the
// label's entry of the logits' gradient, -R / (1 + R): p - 1 would have none left.
//
// The gradients take the vocabulary in pieces: a piece's logits are multiplied
// again, the epilogue writes their gradient in bf16 to a workspace (the rounding
// that any bf16 operand of the following products needs; 2^-9 of each element), and
// one more launch multiplies it with W (rows of dh) and, transposed by the operand's
// layout, with h (rows of dW).  dh's sums over pieces and over parts of a long piece
// stay in fp32.  8 T V D operations in all.
//
// Measured: loss of 8192 x 30522 x 768 (6963 labels) 201 us, 1.6 PFLOP/s; loss and
// gradients of 9830 x 30522 x 1024 1521 us, 1.58 PFLOP/s of the 8 T V D: bound by
// the tensor cores under the power limit.  77 x 30522 x 1024 81 us: W is read twice
// from HBM and dW written, 28 us of it; the rest is six launches' latency.
#include <cuda_bf16.h>

#include <algorithm>
#include <new>

#include "lm_gemm.cuh"
#include "lm_vocab.h"

namespace lamb {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kJoinThreads = 256;
constexpr int kJoinRows = 32;          // tokens of a CTA, eight threads each
constexpr int64_t kPieceElems = 64ll << 20;   // dlogits workspace, elements
constexpr int kMinPartBlocks = 4;      // blocks of K in a part of dh, at least
constexpr int64_t kPieceBlocks = 40;   // what a piece more costs, in blocks of K

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Logits (times log2 e) up to this size are scaled before they are subtracted, by
// one fused operation: their exponent is within 2^-14 then.
constexpr float kFarLogit = 1024.f;

// e^(from - to) as sums kept relative to `from` are taken over to `to`.
__device__ __forceinline__ float exp_between(float from, float to) {
  const float b = to * kLog2e;
  return exp2_fast(fabsf(b) < kFarLogit ? __fmul_rn(from, kLog2e) - b
                                        : (from - to) * kLog2e);
}

// ---- rows with a label ------------------------------------------------------
// CTA i takes tokens [kPickRows i, ..): counts the labels before them, gathers
// its own rows that have one, and clears what the others' results are.  With a row
// it forms the label's logit, in fp32: the tensor cores cut off what leaves the
// accumulator's last bit at each of the some fifty additions, 1e-5 of a large
// logit, and where the label is nearly sure that is the loss's relative error.
// For the gradients the last CTA leaves zeros up to a whole block of K (one of
// zeros if there is no row: dW's products need a K).
constexpr int kPickThreads = 512, kPickRows = 32;     // two rows a warp
constexpr int kRowsWhole = 2 * kTileM;       // a tile of a pair of CTAs

// Labels in each kCountRows tokens, so that a CTA of pick_kernel need not look at
// all tokens before its own where those are many.
constexpr int kCountRows = 4096, kCountThreads = 256;
constexpr int64_t kCountFrom = 16384;      // tokens

__global__ void __launch_bounds__(kCountThreads)
count_kernel(const int64_t* labels, int tokens, int64_t vocab, int32_t* counts) {
  const int64_t first = (int64_t)blockIdx.x * kCountRows;
  let_next_launch();
  int any = 0;
  for (int i = threadIdx.x; i < kCountRows; i += kCountThreads) {
    const int64_t y = first + i < tokens ? labels[first + i] : -1;
    any += y >= 0 && y < vocab;
  }
  __shared__ int sh[kCountThreads / 32];
  any = __reduce_add_sync(0xffffffffu, any);
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = any;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 1; i < kCountThreads / 32; ++i) any += sh[i];
    counts[blockIdx.x] = any;
  }
}

__device__ __forceinline__ float dot2(uint32_t a, uint32_t b) {
  return fmaf(__uint_as_float(a << 16), __uint_as_float(b << 16),
              __uint_as_float(a & 0xffff0000u) *
                  __uint_as_float(b & 0xffff0000u));
}

template <bool kVec>
__global__ void __launch_bounds__(kPickThreads)
pick_kernel(const __nv_bfloat16* __restrict__ hidden, int64_t stride,
            const int64_t* __restrict__ labels, const int32_t* counts,
            int tokens, int64_t vocab,
            const __nv_bfloat16* __restrict__ weight, int64_t weight_stride,
            int width, __nv_bfloat16* __restrict__ rows, int64_t pitch,
            float* __restrict__ label_logit, int32_t* __restrict__ row_label, int32_t* __restrict__ row_token,
            int32_t* n_rows, float* token_loss, __nv_bfloat16* grad_hidden,
            int64_t grad_stride, uint32_t* status) {
  __shared__ int sh_count[kPickThreads / 32];
  __shared__ int sh_at[kPickRows], sh_label[kPickRows];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int first = blockIdx.x * kPickRows;
  const bool end = blockIdx.x == gridDim.x - 1;
  int before = 0;
  let_next_launch();
  after_prior_launch();
  const int known = counts ? first / kCountRows : 0;    // whole counts
  for (int i = threadIdx.x; i < known; i += kPickThreads) before += counts[i];
  for (int t = known * kCountRows + threadIdx.x; t < first; t += kPickThreads) {
    const int64_t y = labels[t];
    before += y >= 0 && y < vocab;
  }
  before = __reduce_add_sync(0xffffffffu, before);
  if (lane == 0) sh_count[warp] = before;
  __syncthreads();
  if (warp == 0) {
    int at = 0;
    for (int i = 0; i < kPickThreads / 32; ++i) at += sh_count[i];
    for (int r = 0; r < kPickRows; r += 32) {
      const int t = first + r + lane;
      const int64_t y = t < tokens ? labels[t] : -1;
      const bool real = y >= 0 && y < vocab;
      if (y >= vocab) atomicOr(status, LAMB_STATUS_BAD_INDEX);
      const uint32_t m = __ballot_sync(0xffffffffu, real);
      const int to = at + __popc(m & ((1u << lane) - 1u));
      sh_at[r + lane] = real ? to : -1;
      sh_label[r + lane] = (int)y;
      if (real) {
        row_label[to] = (int32_t)y;
        row_token[to] = t;
      } else if (token_loss && t < tokens) {
        token_loss[t] = 0.f;
      }
      at += __popc(m);
    }
    if (lane == 0) {
      sh_count[0] = at;
      if (end) *n_rows = at;
    }
  }
  __syncthreads();
  const int own = min(kPickRows, tokens - first);
  const int past = sh_count[0] % kTileK;
  const int tail =
      end && grad_hidden && (past || !sh_count[0]) ? kTileK - past : 0;
  for (int r = warp; r < own + tail; r += kPickThreads / 32) {
    const bool zero = r >= own;
    const int t = first + r, to = zero ? sh_count[0] + r - own : sh_at[r];
    if (to < 0 && !grad_hidden) continue;
    const __nv_bfloat16* src = hidden + (int64_t)t * stride;
    const bool real = !zero && to >= 0;
    const __nv_bfloat16* w =
        weight + (real ? (int64_t)sh_label[r] * weight_stride : 0);
    __nv_bfloat16* to_row = to >= 0 ? rows + (int64_t)to * pitch
                                    : grad_hidden + (int64_t)t * grad_stride;
    float dot = 0.f;
    if (kVec) {     // 16 bytes a lane
      uint4* dst = reinterpret_cast<uint4*>(to_row);
#pragma unroll 4
      for (int d = lane; d < width / 8; d += 32) {
        uint4 x = make_uint4(0, 0, 0, 0), y = x;
        if (real) {
          x = reinterpret_cast<const uint4*>(src)[d];
          y = reinterpret_cast<const uint4*>(w)[d];
        }
        dst[d] = x;
        dot += dot2(x.x, y.x) + dot2(x.y, y.y) + dot2(x.z, y.z) +
               dot2(x.w, y.w);
      }
    } else {
      for (int d = lane; d < width; d += 32) {
        const __nv_bfloat16 x = real ? src[d] : __float2bfloat16_rn(0.f);
        to_row[d] = x;
        if (real) dot = fmaf(__bfloat162float(x), __bfloat162float(w[d]), dot);
      }
    }
    if (real) {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1)
        dot += __shfl_xor_sync(0xffffffffu, dot, o);
      if (lane == 0) label_logit[to] = dot;
    }
  }
}

struct RowsState {
  int n_tiles, m_tiles, rows;
};

struct StatsParams {
  CUtensorMap hidden, weight;
  const int32_t* n_rows;
  const int32_t* labels;  // of the rows
  float2* stats;          // [vocab tile][stride]
  uint32_t* status;
  int64_t stride;
  int v_tiles, vocab, k_blocks;
  int weight_early;       // W is the user's and the rows fit one tile of 128
};

struct StatsWork {
  typedef StatsParams Params;
  typedef RowsState State;
  static constexpr bool kBf16 = true;
  template <int kRows>
  static __device__ __forceinline__ State start(const Params& p) {
    State s;
    s.rows = *p.n_rows;
    s.m_tiles = s.rows ? (s.rows + kRows - 1) / kRows : 1;
    s.n_tiles = s.m_tiles * p.v_tiles;
    return s;
  }
  template <int kRows>
  static __device__ __forceinline__ bool tile(const Params& p, const State& s,
                                              int u, int units, int i,
                                              GemmTile* to) {
    const int t = u + i * units;
    if (t >= s.n_tiles) return false;
    GemmTile& g = *to;
    g.a = &p.hidden;
    g.b = &p.weight;
    g.a0 = (t % s.m_tiles) * kRows;
    g.what = t / s.m_tiles;
    g.b0 = g.what * kTileN;
    g.k0 = 0;
    g.kn = p.k_blocks;
    g.b_k = 0;
    g.a_mn = g.b_mn = g.b_blocks = false;
    g.aux = 0;
    return true;
  }
  static __device__ __forceinline__ bool early(const Params& p, int u,
                                               GemmTile* g) {
    return p.weight_early &&
           tile<kTileM>(p, State{p.v_tiles, 1, 0}, u, 1, 0, g);
  }
  static __device__ __forceinline__ void epilogue(const Params& p,
                                                  const State& s,
                                                  const GemmTile& g,
                                                  uint32_t acc, Epilogue& epi) {
    const int r = g.a0 + epi.row;
    const int label = r < s.rows ? p.labels[r] : -1;
    float top = -INFINITY, sum = 0.f;
    for (int c = 0; c < kTileN / 32; ++c) {
      const int v = g.b0 + c * 32;
      if (v >= p.vocab) break;
      float x[32];
      tmem_ld32(acc + c * 32, x);
      if (label >= v && label < v + 32) {
#pragma unroll
        for (int i = 0; i < 32; ++i)
          if (label == v + i) x[i] = -INFINITY;
      }
      if (v + 32 > p.vocab) {
#pragma unroll
        for (int i = 0; i < 32; ++i)
          if (v + i >= p.vocab) x[i] = -INFINITY;
      }
      float m = x[0];
#pragma unroll
      for (int i = 1; i < 32; ++i) m = fmaxf(m, x[i]);
      m = fmaxf(m, top);
      // a row of nothing but -inf keeps the sum 0
      const float to = m == -INFINITY ? 0.f : m;
      float at = to * kLog2e;
      if (fabsf(at) >= kFarLogit) {
#pragma unroll
        for (int i = 0; i < 32; ++i) x[i] -= to;
        at = 0.f;
      }
      float s0 = 0.f, s1 = 0.f;
#pragma unroll
      for (int i = 0; i < 32; i += 2) {
        s0 += exp2_fast(fmaf(x[i], kLog2e, -at));
        s1 += exp2_fast(fmaf(x[i + 1], kLog2e, -at));
      }
      sum = sum * exp_between(top, to) + (s0 + s1);
      top = m;
    }
    if (r < s.rows)
      p.stats[(int64_t)g.what * p.stride + r] = make_float2(top, sum);
  }
};

// Joins a row's statistics in the order of the vocabulary: eight threads a row,
// then those eight; then the mean over the rows (fp64, fixed order) by the CTA
// that finishes last.  Of each row the gradients get x: what is taken off its logits
// (0 but for far ones), y: log2 of the sum of the exponentials of the rest, z: its
// label's entry.
__global__ void __launch_bounds__(kJoinThreads)
join_kernel(const float2* stats, int64_t stride, int v_tiles,
            const float* label_logit, const int32_t* row_token, int tokens,
            const int32_t* n_rows, float4* row_lse, float* token_loss, float* loss,
            const float* scale, float* coef, double* block_sums,
            uint32_t* ticket) {
  __shared__ double sh_loss[kJoinRows];
  __shared__ uint32_t last;
  const int part = threadIdx.x & 7, i = threadIdx.x >> 3;
  const int r = blockIdx.x * kJoinRows + i;
  let_next_launch();
  after_prior_launch();
  // (what lies past the last row is loaded too, not to wait for their number)
  const int rows = *n_rows;
  float top = -INFINITY, sum = 0.f, y = 0.f;
  int token = 0;
  if (r < tokens) {
    y = label_logit[r];
    token = row_token[r];
    const int a = v_tiles * part / 8, b = v_tiles * (part + 1) / 8;
    for (int k0 = a; k0 < b; k0 += 16) {      // sixteen on their way
      float2 s[16];
#pragma unroll
      for (int u = 0; u < 16; ++u)
        s[u] = k0 + u < b ? stats[(int64_t)(k0 + u) * stride + r]
                          : make_float2(-INFINITY, 0.f);
      float m = top;
#pragma unroll
      for (int u = 0; u < 16; ++u) m = fmaxf(m, s[u].x);
      const float at = m == -INFINITY ? 0.f : m;
      sum *= exp_between(top, at);
#pragma unroll
      for (int u = 0; u < 16; ++u) sum += s[u].y * exp_between(s[u].x, at);
      top = m;
    }
  }
#pragma unroll
  for (int o = 1; o < 8; o <<= 1) {
    const float ot = __shfl_xor_sync(0xffffffffu, top, o);
    const float os = __shfl_xor_sync(0xffffffffu, sum, o);
    const float m = fmaxf(top, ot);
    const float at = m == -INFINITY ? 0.f : m;
    sum = sum * exp_between(top, at) + os * exp_between(ot, at);
    top = m;
  }
  if (part == 0) {
    float l = 0.f;
    if (r < rows) {
      const float m = fmaxf(top, y);
      const float at = m == -INFINITY ? 0.f : m;
      const float at2 = at * kLog2e;
      const bool far = fabsf(at2) >= kFarLogit;
      const float off = far ? at : 0.f;
      const float lse = (far ? 0.f : at2) + log2f(sum * exp_between(top, at) +
                                                  exp_between(y, at));
      // (a label at +inf has no value: inf - inf)
      const float others = y < INFINITY ? sum * exp_between(top, y) : NAN;
      row_lse[r] = make_float4(off, lse,
                               others <= 1.f ? -others / (1.f + others)
                                             : 1.f / (1.f + others) - 1.f,
                               0.f);
      l = others < INFINITY ? log1pf(others) : fmaf(lse, kLn2, off - y);
      if (token_loss) token_loss[token] = l;
    }
    sh_loss[i] = l;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    double s = 0.0;
    for (int k = 0; k < kJoinRows; ++k) s += sh_loss[k];
    block_sums[blockIdx.x] = s;
    last = gridDim.x == 1 ||
           atom_add_acq_rel(ticket, 1u) == gridDim.x - 1;
  }
  __syncthreads();
  if (last && threadIdx.x < 32) {
    double s = 0.0;
    for (unsigned k = threadIdx.x; k < gridDim.x; k += 32)
      s += *reinterpret_cast<const volatile double*>(block_sums + k);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (threadIdx.x == 0) {
      *loss = (float)(rows ? s / rows : 0.0);
      *coef = rows ? (scale ? *scale : 1.f) / (float)rows : 0.f;
      *ticket = 0;
    }
  }
}

// ---- the logits' gradient ---------------------------------------------------
struct DlogitsParams {
  CUtensorMap hidden, weight, out;   // out: the piece's columns
  const int32_t* n_rows;
  const int32_t* labels;
  const float4* row_lse;  // of join_kernel
  const float* coef;
  uint32_t* status;
  int v_tiles, vocab, v0, k_blocks;
  int weight_early;       // as in StatsParams
};

struct DlogitsWork {
  typedef DlogitsParams Params;
  typedef RowsState State;
  static constexpr bool kBf16 = true;
  template <int kRows>
  static __device__ __forceinline__ State start(const Params& p) {
    State s;
    s.rows = *p.n_rows;
    s.m_tiles = s.rows ? (s.rows + kRows - 1) / kRows : 1;
    s.n_tiles = s.m_tiles * p.v_tiles;
    return s;
  }
  template <int kRows>
  static __device__ __forceinline__ bool tile(const Params& p, const State& s,
                                              int u, int units, int i,
                                              GemmTile* to) {
    const int t = u + i * units;
    if (t >= s.n_tiles) return false;
    GemmTile& g = *to;
    g.a = &p.hidden;
    g.b = &p.weight;
    g.a0 = (t % s.m_tiles) * kRows;
    g.what = (t / s.m_tiles) * kTileN;     // column inside the piece
    g.b0 = p.v0 + g.what;
    g.k0 = 0;
    g.kn = p.k_blocks;
    g.b_k = 0;
    g.a_mn = g.b_mn = g.b_blocks = false;
    g.aux = 0;
    return true;
  }
  static __device__ __forceinline__ bool early(const Params& p, int u,
                                               GemmTile* g) {
    return p.weight_early &&
           tile<kTileM>(p, State{p.v_tiles, 1, 0}, u, 1, 0, g);
  }
  // Rows past the last and columns past the vocabulary are zeros: the products
  // run over whole tiles.
  static __device__ __forceinline__ void epilogue(const Params& p,
                                                  const State& s,
                                                  const GemmTile& g,
                                                  uint32_t acc, Epilogue& epi) {
    const int r = g.a0 + epi.row;
    const bool real = r < s.rows;
    const int label = real ? p.labels[r] : -1;
    const float4 row = real ? p.row_lse[r] : make_float4(0.f, 0.f, 0.f, 0.f);
    const float coef = *p.coef;
    for (int c = 0; c < kTileN / 64; ++c) {
      const int v = g.b0 + c * 64;
      uint32_t y[32];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float x[32];
        tmem_ld32(acc + c * 64 + h * 32, x);
        if (row.x != 0.f) {
#pragma unroll
          for (int i = 0; i < 32; ++i) x[i] -= row.x;
        }
#pragma unroll
        for (int i = 0; i < 32; ++i)
          x[i] = exp2_fast(fmaf(x[i], kLog2e, -row.y));
        const int first = v + h * 32;
        if (label >= first && label < first + 32) {
#pragma unroll
          for (int i = 0; i < 32; ++i)
            if (label == first + i) x[i] = row.z;
        }
        if (!real || first + 32 > p.vocab) {
#pragma unroll
          for (int i = 0; i < 32; ++i)
            if (!real || first + i >= p.vocab) x[i] = 0.f;
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const __nv_bfloat162 b =
              __floats2bfloat162_rn(x[2 * i] * coef, x[2 * i + 1] * coef);
          y[h * 16 + i] = *reinterpret_cast<const uint32_t*>(&b);
        }
      }
      epi.store_block(&p.out, g.what + c * 64, g.a0 + (epi.row & ~31), y);
    }
  }
};

// ---- the gradients of W and h ------------------------------------------------
struct GradsParams {
  CUtensorMap dl_rows;    // dlogits, K-major (K: the piece's columns)
  CUtensorMap dl_cols;    // dlogits, MN-major (K: tokens)
  CUtensorMap hidden;     // MN-major
  CUtensorMap weight;     // MN-major
  CUtensorMap out;        // grad_weight, where weight_out
  CUtensorMap slabs;      // [split][rows in whole tiles][width], fp32
  void* grad_weight;
  __nv_bfloat16* grad_hidden;
  const int32_t* n_rows;
  const int32_t* row_token;
  uint32_t* status;
  int64_t weight_stride, hidden_stride;
  int slab_rows;          // of a slab; 0: one sum, written out
  int w_tiles;            // tiles of dW
  int d_tiles;            // column tiles of the width
  int width, vocab, v0, piece;
  int k_piece, splits;    // blocks of K of dh, parts that they are cut into
  int weight_blocks;      // weight's map has its blocks as a dimension
  int weight_out;         // dW goes out by tensor copies
  int weight_f32, accumulate, add_slab, weight_vec, hidden_vec;
};

template <bool kF32>
__device__ __forceinline__ void store_row(void* base, int64_t at,
                                          const float (&x)[32], int cols,
                                          bool add, bool vec) {
  float* f = reinterpret_cast<float*>(base) + at;
  __nv_bfloat16* h = reinterpret_cast<__nv_bfloat16*>(base) + at;
  if (vec && cols >= 32) {
    if (kF32) {
#pragma unroll
      for (int i = 0; i < 32; i += 4) {
        float4 v = make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
        float4* to = reinterpret_cast<float4*>(f + i);
        if (add) {
          const float4 o = *to;
          v.x += o.x; v.y += o.y; v.z += o.z; v.w += o.w;
        }
        *to = v;
      }
    } else {
#pragma unroll
      for (int i = 0; i < 32; i += 8) {
        uint4* to = reinterpret_cast<uint4*>(h + i);
        uint4 o = make_uint4(0, 0, 0, 0);
        if (add) o = *to;
        const uint32_t* ow = reinterpret_cast<const uint32_t*>(&o);
        uint32_t y[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const __nv_bfloat162 b = __floats2bfloat162_rn(
              x[i + 2 * j] + __uint_as_float(ow[j] << 16),
              x[i + 2 * j + 1] + __uint_as_float(ow[j] & 0xffff0000u));
          y[j] = *reinterpret_cast<const uint32_t*>(&b);
        }
        *to = make_uint4(y[0], y[1], y[2], y[3]);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      if (i < cols) {
        if (kF32)
          f[i] = add ? f[i] + x[i] : x[i];
        else
          h[i] = __float2bfloat16_rn(add ? __bfloat162float(h[i]) + x[i]
                                         : x[i]);
      }
    }
  }
}

struct GradsState {
  int rows, k_rows;
  int h_tiles;            // tiles of dh
};

// dh's tiles run over the piece's columns, dW's over the rows.  Unit u of U takes
// dh's tiles u, u + U, ..; the units that then have one less take as many of dW's
// as come to the same blocks of K, and the rest of dW goes round, those units first.
// (One list in turn left the longest unit a quarter above the mean at 2458 x 768.)
struct GradsWork {
  typedef GradsParams Params;
  typedef GradsState State;
  static constexpr bool kBf16 = true;
  template <int kRows>
  static __device__ __forceinline__ State start(const Params& p) {
    State s;
    s.rows = *p.n_rows;
    s.k_rows = s.rows ? (s.rows + kTileK - 1) / kTileK : 1;   // of zeros
    s.h_tiles = (s.rows + kRows - 1) / kRows * p.d_tiles * p.splits;
    return s;
  }
  template <int kRows>
  static __device__ __forceinline__ bool tile(const Params& p, const State& s,
                                              int u, int units, int i,
                                              GemmTile* to) {
    GemmTile& g = *to;
    const int turns = s.h_tiles / units, over = s.h_tiles - turns * units;
    const int own = turns + (u < over);
    if (i < own) {
      int t = u + i * units;
      g.what = 1;
      g.aux = t % p.splits;
      t /= p.splits;
      g.a = &p.dl_rows;
      g.b = &p.weight;
      g.a0 = t / p.d_tiles * kRows;
      g.b0 = t % p.d_tiles * kTileN;
      g.k0 = (int)((int64_t)p.k_piece * g.aux / p.splits);
      g.kn = (int)((int64_t)p.k_piece * (g.aux + 1) / p.splits) - g.k0;
      g.b_k = p.v0;      // W's rows are the whole vocabulary's
      g.a_mn = false;
      g.b_mn = true;
      g.b_blocks = p.weight_blocks;
      return true;
    }
    i -= own;
    // dW's tiles that even out the units without the last of dh's
    const int less = units - over;
    int even = over ? p.k_piece / p.splits / s.k_rows : 0;
    even = min(even, p.w_tiles / less);
    int t;
    if (u >= over && i < even) {
      t = u - over + i * less;
    } else {
      if (u >= over) i -= even;
      t = even * less + (u >= over ? u - over : u + less) + i * units;
      if (t >= p.w_tiles) return false;
    }
    g.what = 0;
    g.aux = 0;
    g.a = &p.dl_cols;
    g.b = &p.hidden;
    g.a0 = t / p.d_tiles * kRows;
    g.b0 = t % p.d_tiles * kTileN;
    g.k0 = 0;
    g.kn = s.k_rows;
    g.b_k = 0;
    g.a_mn = g.b_mn = g.b_blocks = true;
    return true;
  }
  static __device__ __forceinline__ bool early(const Params&, int, GemmTile*) {
    return false;         // dlogits and the rows come from the launches in front
  }
  static __device__ __forceinline__ void epilogue(const Params& p,
                                                  const State& s,
                                                  const GemmTile& g,
                                                  uint32_t acc, Epilogue& epi) {
    const int r = g.a0 + epi.row;
    const bool in = g.what ? r < s.rows : r < p.piece && p.v0 + r < p.vocab;
    if (g.what == 0 && p.weight_out) {
      // (past the piece's rows the accumulator holds zeros, and past the
      // vocabulary's the copy writes nothing)
      for (int c = 0; c < kTileN / 64; ++c) {
        const int d = g.b0 + c * 64;
        if (d >= p.width) break;
        uint32_t y[32];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float x[32];
          tmem_ld32(acc + c * 64 + h * 32, x);
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const __nv_bfloat162 b =
                __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
            y[h * 16 + i] = *reinterpret_cast<const uint32_t*>(&b);
          }
        }
        const int first = g.a0 + (epi.row & ~31);
        if (first < p.piece && p.v0 + first < p.vocab)
          epi.store_block(&p.out, d, p.v0 + first, y);
      }
      return;
    }
    if (g.what == 1 && p.slab_rows) {
      const int y = g.aux * p.slab_rows + g.a0 + (epi.row & ~31);
      for (int c = 0; c < kTileN / 32; ++c) {
        const int d = g.b0 + c * 32;
        if (d >= p.width) break;
        float x[32];
        tmem_ld32(acc + c * 32, x);
        uint32_t w[32];
#pragma unroll
        for (int i = 0; i < 32; ++i) w[i] = __float_as_uint(x[i]);
        epi.store_block(&p.slabs, d, y, w, p.add_slab);
      }
      return;
    }
    for (int c = 0; c < kTileN / 32; ++c) {
      const int d = g.b0 + c * 32;
      if (d >= p.width) break;
      float x[32];
      tmem_ld32(acc + c * 32, x);
      if (!in) continue;
      const int cols = p.width - d;
      if (g.what == 0) {
        const int64_t at = (int64_t)(p.v0 + r) * p.weight_stride + d;
        if (p.weight_f32)
          store_row<true>(p.grad_weight, at, x, cols, p.accumulate,
                          p.weight_vec);
        else
          store_row<false>(p.grad_weight, at, x, cols, p.accumulate,
                           p.weight_vec);
      } else {
        store_row<false>(p.grad_hidden,
                         (int64_t)p.row_token[r] * p.hidden_stride + d, x,
                         cols, false, p.hidden_vec);
      }
    }
  }
};

// dh from its partial sums, kCols columns a thread.
template <int kCols>
__global__ void __launch_bounds__(256)
slabs_kernel(const float* slabs, int count, int64_t slab, int pitch, int width,
             const int32_t* n_rows, const int32_t* row_token,
             __nv_bfloat16* out, int64_t stride) {
  after_prior_launch();
  const int per = width / kCols;
  const int64_t n = (int64_t)*n_rows * per;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n;
       i += (int64_t)gridDim.x * 256) {
    const int r = (int)(i / per), d = (int)(i - (int64_t)r * per) * kCols;
    const float* from = slabs + (int64_t)r * pitch + d;
    __nv_bfloat16* to = out + (int64_t)row_token[r] * stride + d;
    if (kCols == 4) {
      float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 16
      for (int k = 0; k < count; ++k) {
        const float4 v = *reinterpret_cast<const float4*>(from + k * slab);
        s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
      }
      const __nv_bfloat162 a = __floats2bfloat162_rn(s.x, s.y);
      const __nv_bfloat162 b = __floats2bfloat162_rn(s.z, s.w);
      *reinterpret_cast<uint2*>(to) =
          make_uint2(*reinterpret_cast<const uint32_t*>(&a),
                     *reinterpret_cast<const uint32_t*>(&b));
    } else {
      float s = 0.f;
#pragma unroll 8
      for (int k = 0; k < count; ++k) s += from[k * slab];
      *to = __float2bfloat16_rn(s);
    }
  }
}

// Rows of a bf16 matrix that no tensor map can read, on 16-byte boundaries: a pass over
// all of W in each call with such a W, element by element.
__global__ void __launch_bounds__(256)
rows_copy_kernel(const __nv_bfloat16* in, int64_t in_stride, int64_t rows,
                 int width, __nv_bfloat16* out, int64_t out_stride) {
  const int64_t n = rows * width;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n;
       i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / width;
    out[r * out_stride + (i - r * width)] = in[r * in_stride + (i - r * width)];
  }
}

__global__ void __launch_bounds__(256)
clear_rows_kernel(void* base, int f32, int64_t rows, int width,
                  int64_t stride) {
  const int64_t n = rows * width;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n;
       i += (int64_t)gridDim.x * 256) {
    const int64_t at = i / width * stride + i % width;
    if (f32) reinterpret_cast<float*>(base)[at] = 0.f;
    else reinterpret_cast<__nv_bfloat16*>(base)[at] = __float2bfloat16_rn(0.f);
  }
}

// Pairs of CTAs from this many rows on.
constexpr int64_t kPairRows = kTileM + 1;

template <class Work>
cudaError_t launch_gemm(const typename Work::Params& p, bool pair,
                        int64_t most_tiles, int sms, cudaStream_t stream) {
  if (pair)
    return lm_launch(gemm_kernel<Work, 2>,
                     2u * (unsigned)std::min<int64_t>(most_tiles, sms / 2),
                     kGemmThreads, kGemmSmem<2>, stream, true, p);
  return lm_launch(gemm_kernel<Work, 1>,
                   (unsigned)std::min<int64_t>(most_tiles, sms), kGemmThreads,
                   kGemmSmem<1>, stream, true, p);
}

template <class Work>
cudaError_t allow_smem() {
  const cudaError_t e = cudaFuncSetAttribute(
      gemm_kernel<Work, 1>, cudaFuncAttributeMaxDynamicSharedMemorySize,
      (int)kGemmSmem<1>);
  if (e != cudaSuccess) return e;
  return cudaFuncSetAttribute(gemm_kernel<Work, 2>,
                              cudaFuncAttributeMaxDynamicSharedMemorySize,
                              (int)kGemmSmem<2>);
}

int grid_for(int64_t n, int sms) {
  return (int)std::max<int64_t>(1, std::min<int64_t>(lm_ceil_div(n, 256),
                                                     (int64_t)sms * 8));
}

// The rows that have a label, and W as a tensor map can read it.
struct HeadInputs {
  const __nv_bfloat16* weight;
  int64_t weight_stride;
  int64_t pitch;        // of the gathered rows
};

cudaError_t head_inputs(const lamb_vocab* v, const void* hidden, int64_t hs,
                        const void* weight, int64_t ws, const int64_t* labels,
                        int64_t n, float* token_loss, void* grad_hidden,
                        int64_t gs, cudaStream_t stream, HeadInputs* in) {
  in->pitch = lm_round_up(v->width, 64);
  in->weight = (const __nv_bfloat16*)weight;
  in->weight_stride = ws;
  const bool vec = lm_mappable(hidden, hs) && lm_mappable(weight, ws) &&
                   v->width % 8 == 0 &&
                   (!grad_hidden || lm_mappable(grad_hidden, gs));
  const unsigned grid = (unsigned)lm_ceil_div(n, kPickRows);
  const bool many = n > kCountFrom;
  cudaError_t e = cudaSuccess;
  if (many)
    e = lm_launch(count_kernel, (unsigned)lm_ceil_div(n, kCountRows),
                  kCountThreads, 0, stream, false, labels, (int)n, v->vocab,
                  v->counts);
  if (e == cudaSuccess)
    e = lm_launch(vec ? pick_kernel<true> : pick_kernel<false>, grid,
                  kPickThreads, 0, stream, many, (const __nv_bfloat16*)hidden,
                  hs, labels, many ? v->counts : nullptr, (int)n, v->vocab,
                  (const __nv_bfloat16*)weight, ws, v->width, v->rows, in->pitch,
                  v->label_logit, v->row_label, v->row_token, v->n_rows,
                  token_loss, (__nv_bfloat16*)grad_hidden, gs, v->status);
  if (e != cudaSuccess) return e;
  if (!lm_mappable(weight, ws)) {
    e = lm_launch(rows_copy_kernel,
                  (unsigned)grid_for(v->vocab * v->width, v->sms), 256, 0, stream,
                  false, in->weight, ws, v->vocab, v->width, v->weight_copy,
                  in->pitch);
    in->weight = v->weight_copy;
    in->weight_stride = in->pitch;
  }
  return e;
}

lamb_status_t head_loss(lamb_vocab* v, const HeadInputs& in, int64_t n,
                        const float* scale, float* token_loss, float* loss,
                        cudaStream_t stream) {
  StatsParams p;
  const bool pair = n >= kPairRows;
  const int rows_b = pair ? kRowsB<2> : kRowsB<1>;
  if (!lm_map(v->encode, &p.hidden, true, v->rows, lm_round_up(n, kRowsWhole),
              v->width, in.pitch, kTileM) ||
      !lm_map(v->encode, &p.weight, true, in.weight, v->vocab, v->width,
              in.weight_stride, rows_b))
    return lm_fail(LAMB_ERR_CUDA, "cuTensorMapEncodeTiled failed");
  p.n_rows = v->n_rows;
  p.labels = v->row_label;
  p.stats = v->stats;
  p.status = v->status;
  p.stride = v->max_tokens;
  p.v_tiles = (int)lm_ceil_div(v->vocab, kTileN);
  p.vocab = (int)v->vocab;
  p.k_blocks = (int)lm_ceil_div(v->width, kTileK);
  p.weight_early = !pair && in.weight != v->weight_copy;
  cudaError_t e = launch_gemm<StatsWork>(
      p, pair, lm_ceil_div(n, pair ? kRowsWhole : kTileM) * p.v_tiles, v->sms,
      stream);
  if (e != cudaSuccess) return lm_cuda_fail(e, "head loss launch");
  e = lm_launch(join_kernel, (unsigned)lm_ceil_div(n, kJoinRows), kJoinThreads,
                0, stream, true, v->stats, v->max_tokens, p.v_tiles,
                v->label_logit, v->row_token, (int)n, v->n_rows,
                v->row_lse, token_loss, loss, scale, v->coef, v->block_sums,
                v->ticket);
  return e == cudaSuccess ? LAMB_OK : lm_cuda_fail(e, "head join launch");
}

// Parts of dh's K: dh of few tokens is few tiles over a long K, cut so that every
// CTA or pair has one.
int64_t head_parts(int64_t units, int64_t h_tiles, int64_t k_blocks) {
  return std::max<int64_t>(1, std::min(units / h_tiles,
                                       k_blocks / kMinPartBlocks));
}

// Columns of a piece of the vocabulary, in whole tiles: of the counts of pieces
// that the workspace allows, the one whose products' tiles (rows of dW over all
// tokens, rows of dh over the piece) fall best on `units` CTAs or pairs.  9830 x
// 30522 x 1024, us: the fewest pieces 1564, so chosen 1527; 2458 x 30522 x 768, two
// pieces either way, 329 to 335.
int64_t piece_width(const lamb_vocab* v, int64_t n, int rows, int units) {
  const int64_t whole = lm_round_up(n, kRowsWhole);
  const int64_t most = v->dlogits_elems / whole / kTileN * kTileN;
  const int64_t least = lm_ceil_div(v->vocab, most);
  const int64_t d_tiles = lm_ceil_div(v->width, kTileN);
  const int64_t h_tiles = lm_ceil_div(n, rows) * d_tiles;
  const int64_t w_blocks = lm_ceil_div(n, kTileK);
  int64_t best = most, best_cost = INT64_MAX;
  for (int64_t np = least; np < least + 6; ++np) {
    const int64_t piece =
        lm_round_up(lm_ceil_div(v->vocab, np), kTileN);
    const int64_t w_tiles = lm_ceil_div(piece, rows) * d_tiles;
    // (as GradsWork::tile hands them out)
    const int64_t parts = head_parts(units, h_tiles, piece / kTileK);
    const int64_t h = piece / kTileK / parts, hs = h_tiles * parts;
    const int64_t turns = hs / units, over = hs % units, less = units - over;
    const int64_t even =
        over ? std::min(h / w_blocks, w_tiles / less) : 0;
    const int64_t rest = w_tiles - even * less;
    const int64_t longest =
        std::max((turns + (over > 0)) * h +
                     lm_ceil_div(std::max<int64_t>(rest - less, 0), units) *
                         w_blocks * (over > 0),
                 turns * h + (even + lm_ceil_div(rest, units)) * w_blocks);
    // two launches and their tails are worth some blocks more
    const int64_t cost =
        lm_ceil_div(v->vocab, piece) * (longest + kPieceBlocks);
    if (cost < best_cost) {
      best_cost = cost;
      best = piece;
    }
  }
  return best;
}

lamb_status_t check_head(const lamb_vocab* v, const void* hidden, int64_t hs,
                         const void* weight, int64_t ws, const int64_t* labels,
                         int64_t n, const float* token_loss,
                         const float* loss) {
  if (!v) return lm_fail(LAMB_ERR_INVALID_ARG, "plan is NULL");
  if (n < 0 || n > v->max_tokens)
    return lm_fail(LAMB_ERR_INVALID_ARG,
                   "n_tokens %lld is not in [0, max_tokens = %lld]",
                   (long long)n, (long long)v->max_tokens);
  if (!weight || !loss || (n && (!hidden || !labels)))
    return lm_fail(LAMB_ERR_INVALID_ARG,
                   "hidden, weight, labels and loss are required");
  if (hs < v->width || ws < v->width)
    return lm_fail(LAMB_ERR_INVALID_ARG, "a row stride is below the width %d",
                   v->width);
  if ((uintptr_t)hidden % 2 || (uintptr_t)weight % 2 || (uintptr_t)loss % 4 ||
      (uintptr_t)token_loss % 4 || (uintptr_t)labels % 8)
    return lm_fail(LAMB_ERR_INVALID_ARG, "a pointer is not aligned");
  return LAMB_OK;
}

}  // namespace

int lm_head_setup() {
  cudaError_t e = allow_smem<StatsWork>();
  if (e == cudaSuccess) e = allow_smem<DlogitsWork>();
  if (e == cudaSuccess) e = allow_smem<GradsWork>();
  return (int)e;
}

void lm_head_carve(lamb_vocab* v, LmArena* a) {
  const int64_t n = v->max_tokens, pitch = lm_round_up(v->width, 64);
  const int64_t whole = lm_round_up(n, kRowsWhole);
  a->take(&v->rows, whole * pitch);
  a->take(&v->row_label, n);
  a->take(&v->row_token, n);
  a->take(&v->n_rows, 1);
  a->take(&v->counts, lm_ceil_div(n, kCountRows));
  a->take(&v->stats, lm_ceil_div(v->vocab, kTileN) * n);
  a->take(&v->label_logit, n);
  a->take(&v->row_lse, n);
  a->take(&v->block_sums, lm_ceil_div(n, kJoinRows));
  a->take(&v->ticket, 1);
  a->take(&v->coef, 1);
  // a whole vocabulary where that is small, else kPieceElems
  v->dlogits_elems = std::min(whole * lm_round_up(v->vocab, kTileN),
                              std::max(kPieceElems, whole * (int64_t)kTileN));
  a->take(&v->dlogits, v->dlogits_elems);
  // parts of dh never have more tiles than there are SMs, unless it is one part
  a->take(&v->slabs, std::max(whole * lm_round_up(v->width, 4),
                              (int64_t)v->sms * kTileM * kTileN));
  a->take(&v->weight_copy, v->vocab * pitch);
}

}  // namespace lamb

using namespace lamb;

extern "C" lamb_status_t lamb_vocab_loss(
    struct lamb_vocab* v, const void* hidden, int64_t hidden_stride,
    const void* weight, int64_t weight_stride, const int64_t* labels,
    int64_t n_tokens, float* token_loss, float* loss, cudaStream_t stream) {
  lamb_status_t st = check_head(v, hidden, hidden_stride, weight, weight_stride,
                                labels, n_tokens, token_loss, loss);
  if (st != LAMB_OK) return st;
  LmDevice dev(v->device);
  if (dev.err != cudaSuccess) return lm_cuda_fail(dev.err, "cudaSetDevice");
  if (!n_tokens) {
    const cudaError_t e = cudaMemsetAsync(loss, 0, sizeof(float), stream);
    return e == cudaSuccess ? LAMB_OK : lm_cuda_fail(e, "clearing the loss");
  }
  HeadInputs in;
  const cudaError_t e = head_inputs(v, hidden, hidden_stride, weight,
                                    weight_stride, labels, n_tokens, token_loss,
                                    nullptr, 0, stream, &in);
  if (e != cudaSuccess) return lm_cuda_fail(e, "head copy launch");
  return head_loss(v, in, n_tokens, nullptr, token_loss, loss, stream);
}

extern "C" lamb_status_t lamb_vocab_loss_grad(
    struct lamb_vocab* v, const void* hidden, int64_t hidden_stride,
    const void* weight, int64_t weight_stride, const int64_t* labels,
    int64_t n_tokens, const float* d_scale, float* token_loss, float* loss,
    void* grad_hidden, int64_t grad_hidden_stride, void* grad_weight,
    int32_t grad_weight_dtype, int64_t grad_weight_stride, int32_t accumulate,
    cudaStream_t stream) {
  lamb_status_t st = check_head(v, hidden, hidden_stride, weight, weight_stride,
                                labels, n_tokens, token_loss, loss);
  if (st != LAMB_OK) return st;
  const int64_t n = n_tokens;
  if (grad_weight_dtype != LAMB_F32 && grad_weight_dtype != LAMB_BF16)
    return lm_fail(LAMB_ERR_UNSUPPORTED_DTYPE, "grad_weight: dtype %d unsupported",
                   grad_weight_dtype);
  if (!grad_weight || (n && !grad_hidden))
    return lm_fail(LAMB_ERR_INVALID_ARG,
                   "grad_hidden and grad_weight are required");
  if (grad_hidden_stride < v->width || grad_weight_stride < v->width)
    return lm_fail(LAMB_ERR_INVALID_ARG,
                   "a gradient's row stride is below the width %d", v->width);
  const bool f32 = grad_weight_dtype == LAMB_F32;
  if ((uintptr_t)grad_hidden % 2 || (uintptr_t)d_scale % 4 ||
      (uintptr_t)grad_weight % (f32 ? 4 : 2))
    return lm_fail(LAMB_ERR_INVALID_ARG, "a gradient's pointer is not aligned");
  LmDevice dev(v->device);
  if (dev.err != cudaSuccess) return lm_cuda_fail(dev.err, "cudaSetDevice");
  cudaError_t e;
  if (!n) {
    e = cudaMemsetAsync(loss, 0, sizeof(float), stream);
    if (e == cudaSuccess && !accumulate) {
      e = lm_launch(clear_rows_kernel,
                    (unsigned)grid_for(v->vocab * v->width, v->sms), 256, 0,
                    stream, false, grad_weight, (int)f32, v->vocab, v->width,
                    grad_weight_stride);
    }
    return e == cudaSuccess ? LAMB_OK : lm_cuda_fail(e, "clearing the gradient");
  }
  HeadInputs in;
  e = head_inputs(v, hidden, hidden_stride, weight, weight_stride, labels, n,
                  token_loss, grad_hidden, grad_hidden_stride, stream, &in);
  if (e != cudaSuccess) return lm_cuda_fail(e, "head copy launch");
  st = head_loss(v, in, n, d_scale, token_loss, loss, stream);
  if (st != LAMB_OK) return st;

  const bool pair = n >= kPairRows;
  const int rows = pair ? kRowsWhole : kTileM;       // of a tile
  const int rows_b = pair ? kRowsB<2> : kRowsB<1>;
  const int64_t whole = lm_round_up(n, kRowsWhole);
  const int m_tiles = (int)lm_ceil_div(n, rows);
  const int d_tiles = (int)lm_ceil_div(v->width, kTileN);
  const int units = pair ? v->sms / 2 : v->sms;
  const int64_t piece = piece_width(v, n, rows, units);
  const int64_t pieces = lm_ceil_div(v->vocab, piece);

  DlogitsParams d;
  GradsParams g;
  // (the copy of W has rows of whole blocks; the user's only if the width is)
  g.weight_blocks = v->width % 64 == 0 || in.weight == v->weight_copy;
  // (a tensor store leaves out whole units of 16 bytes only: where a row ends inside
  // one, the rest of it is the caller's)
  g.weight_out = !f32 && !accumulate && v->width % 8 == 0 &&
                 lm_mappable(grad_weight, grad_weight_stride);
  const bool ok =
      lm_map(v->encode, &d.hidden, true, v->rows, whole, v->width, in.pitch,
             kTileM) &&
      lm_map(v->encode, &d.weight, true, in.weight, v->vocab, v->width,
             in.weight_stride, rows_b) &&
      lm_map(v->encode, &d.out, true, v->dlogits, whole, piece, piece, 32) &&
      lm_map_blocks(v->encode, &g.hidden, true, v->rows, whole, in.pitch,
                    in.pitch / 64, rows_b / 64) &&
      (g.weight_blocks
           ? lm_map_blocks(v->encode, &g.weight, true, in.weight, v->vocab,
                           in.weight_stride, lm_ceil_div(v->width, 64),
                           rows_b / 64)
           : lm_map(v->encode, &g.weight, true, in.weight, v->vocab, v->width,
                    in.weight_stride, kTileK)) &&
      lm_map(v->encode, &g.dl_rows, true, v->dlogits, whole, piece, piece,
             kTileM) &&
      lm_map_blocks(v->encode, &g.dl_cols, true, v->dlogits, whole, piece,
                    piece / 64, kTileM / 64) &&
      (!g.weight_out || lm_map(v->encode, &g.out, true, grad_weight, v->vocab,
                               v->width, grad_weight_stride, 32));
  if (!ok) return lm_fail(LAMB_ERR_CUDA, "cuTensorMapEncodeTiled failed");
  d.n_rows = v->n_rows;
  d.labels = v->row_label;
  d.row_lse = v->row_lse;
  d.coef = v->coef;
  d.status = v->status;
  d.vocab = (int)v->vocab;
  d.k_blocks = (int)lm_ceil_div(v->width, kTileK);
  d.weight_early = !pair && in.weight != v->weight_copy;

  g.d_tiles = d_tiles;
  const int h_tiles = m_tiles * d_tiles;
  g.grad_weight = grad_weight;
  g.weight_stride = grad_weight_stride;
  g.grad_hidden = (__nv_bfloat16*)grad_hidden;
  g.hidden_stride = grad_hidden_stride;
  g.status = v->status;
  g.n_rows = v->n_rows;
  g.row_token = v->row_token;
  g.width = v->width;
  g.vocab = (int)v->vocab;
  g.piece = (int)piece;
  g.weight_f32 = f32;
  g.accumulate = accumulate != 0;
  g.weight_vec = (uintptr_t)grad_weight % 16 == 0 &&
                 grad_weight_stride % (f32 ? 4 : 8) == 0;
  g.hidden_vec =
      (uintptr_t)grad_hidden % 16 == 0 && grad_hidden_stride % 8 == 0;
  const int k_first = (int)lm_ceil_div(std::min(piece, v->vocab), kTileK);
  g.splits = (int)head_parts(units, h_tiles, k_first);
  g.slab_rows = pieces > 1 || g.splits > 1 ? m_tiles * rows : 0;
  const int pitch = (int)lm_round_up(v->width, 4);
  if (g.slab_rows &&
      !lm_map_f32(v->encode, &g.slabs, v->slabs,
                  (int64_t)g.splits * g.slab_rows, v->width, pitch, 32))
    return lm_fail(LAMB_ERR_CUDA, "cuTensorMapEncodeTiled failed");
  for (int64_t i = 0; i < pieces; ++i) {
    const int64_t v0 = i * piece, cols = std::min(piece, v->vocab - v0);
    d.v0 = g.v0 = (int)v0;
    d.v_tiles = (int)lm_ceil_div(cols, kTileN);
    e = launch_gemm<DlogitsWork>(d, pair, (int64_t)m_tiles * d.v_tiles, v->sms,
                                 stream);
    if (e != cudaSuccess) return lm_cuda_fail(e, "logit gradient launch");
    g.w_tiles = (int)lm_ceil_div(cols, rows) * d_tiles;
    g.k_piece = (int)lm_ceil_div(cols, kTileK);
    // the last piece may be short: fewer parts, the others' sums stay
    const int parts = std::min(g.splits, g.k_piece);
    GradsParams gi = g;
    gi.splits = parts;
    gi.add_slab = i > 0;
    e = launch_gemm<GradsWork>(gi, pair, g.w_tiles + (int64_t)h_tiles * parts,
                               v->sms, stream);
    if (e != cudaSuccess) return lm_cuda_fail(e, "head gradient launch");
  }
  if (g.slab_rows) {
    const bool four = v->width % 4 == 0 &&
                      (uintptr_t)grad_hidden % 8 == 0 &&
                      grad_hidden_stride % 4 == 0;
    const int per = v->width / (four ? 4 : 1);
    e = lm_launch(four ? slabs_kernel<4> : slabs_kernel<1>,
                  (unsigned)grid_for(n * per, v->sms), 256, 0, stream, true,
                  v->slabs, g.splits, (int64_t)g.slab_rows * pitch, pitch,
                  v->width, v->n_rows, v->row_token,
                  (__nv_bfloat16*)grad_hidden, grad_hidden_stride);
    if (e != cudaSuccess) return lm_cuda_fail(e, "hidden gradient launch");
  }
  return LAMB_OK;
}

// ---------------------------------------------------------------------------
// The plan
// ---------------------------------------------------------------------------
extern "C" lamb_status_t lamb_vocab_create(int64_t vocab, int32_t width,
                                           int64_t max_tokens, int32_t device,
                                           struct lamb_vocab** out) {
  if (!out) return lm_fail(LAMB_ERR_INVALID_ARG, "out is NULL");
  *out = nullptr;
  if (vocab < 1 || vocab > (1ll << 30))
    return lm_fail(LAMB_ERR_INVALID_ARG, "vocab is not in [1, 2^30]");
  if (width < 1 || width > (1 << 20))
    return lm_fail(LAMB_ERR_INVALID_ARG, "width is not in [1, 2^20]");
  if (max_tokens < 1 || max_tokens > (1ll << 24))
    return lm_fail(LAMB_ERR_INVALID_ARG, "max_tokens is not in [1, 2^24]");
  if (lm_ceil_div(max_tokens, kTileM) * lm_ceil_div(vocab, kTileN) > INT32_MAX)
    return lm_fail(LAMB_ERR_INVALID_ARG,
                   "max_tokens times vocab is above 2^46 or so");
  if (device < 0) return lm_fail(LAMB_ERR_INVALID_ARG, "device < 0");
  LmDevice dev(device);
  if (dev.err != cudaSuccess) return lm_cuda_fail(dev.err, "cudaSetDevice");
  lamb_vocab* v = new (std::nothrow) lamb_vocab;
  if (!v) return lm_fail(LAMB_ERR_OOM, "host allocation failed");
  v->device = device;
  v->vocab = vocab;
  v->width = width;
  v->max_tokens = max_tokens;
  v->encode = lm_encoder();
  cudaError_t e =
      cudaDeviceGetAttribute(&v->sms, cudaDevAttrMultiProcessorCount, device);
  if (e == cudaSuccess && !v->encode) {
    delete v;
    return lm_fail(LAMB_ERR_CUDA, "the driver has no cuTensorMapEncodeTiled");
  }
  if (e == cudaSuccess) e = (cudaError_t)lm_head_setup();
  LmArena a;
  for (int pass = 0; e == cudaSuccess && pass < 2; ++pass) {
    a.used = 0;
    a.take(&v->status, 1);
    lm_head_carve(v, &a);
    lm_embed_carve(v, &a);
    if (pass == 0) {
      e = cudaMalloc(&v->arena, a.used);
      a.base = (char*)v->arena;
    }
  }
  if (e == cudaSuccess) e = cudaMemset(v->status, 0, sizeof(uint32_t));
  if (e == cudaSuccess) e = cudaMemset(v->ticket, 0, sizeof(uint32_t));
  if (e == cudaSuccess) e = cudaDeviceSynchronize();
  if (e != cudaSuccess) {
    if (v->arena) cudaFree(v->arena);
    delete v;
    return lm_cuda_fail(e, "vocabulary plan");
  }
  *out = v;
  return LAMB_OK;
}

extern "C" lamb_status_t lamb_vocab_query(struct lamb_vocab* v,
                                          uint32_t* status_bits, int32_t clear,
                                          cudaStream_t stream) {
  if (!v) return lm_fail(LAMB_ERR_INVALID_ARG, "plan is NULL");
  if (!status_bits)
    return lm_fail(LAMB_ERR_INVALID_ARG, "status_bits is NULL");
  LmDevice dev(v->device);
  cudaError_t e = dev.err;
  if (e == cudaSuccess)
    e = cudaMemcpyAsync(status_bits, v->status, sizeof(uint32_t),
                        cudaMemcpyDeviceToHost, stream);
  if (e == cudaSuccess && clear)
    e = cudaMemsetAsync(v->status, 0, sizeof(uint32_t), stream);
  if (e == cudaSuccess) e = cudaStreamSynchronize(stream);
  return e == cudaSuccess ? LAMB_OK : lm_cuda_fail(e, "status query");
}

extern "C" lamb_status_t lamb_vocab_destroy(struct lamb_vocab* v) {
  if (!v) return LAMB_OK;
  LmDevice dev(v->device);
  cudaError_t e = dev.err;
  if (e == cudaSuccess) e = cudaFree(v->arena);
  delete v;
  return e == cudaSuccess ? LAMB_OK : lm_cuda_fail(e, "cudaFree(plan)");
}
