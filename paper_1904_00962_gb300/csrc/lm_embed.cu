// Word-table lookup with a scale, and its gradient by sorted tokens.
//
//   out[t]  = s E[id_t]                         (a row of zeros for id_t < 0)
//   dE[v] (+)= s sum over t with id_t = v of dY[t]
//
// Lookup: a copy with a gather, bound by HBM (each row read and written once); a
// warp takes a row, 16 bytes a lane.
//
// Gradient: the token positions are sorted by id (stable, least significant
// digit first, 8 bits a pass), so that every word's rows are added in the order
// of the tokens, the same in each run, and every row of dE is written once.
// Ids are Zipf-like: most words have few tokens, a handful (a mask token) have
// thousands.  Up to kLongRow tokens a word is summed by the warp that writes
// its row; a longer one is cut at every kChunk-th sorted position into partial
// sums of fixed length, which that warp adds in their order.  Sums are fp32.
#include <cuda_bf16.h>

#include "lm_vocab.h"

namespace lamb {
namespace {

constexpr int kEmbedThreads = 256;
constexpr int kSortThreads = 256;
constexpr int kSortItems = 16;                      // keys of a thread
constexpr int kSortTile = kSortThreads * kSortItems;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kChunk = 128;                         // sorted positions
constexpr int kLongRow = kChunk;
constexpr uint32_t kStatusBadIndex = LAMB_STATUS_BAD_INDEX;

__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ float load1(const __nv_bfloat16* p) {
  return __bfloat162float(*p);
}
__device__ __forceinline__ void store1(float* p, float x) { *p = x; }
__device__ __forceinline__ void store1(__nv_bfloat16* p, float x) {
  *p = __float2bfloat16_rn(x);
}
__device__ __forceinline__ void load4(const float* p, float (&x)[4]) {
  const float4 v = *reinterpret_cast<const float4*>(p);
  x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
}
__device__ __forceinline__ void load4(const __nv_bfloat16* p, float (&x)[4]) {
  const uint2 v = *reinterpret_cast<const uint2*>(p);
  x[0] = __uint_as_float(v.x << 16);
  x[1] = __uint_as_float(v.x & 0xffff0000u);
  x[2] = __uint_as_float(v.y << 16);
  x[3] = __uint_as_float(v.y & 0xffff0000u);
}
__device__ __forceinline__ void store4(float* p, const float (&x)[4]) {
  *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
}
__device__ __forceinline__ void store4(__nv_bfloat16* p, const float (&x)[4]) {
  __nv_bfloat162 a = __floats2bfloat162_rn(x[0], x[1]);
  __nv_bfloat162 b = __floats2bfloat162_rn(x[2], x[3]);
  *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<uint32_t*>(&a),
                                            *reinterpret_cast<uint32_t*>(&b));
}

// ---- lookup -----------------------------------------------------------------
template <class TI, class TO, bool kVec>
__global__ void __launch_bounds__(kEmbedThreads)
embed_kernel(const TI* __restrict__ table, int64_t table_stride,
             const int64_t* __restrict__ ids, int64_t n, int width,
             int64_t vocab, float scale, TO* __restrict__ out,
             int64_t out_stride, uint32_t* status) {
  const int lane = threadIdx.x & 31;
  const int64_t t =
      (int64_t)blockIdx.x * (kEmbedThreads / 32) + (threadIdx.x >> 5);
  if (t >= n) return;
  const int64_t id = ids[t];
  const bool real = id >= 0 && id < vocab;
  if (id >= vocab && lane == 0) atomicOr(status, kStatusBadIndex);
  const TI* src = table + (real ? id : 0) * table_stride;
  TO* dst = out + t * out_stride;
  if (kVec) {
    for (int d = lane * 4; d < width; d += 128) {
      float x[4] = {0.f, 0.f, 0.f, 0.f};
      if (real) load4(src + d, x);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] *= scale;
      if (!real) x[0] = x[1] = x[2] = x[3] = 0.f;
      store4(dst + d, x);
    }
  } else {
    for (int d = lane; d < width; d += 32)
      store1(dst + d, real ? load1(src + d) * scale : 0.f);
  }
}

// ---- sort -------------------------------------------------------------------
__device__ __forceinline__ uint32_t key_of(int64_t id, int64_t vocab,
                                           uint32_t* status) {
  if (id >= vocab) atomicOr(status, kStatusBadIndex);
  return id < 0 || id >= vocab ? (uint32_t)vocab : (uint32_t)id;
}

// How many keys of each tile have each value of the digit.
__global__ void __launch_bounds__(kSortThreads)
digit_count_kernel(const int64_t* ids, const uint32_t* keys, int64_t n,
                   int64_t vocab, int shift, int32_t* hist, int tiles,
                   uint32_t* status) {
  __shared__ int32_t count[256];
  count[threadIdx.x] = 0;
  __syncthreads();
  const int64_t base = (int64_t)blockIdx.x * kSortTile;
  for (int i = 0; i < kSortItems; ++i) {
    const int64_t at = base + i * kSortThreads + threadIdx.x;
    if (at < n) {
      const uint32_t key = ids ? key_of(ids[at], vocab, status) : keys[at];
      atomicAdd(&count[(key >> shift) & 255u], 1);
    }
  }
  __syncthreads();
  hist[(int64_t)threadIdx.x * tiles + blockIdx.x] = count[threadIdx.x];
}

// Exclusive sums in place, one CTA.
__global__ void __launch_bounds__(1024) scan_kernel(int32_t* x, int64_t n) {
  __shared__ int32_t warp_sum[32];
  __shared__ int32_t carry;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (threadIdx.x == 0) carry = 0;
  __syncthreads();
  for (int64_t base = 0; base < n; base += 1024) {
    const int64_t at = base + threadIdx.x;
    const int32_t v = at < n ? x[at] : 0;
    int32_t s = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int32_t y = __shfl_up_sync(0xffffffffu, s, o);
      if (lane >= o) s += y;
    }
    if (lane == 31) warp_sum[warp] = s;
    __syncthreads();
    if (warp == 0) {
      int32_t w = warp_sum[lane];
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int32_t y = __shfl_up_sync(0xffffffffu, w, o);
        if (lane >= o) w += y;
      }
      warp_sum[lane] = w;
    }
    __syncthreads();
    const int32_t before = carry + (warp ? warp_sum[warp - 1] : 0);
    if (at < n) x[at] = before + s - v;
    __syncthreads();
    if (threadIdx.x == 0) carry += warp_sum[31];
    __syncthreads();
  }
}

// Moves a tile's keys to their places: hist holds where the tile's first key
// of each digit goes.  A warp takes consecutive keys, 32 at a time in order, so
// that equal digits keep their order.
__global__ void __launch_bounds__(kSortThreads)
digit_move_kernel(const int64_t* ids, const uint32_t* keys, const int32_t* pos,
                  int64_t n, int64_t vocab, int shift, const int32_t* hist,
                  int tiles, uint32_t* keys_out, int32_t* pos_out,
                  uint32_t* status) {
  __shared__ int32_t count[kSortWarps][256];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  for (int i = threadIdx.x; i < kSortWarps * 256; i += kSortThreads)
    count[i >> 8][i & 255] = 0;
  __syncthreads();
  const int64_t base =
      (int64_t)blockIdx.x * kSortTile + warp * (kSortItems * 32);
  uint32_t key[kSortItems];
  int32_t rank[kSortItems];
#pragma unroll
  for (int i = 0; i < kSortItems; ++i) {
    const int64_t at = base + i * 32 + lane;
    const bool in = at < n;
    key[i] = !in ? 0u : ids ? key_of(ids[at], vocab, status) : keys[at];
    const uint32_t digit = in ? (key[i] >> shift) & 255u : 256u;
    const uint32_t same = __match_any_sync(0xffffffffu, digit);
    const int before = __popc(same & ((1u << lane) - 1u));
    rank[i] = 0;
    if (in) rank[i] = count[warp][digit] + before;
    __syncwarp();
    if (in && before == 0) count[warp][digit] += __popc(same);
    __syncwarp();
  }
  __syncthreads();
  {   // where each warp's keys of a digit start
    int32_t at = hist[(int64_t)threadIdx.x * tiles + blockIdx.x];
    for (int w = 0; w < kSortWarps; ++w) {
      const int32_t c = count[w][threadIdx.x];
      count[w][threadIdx.x] = at;
      at += c;
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kSortItems; ++i) {
    const int64_t at = base + i * 32 + lane;
    if (at >= n) continue;
    const int32_t to = count[warp][(key[i] >> shift) & 255u] + rank[i];
    keys_out[to] = key[i];
    pos_out[to] = pos ? pos[at] : (int32_t)at;
  }
}

// start[v]: first sorted position with a key of v or above.
__global__ void __launch_bounds__(256)
segments_kernel(const uint32_t* keys, int64_t n, int64_t vocab,
                int32_t* start) {
  const int64_t v = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (v > vocab) return;
  int64_t lo = 0, hi = n;
  while (lo < hi) {
    const int64_t mid = (lo + hi) >> 1;
    if (keys[mid] < (uint32_t)v) lo = mid + 1; else hi = mid;
  }
  start[v] = (int32_t)lo;
}

// ---- sums -------------------------------------------------------------------
// Sum over sorted positions [a, b) of columns d .. d + 3.
template <class TG, bool kVec>
__device__ __forceinline__ void sum_rows(const TG* grad, int64_t stride,
                                         const int32_t* pos, int a, int b,
                                         int d, int width, float (&s)[4]) {
  s[0] = s[1] = s[2] = s[3] = 0.f;
#pragma unroll 4
  for (int i = a; i < b; ++i) {
    const TG* row = grad + (int64_t)pos[i] * stride;
    if (kVec) {
      float x[4];
      load4(row + d, x);
#pragma unroll
      for (int j = 0; j < 4; ++j) s[j] += x[j];
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (d + j < width) s[j] += load1(row + d + j);
    }
  }
}

// The part that each word with a long row has in chunk blockIdx.x: the word
// that reaches into the chunk from before it (0) and the one that goes on past
// its end, or ends with it (1).
template <class TG, bool kVec>
__global__ void __launch_bounds__(kEmbedThreads)
long_rows_kernel(const TG* __restrict__ grad, int64_t stride,
                 const uint32_t* __restrict__ keys,
                 const int32_t* __restrict__ pos, int64_t n, int64_t vocab,
                 const int32_t* __restrict__ start, int width,
                 float* __restrict__ part) {
  const int64_t c0 = (int64_t)blockIdx.x * kChunk;
  const int64_t c1 = min(c0 + kChunk, n);
  const uint32_t first = keys[c0], last = keys[c1 - 1];
  for (int which = 0; which < 2; ++which) {
    const uint32_t v = which ? last : first;
    if (which && last == first) break;
    if (v >= (uint32_t)vocab) continue;
    const int64_t a = start[v], b = start[v + 1];
    if (b - a <= kLongRow) continue;
    const int from = (int)max(a, c0), to = (int)min(b, c1);
    for (int d = threadIdx.x * 4; d < width; d += kEmbedThreads * 4) {
      float s[4];
      sum_rows<TG, kVec>(grad, stride, pos, from, to, d, width, s);
      float* p = part + ((int64_t)blockIdx.x * 2 + which) * width + d;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (d + j < width) p[j] = s[j];
    }
  }
}

// One warp for each row of the table.
template <class TG, class TT, bool kVec>
__global__ void __launch_bounds__(kEmbedThreads)
embed_grad_kernel(const TG* __restrict__ grad, int64_t stride,
                  const uint32_t* __restrict__ keys,
                  const int32_t* __restrict__ pos,
                  const int32_t* __restrict__ start, int64_t vocab, int width,
                  const float* __restrict__ part, float scale, bool add,
                  TT* __restrict__ out, int64_t out_stride) {
  const int lane = threadIdx.x & 31;
  const int64_t v =
      (int64_t)blockIdx.x * (kEmbedThreads / 32) + (threadIdx.x >> 5);
  if (v >= vocab) return;
  const int a = start[v], b = start[v + 1];
  if (a == b && add) return;
  TT* dst = out + v * out_stride;
  for (int d = lane * 4; d < width; d += 128) {
    float s[4];
    if (b - a <= kLongRow) {
      sum_rows<TG, kVec>(grad, stride, pos, a, b, d, width, s);
    } else {
      s[0] = s[1] = s[2] = s[3] = 0.f;
      for (int c = a / kChunk; c <= (b - 1) / kChunk; ++c) {
        const int which = keys[(int64_t)c * kChunk] == (uint32_t)v ? 0 : 1;
        const float* p = part + ((int64_t)c * 2 + which) * width + d;
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (d + j < width) s[j] += p[j];
      }
    }
    if (kVec) {
      float x[4] = {0.f, 0.f, 0.f, 0.f};
      if (add) load4(dst + d, x);
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = add ? x[j] + s[j] * scale : s[j] * scale;
      store4(dst + d, x);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (d + j < width)
          store1(dst + d + j,
                 add ? load1(dst + d + j) + s[j] * scale : s[j] * scale);
    }
  }
}

bool vec_ok(const void* p, int dtype, int64_t stride, int width) {
  const uintptr_t bytes = dtype == LAMB_F32 ? 16 : 8;
  return (uintptr_t)p % bytes == 0 && stride % 4 == 0 && width % 4 == 0;
}

template <class TI, class TO>
void launch_embed(const lamb_vocab* v, const void* table, int64_t ts,
                  const int64_t* ids, int64_t n, float scale, void* out,
                  int64_t os, bool vec, cudaStream_t stream) {
  const unsigned grid = (unsigned)lm_ceil_div(n, kEmbedThreads / 32);
  if (vec)
    embed_kernel<TI, TO, true><<<grid, kEmbedThreads, 0, stream>>>(
        (const TI*)table, ts, ids, n, v->width, v->vocab, scale, (TO*)out, os,
        v->status);
  else
    embed_kernel<TI, TO, false><<<grid, kEmbedThreads, 0, stream>>>(
        (const TI*)table, ts, ids, n, v->width, v->vocab, scale, (TO*)out, os,
        v->status);
}

template <class TG, class TT, bool kVec>
void launch_sums(const lamb_vocab* v, const void* grad, int64_t gs, int64_t n,
                 const uint32_t* keys, const int32_t* pos, float scale,
                 bool add, void* out, int64_t os, cudaStream_t stream) {
  if (n > kLongRow)
    long_rows_kernel<TG, kVec>
        <<<(unsigned)lm_ceil_div(n, kChunk), kEmbedThreads, 0, stream>>>(
            (const TG*)grad, gs, keys, pos, n, v->vocab, v->start, v->width,
            v->part);
  embed_grad_kernel<TG, TT, kVec>
      <<<(unsigned)lm_ceil_div(v->vocab, kEmbedThreads / 32), kEmbedThreads, 0,
         stream>>>((const TG*)grad, gs, keys, pos, v->start, v->vocab, v->width,
                   v->part, scale, add, (TT*)out, os);
}

template <class TG, class TT>
void launch_grad(const lamb_vocab* v, const void* grad, int64_t gs, int64_t n,
                 const uint32_t* keys, const int32_t* pos, float scale,
                 bool add, void* out, int64_t os, bool vec,
                 cudaStream_t stream) {
  if (vec)
    launch_sums<TG, TT, true>(v, grad, gs, n, keys, pos, scale, add, out, os,
                              stream);
  else
    launch_sums<TG, TT, false>(v, grad, gs, n, keys, pos, scale, add, out, os,
                               stream);
}

lamb_status_t check_common(const lamb_vocab* v, const void* a, const char* an,
                           int a_dtype, int64_t a_stride, const int64_t* ids,
                           int64_t n, const void* b, const char* bn,
                           int b_dtype, int64_t b_stride) {
  if (!v) return lm_fail(LAMB_ERR_INVALID_ARG, "plan is NULL");
  if (n < 0 || n > v->max_tokens)
    return lm_fail(LAMB_ERR_INVALID_ARG,
                   "n_tokens %lld is not in [0, max_tokens = %lld]",
                   (long long)n, (long long)v->max_tokens);
  for (int i = 0; i < 2; ++i) {
    const int dt = i ? b_dtype : a_dtype;
    const char* name = i ? bn : an;
    if (dt != LAMB_F32 && dt != LAMB_BF16)
      return lm_fail(LAMB_ERR_UNSUPPORTED_DTYPE, "%s: dtype %d unsupported",
                     name, dt);
    if ((i ? b_stride : a_stride) < v->width)
      return lm_fail(LAMB_ERR_INVALID_ARG, "%s: row stride below the width %d",
                     name, v->width);
    const void* p = i ? b : a;
    if ((uintptr_t)p % lm_elem_size(dt))
      return lm_fail(LAMB_ERR_INVALID_ARG, "%s: pointer not aligned", name);
  }
  if (n && !ids) return lm_fail(LAMB_ERR_INVALID_ARG, "ids is NULL");
  return LAMB_OK;
}

}  // namespace

void lm_embed_carve(lamb_vocab* v, LmArena* a) {
  const int64_t n = v->max_tokens;
  v->sort_passes = 1;
  while (v->vocab >> (8 * v->sort_passes)) ++v->sort_passes;
  v->sort_tiles = lm_ceil_div(n, kSortTile);
  for (int i = 0; i < 2; ++i) {
    a->take(&v->keys[i], n);
    a->take(&v->pos[i], n);
  }
  a->take(&v->hist, 256 * v->sort_tiles);
  a->take(&v->start, v->vocab + 1);
  a->take(&v->part, lm_ceil_div(n, kChunk) * 2 * v->width);
}

}  // namespace lamb

using namespace lamb;

extern "C" lamb_status_t lamb_vocab_embed(
    struct lamb_vocab* v, const void* table, int32_t table_dtype,
    int64_t table_stride, const int64_t* ids, int64_t n_tokens, double scale,
    void* out, int32_t out_dtype, int64_t out_stride, cudaStream_t stream) {
  lamb_status_t st =
      check_common(v, table, "table", table_dtype, table_stride, ids, n_tokens,
                   out, "out", out_dtype, out_stride);
  if (st != LAMB_OK) return st;
  if (!n_tokens) return LAMB_OK;
  if (!table || !out)
    return lm_fail(LAMB_ERR_INVALID_ARG, "table and out are required");
  LmDevice dev(v->device);
  if (dev.err != cudaSuccess) return lm_cuda_fail(dev.err, "cudaSetDevice");
  const bool vec = vec_ok(table, table_dtype, table_stride, v->width) &&
                   vec_ok(out, out_dtype, out_stride, v->width);
  const float s = (float)scale;
  typedef __nv_bfloat16 bf;
  if (table_dtype == LAMB_F32 && out_dtype == LAMB_F32)
    launch_embed<float, float>(v, table, table_stride, ids, n_tokens, s, out,
                               out_stride, vec, stream);
  else if (table_dtype == LAMB_F32)
    launch_embed<float, bf>(v, table, table_stride, ids, n_tokens, s, out,
                            out_stride, vec, stream);
  else if (out_dtype == LAMB_F32)
    launch_embed<bf, float>(v, table, table_stride, ids, n_tokens, s, out,
                            out_stride, vec, stream);
  else
    launch_embed<bf, bf>(v, table, table_stride, ids, n_tokens, s, out,
                         out_stride, vec, stream);
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? LAMB_OK : lm_cuda_fail(e, "embed launch");
}

extern "C" lamb_status_t lamb_vocab_embed_grad(
    struct lamb_vocab* v, const void* grad_out, int32_t grad_dtype,
    int64_t grad_stride, const int64_t* ids, int64_t n_tokens, double scale,
    void* table_grad, int32_t table_dtype, int64_t table_stride,
    int32_t accumulate, cudaStream_t stream) {
  lamb_status_t st = check_common(v, grad_out, "grad_out", grad_dtype,
                                  grad_stride, ids, n_tokens, table_grad,
                                  "table_grad", table_dtype, table_stride);
  if (st != LAMB_OK) return st;
  if (!table_grad || (n_tokens && !grad_out))
    return lm_fail(LAMB_ERR_INVALID_ARG, "grad_out and table_grad are required");
  if (!n_tokens && accumulate) return LAMB_OK;
  LmDevice dev(v->device);
  if (dev.err != cudaSuccess) return lm_cuda_fail(dev.err, "cudaSetDevice");
  const int64_t n = n_tokens;
  const int tiles = (int)lm_ceil_div(n, kSortTile);
  int in = 0;
  for (int pass = 0; n && pass < v->sort_passes; ++pass) {
    const int64_t* src = pass ? nullptr : ids;
    digit_count_kernel<<<tiles, kSortThreads, 0, stream>>>(
        src, v->keys[in], n, v->vocab, 8 * pass, v->hist, tiles, v->status);
    scan_kernel<<<1, 1024, 0, stream>>>(v->hist, 256 * (int64_t)tiles);
    digit_move_kernel<<<tiles, kSortThreads, 0, stream>>>(
        src, v->keys[in], pass ? v->pos[in] : nullptr, n, v->vocab, 8 * pass,
        v->hist, tiles, v->keys[in ^ 1], v->pos[in ^ 1], v->status);
    in ^= 1;
  }
  segments_kernel<<<(unsigned)lm_ceil_div(v->vocab + 1, 256), 256, 0, stream>>>(
      v->keys[in], n, v->vocab, v->start);
  const bool vec = vec_ok(grad_out, grad_dtype, grad_stride, v->width) &&
                   vec_ok(table_grad, table_dtype, table_stride, v->width);
  const float s = (float)scale;
  const bool add = accumulate != 0;
  typedef __nv_bfloat16 bf;
  if (grad_dtype == LAMB_F32 && table_dtype == LAMB_F32)
    launch_grad<float, float>(v, grad_out, grad_stride, n, v->keys[in],
                              v->pos[in], s, add, table_grad, table_stride, vec,
                              stream);
  else if (grad_dtype == LAMB_F32)
    launch_grad<float, bf>(v, grad_out, grad_stride, n, v->keys[in], v->pos[in],
                           s, add, table_grad, table_stride, vec, stream);
  else if (table_dtype == LAMB_F32)
    launch_grad<bf, float>(v, grad_out, grad_stride, n, v->keys[in], v->pos[in],
                           s, add, table_grad, table_stride, vec, stream);
  else
    launch_grad<bf, bf>(v, grad_out, grad_stride, n, v->keys[in], v->pos[in], s,
                        add, table_grad, table_stride, vec, stream);
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? LAMB_OK : lm_cuda_fail(e, "embed gradient launch");
}
