// Word-table lookup with a scale, and its gradient by sorted tokens.
//
//   out[t]  = s E[id_t]                         (a row of zeros for id_t < 0)
//   dE[v] (+)= s sum over t with id_t = v of dY[t]
//
// Lookup: a copy with a gather (each row read and written once); a warp takes a row,
// four columns a lane at a time.  Bound by loads in flight: DRAM is 44% busy, as words
// that come again and half of what is written stay in L2.
//
// Gradient: the token positions are sorted by id (stable, least significant digit
// first, 8 bits a pass), so that every word's rows are added in the order of the
// tokens, the same in each run.  The sorted list is cut every 16 to 128 positions,
// whatever the words: ids are Zipf-like, most words have few tokens and a mask
// token thousands.  A chunk writes the rows of the words that lie inside it and
// leaves the sum of a word that goes on; one more launch adds those, in order.
// Sums are fp32.  Rows of words without a token are cleared during the sort.
//
// Launches follow one another early (griddepcontrol): count, a move for each digit
// (which counts the next digit), sums, joins; up to 4096 tokens are sorted in one.
//
// Measured: lookup of 65536 x 768 (fp32 to bf16) 28 us, 5.0 TB/s of its own bytes;
// gradient of 65536 x 1024 (bf16) into a fresh table 73 us, of which the sort takes 23
// with the clearing, the sums 38 and the joins 8: 27 us of HBM traffic, the rest
// latency of the longest word and of four launches in front; 4095 x 768 added to a tied
// table 20 us.
#include <cuda_bf16.h>

#include <algorithm>

#include "lamb_sync.cuh"
#include "lm_vocab.h"

namespace lamb {
namespace {

constexpr int kEmbedThreads = 256;
constexpr int kSortThreads = 512;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kSortTiles = 128;        // at most: each reads all tiles' counts
// Sorted positions of a chunk: short ones fill the SMs, long ones leave fewer sums
// to join.  us at 4095 x 768 tokens: 16 positions 23, 32 27, 64 36; at 65536 x 1024:
// 32 113, 64 85, 128 70.
constexpr int kLeastChunk = 16;
int chunk_of(int64_t n) { return n <= 8192 ? 16 : n <= 32768 ? 64 : 128; }
constexpr int kJoinThreads = 256, kJoinBatch = 8;
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

// ---- rows of zeros ------------------------------------------------------------
// The rows of a fresh table gradient are cleared by further CTAs of the sort's
// launches, whose own are too few to fill the GPU; the sums write the words with
// tokens again.  Instead of it, looking every word up in the sorted list beside the
// sums (us, V = 30522): 1 x 768 tokens to fp32 33 (now 19), 512 x 768 37 (25), 8192 x
// 1024 to bf16 41 (34), 65536 x 1024 to bf16 73 (76: a third is written twice).
constexpr int kClearRows = 32;         // of a CTA

struct Clear {
  void* out;
  int64_t stride;          // elements of `unit` bytes
  int64_t first, rows;     // of this launch
  int width, unit;
};

template <class T>
__device__ __forceinline__ void clear_rows(const Clear& c, int64_t v0, T zero) {
  const int64_t end = min(v0 + kClearRows, c.first + c.rows);
  const int lane = threadIdx.x & 31;
  for (int64_t v = v0 + (threadIdx.x >> 5); v < end; v += blockDim.x >> 5) {
    T* row = reinterpret_cast<T*>(c.out) + v * c.stride;
    for (int d = lane; d < c.width; d += 32) row[d] = zero;
  }
}
__device__ void clear_part(const Clear& c, int part) {
  const int64_t v0 = c.first + (int64_t)part * kClearRows;
  if (c.unit == 16) clear_rows(c, v0, make_uint4(0, 0, 0, 0));
  else if (c.unit == 4) clear_rows(c, v0, 0u);
  else clear_rows(c, v0, (uint16_t)0);
}
unsigned clear_ctas(const Clear& c) {
  return (unsigned)lm_ceil_div(c.rows, kClearRows);
}
__global__ void __launch_bounds__(kSortThreads) clear_kernel(Clear clear) {
  clear_part(clear, blockIdx.x);
}

// ---- sort -------------------------------------------------------------------
__device__ __forceinline__ uint32_t key_of(int64_t id, int64_t vocab,
                                           uint32_t* status) {
  if (id >= vocab) atomicOr(status, kStatusBadIndex);
  return id < 0 || id >= vocab ? (uint32_t)vocab : (uint32_t)id;
}

// The lanes with this lane's digit: a ballot for each of its eight bits (4095 keys
// in two passes 9.4 us, by the warp's match instruction 10.5).  Lanes that are not
// `in` have none.
__device__ __forceinline__ uint32_t same_digit(uint32_t digit, bool in) {
  uint32_t m = __ballot_sync(0xffffffffu, in);
#pragma unroll
  for (int b = 0; b < 8; ++b) {
    const bool bit = digit >> b & 1u;
    const uint32_t with = __ballot_sync(0xffffffffu, bit);
    m &= bit ? with : ~with;
  }
  return m;
}

// How many keys of each tile have each value of the first digit; clears what the
// moves count in.  A tile is kSortWarps runs of 32 * rounds keys, a warp's each.
__global__ void __launch_bounds__(kSortThreads)
digit_count_kernel(const int64_t* ids, int n, int64_t vocab, int rounds,
                   int passes, int32_t* hist, uint32_t* status) {
  __shared__ int32_t count[256];
  let_next_launch();
  if (threadIdx.x < 256) count[threadIdx.x] = 0;
  __syncthreads();
  const int tile = kSortThreads * rounds;
  const int64_t base = (int64_t)blockIdx.x * tile;
  for (int i = threadIdx.x; i < tile && base + i < n; i += kSortThreads)
    atomicAdd(&count[key_of(ids[base + i], vocab, status) & 255u], 1);
  __syncthreads();
  for (int i = threadIdx.x; i < 256 * passes; i += kSortThreads)
    hist[((int64_t)(i >> 8) * kSortTiles + blockIdx.x) * 256 + (i & 255)] =
        i < 256 ? count[i] : 0;
}

// Moves a tile's keys to their places in the order of one digit, equal digits in
// the order they had, and counts the next digit of the new tiles.
__global__ void __launch_bounds__(kSortThreads)
digit_move_kernel(const int64_t* ids, const uint32_t* keys, const int32_t* pos,
                  int n, int64_t vocab, int rounds, int shift,
                  const int32_t* hist, int32_t* next_hist, uint32_t* keys_out,
                  int32_t* pos_out, uint32_t* status, int tiles, Clear clear) {
  __shared__ int32_t count[kSortWarps][256];
  __shared__ int32_t half[2][2][256];      // [half][before the tile, in all]
  __shared__ int32_t scan[256];
  if ((int)blockIdx.x >= tiles) {
    let_next_launch();
    return clear_part(clear, blockIdx.x - tiles);
  }
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  for (int i = threadIdx.x; i < kSortWarps * 256; i += kSortThreads)
    count[i >> 8][i & 255] = 0;
  let_next_launch();
  after_prior_launch();
  {   // all tiles' counts of a digit, half of the tiles a thread
    const int d = threadIdx.x & 255, h = threadIdx.x >> 8;
    const int mid = (tiles + 1) / 2;
    int before = 0, total = 0;
#pragma unroll 16
    for (int t = h * mid; t < (h ? tiles : mid); ++t) {
      const int c = hist[t * 256 + d];
      total += c;
      if (t < (int)blockIdx.x) before += c;
    }
    half[h][0][d] = before;
    half[h][1][d] = total;
  }
  __syncthreads();
  const int64_t base =
      ((int64_t)blockIdx.x * kSortWarps + warp) * (rounds * 32);
  for (int i = 0; i < rounds; ++i) {
    const int64_t at = base + i * 32 + lane;
    const bool in = at < n;
    const uint32_t key =
        !in ? 0u : ids ? key_of(ids[at], vocab, status) : keys[at];
    const uint32_t digit = (key >> shift) & 255u;
    const uint32_t same = same_digit(digit, in);
    if (in && (same & ((1u << lane) - 1u)) == 0)
      count[warp][digit] += __popc(same);
    __syncwarp();
  }
  // exclusive sum over the digits, by the first warps
  int total = 0;
  if (threadIdx.x < 256) {
    total = half[0][1][threadIdx.x] + half[1][1][threadIdx.x];
    int s = total;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, s, o);
      if (lane >= o) s += y;
    }
    scan[threadIdx.x] = s;
  }
  __syncthreads();
  if (threadIdx.x < 256) {
    int at = scan[threadIdx.x] - total;
    for (int w = 0; w < warp; ++w) at += scan[w * 32 + 31];
    at += half[0][0][threadIdx.x] + half[1][0][threadIdx.x];
    for (int w = 0; w < kSortWarps; ++w) {
      const int c = count[w][threadIdx.x];
      count[w][threadIdx.x] = at;
      at += c;
    }
  }
  __syncthreads();
  const int tile = kSortThreads * rounds;
  for (int i = 0; i < rounds; ++i) {
    const int64_t at = base + i * 32 + lane;
    const bool in = at < n;
    const uint32_t key =
        !in ? 0u : ids ? key_of(ids[at], vocab, status) : keys[at];
    const uint32_t digit = (key >> shift) & 255u;
    const uint32_t same = same_digit(digit, in);
    const int before = __popc(same & ((1u << lane) - 1u));
    int to = 0;
    if (in) to = count[warp][digit] + before;
    __syncwarp();
    if (in && before == 0) count[warp][digit] += __popc(same);
    __syncwarp();
    if (in) {
      keys_out[to] = key;
      pos_out[to] = pos ? pos[at] : (int32_t)at;
    }
    if (next_hist) {      // one addition for a warp's equal places
      const int where =
          in ? to / tile * 256 + (int)((key >> (shift + 8)) & 255u) : -1;
      const uint32_t m = __match_any_sync(0xffffffffu, where);
      if (in && (m & ((1u << lane) - 1u)) == 0)
        atomicAdd(&next_hist[where], __popc(m));
    }
  }
}

// All passes for up to kSmallSort keys in one CTA: a warp's keys are consecutive,
// kSmallItems a lane.
constexpr int kSmallThreads = 1024, kSmallItems = 4;
constexpr int kSmallSort = kSmallThreads * kSmallItems;

__global__ void __launch_bounds__(kSmallThreads)
sort_small_kernel(const int64_t* ids, int n, int64_t vocab, int passes,
                  uint32_t* keys_out, int32_t* pos_out, uint32_t* status,
                  Clear clear) {
  constexpr int kWarps = kSmallThreads / 32;
  __shared__ uint32_t sm_key[kSmallSort];
  __shared__ uint16_t sm_pos[kSmallSort];
  __shared__ uint16_t count[kWarps][256];
  __shared__ int scan[256];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t past = 0xffffffffu;        // sorts behind every key
  let_next_launch();
  if (blockIdx.x) return clear_part(clear, blockIdx.x - 1);
  uint32_t key[kSmallItems], pos[kSmallItems];
#pragma unroll
  for (int i = 0; i < kSmallItems; ++i) {
    const int at = (warp * kSmallItems + i) * 32 + lane;
    key[i] = at < n ? key_of(ids[at], vocab, status) : past;
    pos[i] = at;
  }
  for (int p = 0; p < passes; ++p) {
    const int shift = 8 * p;
    for (int i = threadIdx.x; i < kWarps * 256; i += kSmallThreads)
      count[i >> 8][i & 255] = 0;
    __syncthreads();
    int rank[kSmallItems];
#pragma unroll
    for (int i = 0; i < kSmallItems; ++i) {
      const uint32_t digit = (key[i] >> shift) & 255u;
      const uint32_t same = same_digit(digit, true);
      const int before = __popc(same & ((1u << lane) - 1u));
      rank[i] = count[warp][digit] + before;
      __syncwarp();
      if (before == 0) count[warp][digit] += (uint16_t)__popc(same);
      __syncwarp();
    }
    __syncthreads();
    int total = 0, s = 0;
    int held[kWarps];           // the warps' counts of a digit
    if (threadIdx.x < 256) {
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        held[w] = count[w][threadIdx.x];
        total += held[w];
      }
      s = total;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, s, o);
        if (lane >= o) s += y;
      }
      scan[threadIdx.x] = s;
    }
    __syncthreads();
    if (threadIdx.x < 256) {
      int at = s - total;
      for (int w = 0; w < warp; ++w) at += scan[w * 32 + 31];
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        count[w][threadIdx.x] = (uint16_t)at;
        at += held[w];
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kSmallItems; ++i) {
      const int to = count[warp][(key[i] >> shift) & 255u] + rank[i];
      sm_key[to] = key[i];
      sm_pos[to] = (uint16_t)pos[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kSmallItems; ++i) {
      const int at = (warp * kSmallItems + i) * 32 + lane;
      key[i] = sm_key[at];
      pos[i] = sm_pos[at];
    }
  }
#pragma unroll
  for (int i = 0; i < kSmallItems; ++i) {
    const int at = (warp * kSmallItems + i) * 32 + lane;
    if (at < n) {
      keys_out[at] = key[i];
      pos_out[at] = (int32_t)pos[i];
    }
  }
}

// ---- sums -------------------------------------------------------------------
// kN columns of a row, kVec by whole accesses.
template <class T, int kN, bool kVec>
__device__ __forceinline__ void load_row(const T* p, int d, int width,
                                         float (&x)[kN]) {
#pragma unroll
  for (int q = 0; q < kN; q += 4) {
    if (kVec) {
      float v[4];
      load4(p + d + q, v);
#pragma unroll
      for (int j = 0; j < 4; ++j) x[q + j] = v[j];
    } else {
#pragma unroll
      for (int j = q; j < q + 4; ++j) x[j] = d + j < width ? load1(p + d + j) : 0.f;
    }
  }
}
__device__ __forceinline__ void fetch_line(const void* p) {
  asm volatile("prefetch.global.L2 [%0];" ::"l"(p));
}
// Adding to fp32 is left to the memory, which nobody waits for: each element is
// added to once in a call, so no order matters.  (It takes subnormals for zeros.)
// 32768 x 768 tokens added 62 us with a read, 50 so.  A bf16 element is read, so that
// its sum is rounded once; its line is fetched with the batch: 65536 x 1024 115 us
// without, 97 with.
__device__ __forceinline__ void add4(float* p, const float (&x)[4]) {
  asm volatile("red.global.add.v4.f32 [%0], {%1, %2, %3, %4};" ::"l"(p),
               "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3])
               : "memory");
}
__device__ __forceinline__ void add4(__nv_bfloat16*, const float (&)[4]) {}
__device__ __forceinline__ void add1(float* p, float x) {
  asm volatile("red.global.add.f32 [%0], %1;" ::"l"(p), "f"(x) : "memory");
}
__device__ __forceinline__ void add1(__nv_bfloat16*, float) {}

template <class T, int kN, bool kVec>
__device__ __forceinline__ void write_row(T* p, int d, int width,
                                          const float (&s)[kN], float scale,
                                          bool add) {
  const bool in_memory = sizeof(T) == 4 && add;
  float x[kN];
#pragma unroll
  for (int j = 0; j < kN; ++j) x[j] = 0.f;
  if (add && !in_memory) load_row<T, kN, kVec>(p, d, width, x);
#pragma unroll
  for (int j = 0; j < kN; ++j)
    x[j] = add && !in_memory ? x[j] + s[j] * scale : s[j] * scale;
  if (kVec) {
#pragma unroll
    for (int q = 0; q < kN; q += 4) {
      const float v[4] = {x[q], x[q + 1], x[q + 2], x[q + 3]};
      if (in_memory) add4(p + d + q, v);
      else store4(p + d + q, v);
    }
  } else {
#pragma unroll
    for (int j = 0; j < kN; ++j) {
      if (d + j >= width) continue;
      if (in_memory) add1(p + d + j, x[j]);
      else store1(p + d + j, x[j]);
    }
  }
}

// Rows of the gradient on their way: 16 bytes of each as they are (kVec).
template <class T, bool kVec>
struct Raw {
  static constexpr int kN = kVec ? 16 / (int)sizeof(T) : 4;
  uint4 w;
  float x[kVec ? 1 : 4];
  __device__ __forceinline__ void load(const T* p, int d, int width) {
    if (kVec) {
      w = *reinterpret_cast<const uint4*>(p + d);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        x[kVec ? 0 : j] = d + j < width ? load1(p + d + j) : 0.f;
    }
  }
  __device__ __forceinline__ void add_to(float (&s)[kN]) const {
    if (!kVec) {
#pragma unroll
      for (int j = 0; j < kN; ++j) s[j] += x[kVec ? 0 : j];
    } else {
      const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (sizeof(T) == 4) {
          s[j] += __uint_as_float(v[j]);
        } else {
          s[(2 * j) % kN] += __uint_as_float(v[j] << 16);
          s[(2 * j + 1) % kN] += __uint_as_float(v[j] & 0xffff0000u);
        }
      }
    }
  }
};

// tx threads take a chunk's rows, 16 bytes of each; kEmbedThreads / tx chunks a
// CTA.  kBatch rows are on their way at a time: HBM's latency over rows that lie
// anywhere takes some 100 KB in flight on an SM.
constexpr int kBatch = 16, kLeastTx = 8;

template <class TG, class TT, bool kVec>
__global__ void __launch_bounds__(kEmbedThreads)
embed_sums_kernel(const TG* __restrict__ grad, int64_t stride,
                  const uint32_t* __restrict__ keys,
                  const int32_t* __restrict__ pos, int n, int64_t vocab,
                  int width, int chunk, int tx, float* __restrict__ part, float scale, bool add,
                  TT* __restrict__ out, int64_t out_stride) {
  typedef Raw<TG, kVec> R;
  constexpr int kN = R::kN;
  extern __shared__ uint32_t sh_key[];       // the CTA's keys and neighbours
  let_next_launch();
  after_prior_launch();
  const int ty = kEmbedThreads / tx;
  int32_t* const sh_pos = reinterpret_cast<int32_t*>(sh_key) + ty * chunk + 2;
  const int chunk0 = blockIdx.x * ty, first = chunk0 * chunk;
  const int held = min(ty * chunk, n - first);
  const int y = threadIdx.x / tx, x0 = threadIdx.x % tx;
  const uint32_t none = 0xffffffffu;
  for (int i = threadIdx.x; i < held; i += kEmbedThreads) {
    sh_key[i + 1] = keys[first + i];
    sh_pos[i] = pos[first + i];
  }
  if (threadIdx.x == 0) {
    sh_key[0] = first ? keys[first - 1] : none;
    sh_key[held + 1] = first + held < n ? keys[first + held] : none;
  }
  __syncthreads();
  const int at0 = y * chunk;                        // inside the CTA's keys
  const int m = min(chunk, held - at0);
  if (m <= 0) return;
  float* const mine = part + (int64_t)(chunk0 + y) * 2 * width;
  const uint32_t* const key = sh_key + at0 + 1;     // -1 .. m: with neighbours
  for (int d = x0 * kN; d < width; d += tx * kN) {
    float s[kN] = {};
    bool from_before = key[-1] == key[0];
    for (int i0 = 0; i0 < m; i0 += kBatch) {
      R x[kBatch];
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        const int i = i0 + u;
        if (i < m && key[i] < (uint32_t)vocab)
          x[u].load(grad + (int64_t)sh_pos[at0 + i] * stride, d, width);
        if (sizeof(TT) == 2 && add && i < m && key[i] < (uint32_t)vocab &&
            key[i + 1] != key[i])
          fetch_line(out + (int64_t)key[i] * out_stride + d);
      }
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        const int i = i0 + u;
        if (i >= m) break;
        const uint32_t v = key[i];
        if (v >= (uint32_t)vocab) break;            // none follows either
        x[u].add_to(s);
        const bool goes_on = key[i + 1] == v;
        if (goes_on && i + 1 < m) continue;
        if (!from_before && !goes_on)
          write_row<TT, kN, kVec>(out + (int64_t)v * out_stride, d, width, s,
                                  scale, add);
        else
          write_row<float, kN, kVec>(mine + (from_before ? 0 : width), d, width,
                                     s, 1.f, false);
#pragma unroll
        for (int j = 0; j < kN; ++j) s[j] = 0.f;
        from_before = false;
      }
    }
  }
}

// The words that go on past the chunk they begin in: the CTA of that chunk adds
// the chunks' sums in their order, kJoinBatch on their way at a time.
template <class TT, bool kVec>
__global__ void __launch_bounds__(kJoinThreads)
embed_join_kernel(const uint32_t* __restrict__ keys, int n, int64_t vocab,
                  int width, int chunk, const float* __restrict__ part,
                  float scale, bool add, TT* __restrict__ out,
                  int64_t out_stride) {
  after_prior_launch();
  const int chunks = (n + chunk - 1) / chunk, c = blockIdx.x;
  const int64_t first = (int64_t)c * chunk, last = first + chunk - 1;
  if (last + 1 >= n) return;
  const uint32_t v = keys[last], after = keys[last + 1], head = keys[first];
  const uint32_t before = keys[first > 0 ? first - 1 : 0];
  if (v >= (uint32_t)vocab || after != v) return;
  if (first > 0 && head == v && before == v) return;
  // how many chunks after this one begin with the word: all threads look, in
  // steps that get shorter; count is one past the last that was seen
  int count = 1, step = (chunks - c + kJoinThreads - 1) / kJoinThreads;
  for (;;) {
    const int64_t at = c + count + (int64_t)threadIdx.x * step;
    const int with =
        __syncthreads_count(at < chunks && keys[at * chunk] == v);
    if (with > 0) count += (with - 1) * step + 1;
    if (step == 1) break;
    step = (step + kJoinThreads - 1) / kJoinThreads;
  }
  TT* dst = out + (int64_t)v * out_stride;
  for (int d = threadIdx.x * 4; d < width; d += kJoinThreads * 4) {
    float s[4];
    load_row<float, 4, kVec>(part + ((int64_t)c * 2 + 1) * width, d, width, s);
    for (int k0 = 1; k0 < count; k0 += kJoinBatch) {
      float y[kJoinBatch][4];
#pragma unroll
      for (int u = 0; u < kJoinBatch; ++u) {
        y[u][0] = y[u][1] = y[u][2] = y[u][3] = 0.f;
        if (k0 + u < count)
          load_row<float, 4, kVec>(part + (int64_t)(c + k0 + u) * 2 * width, d,
                                   width, y[u]);
      }
#pragma unroll
      for (int u = 0; u < kJoinBatch; ++u)
#pragma unroll
        for (int j = 0; j < 4; ++j) s[j] += y[u][j];
    }
    write_row<TT, 4, kVec>(dst, d, width, s, scale, add);
  }
}

// Whether rows can be taken four columns at a time (`cols`: that many).
bool vec_ok(const void* p, int dtype, int64_t stride, int width, int cols = 4) {
  const uintptr_t bytes = dtype == LAMB_F32 ? 16 : 2 * (uintptr_t)cols;
  return (uintptr_t)p % bytes == 0 && stride % cols == 0 && width % cols == 0;
}

template <class TI, class TO>
cudaError_t launch_embed(const lamb_vocab* v, const void* table, int64_t ts,
                  const int64_t* ids, int64_t n, float scale, void* out,
                  int64_t os, bool vec, cudaStream_t stream) {
  const unsigned grid = (unsigned)lm_ceil_div(n, kEmbedThreads / 32);
  return lm_launch(vec ? embed_kernel<TI, TO, true> : embed_kernel<TI, TO, false>,
                   grid, kEmbedThreads, 0, stream, false, (const TI*)table, ts,
                   ids, n, v->width, v->vocab, scale, (TO*)out, os, v->status);
}

template <class TG, class TT, bool kVec>
cudaError_t launch_sums(const lamb_vocab* v, const void* grad, int64_t gs,
                        int n, int in, float scale, bool add, void* out,
                        int64_t os, cudaStream_t stream) {
  // threads of a chunk: its columns, kLeastTx at least
  constexpr int kN = Raw<TG, kVec>::kN;
  int tx = kEmbedThreads;
  while (tx > kLeastTx && tx / 2 * kN >= v->width) tx /= 2;
  const int chunk = chunk_of(n), ty = kEmbedThreads / tx;
  const int chunks = (int)lm_ceil_div(n, chunk);
  const int ctas = (int)lm_ceil_div(chunks, ty);
  const size_t smem = (2 * (size_t)ty * chunk + 2) * 4;
  cudaError_t e = lm_launch(
      embed_sums_kernel<TG, TT, kVec>, (unsigned)ctas, kEmbedThreads, smem,
      stream, true, (const TG*)grad, gs, v->keys[in], v->pos[in], n, v->vocab,
      v->width, chunk, tx, v->part, scale, add, (TT*)out, os);
  if (e == cudaSuccess && chunks > 1)
    e = lm_launch(embed_join_kernel<TT, kVec>, (unsigned)(chunks - 1),
                  kJoinThreads, 0, stream, true, v->keys[in], n, v->vocab,
                  v->width, chunk, v->part, scale, add, (TT*)out, os);
  return e;
}

template <class TG, class TT>
cudaError_t launch_grad(const lamb_vocab* v, const void* grad, int64_t gs,
                        int n, int in, float scale, bool add, void* out,
                        int64_t os, bool vec, cudaStream_t stream) {
  return vec ? launch_sums<TG, TT, true>(v, grad, gs, n, in, scale, add, out,
                                         os, stream)
             : launch_sums<TG, TT, false>(v, grad, gs, n, in, scale, add, out,
                                          os, stream);
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
  if ((uintptr_t)ids % 8)
    return lm_fail(LAMB_ERR_INVALID_ARG, "ids: pointer not aligned");
  return LAMB_OK;
}

}  // namespace

void lm_embed_carve(lamb_vocab* v, LmArena* a) {
  const int64_t n = v->max_tokens;
  v->sort_passes = 1;
  while (v->vocab >> (8 * v->sort_passes)) ++v->sort_passes;
  for (int i = 0; i < 2; ++i) {
    a->take(&v->keys[i], n);
    a->take(&v->pos[i], n);
  }
  a->take(&v->hist, (int64_t)v->sort_passes * kSortTiles * 256);
  a->take(&v->part, lm_ceil_div(n, kLeastChunk) * 2 * v->width);
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
  cudaError_t e;
  if (table_dtype == LAMB_F32 && out_dtype == LAMB_F32)
    e = launch_embed<float, float>(v, table, table_stride, ids, n_tokens, s, out,
                                   out_stride, vec, stream);
  else if (table_dtype == LAMB_F32)
    e = launch_embed<float, bf>(v, table, table_stride, ids, n_tokens, s, out,
                                out_stride, vec, stream);
  else if (out_dtype == LAMB_F32)
    e = launch_embed<bf, float>(v, table, table_stride, ids, n_tokens, s, out,
                                out_stride, vec, stream);
  else
    e = launch_embed<bf, bf>(v, table, table_stride, ids, n_tokens, s, out,
                             out_stride, vec, stream);
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
  const int n = (int)n_tokens;
  const int rounds =
      (int)std::max<int64_t>(1, lm_ceil_div(n, kSortTiles * kSortThreads));
  const unsigned tiles = (unsigned)lm_ceil_div(n, kSortThreads * rounds);
  cudaError_t e = cudaSuccess;
  int in = 0;
  // what is to be cleared, a part with each pass of the sort
  const size_t size = lm_elem_size(table_dtype);
  const uint64_t bytes = (uint64_t)table_stride * size,
                 used = (uint64_t)v->width * size;
  const int unit =
      ((uint64_t)table_grad | bytes | used) % 16 == 0 ? 16 : (int)size;
  const auto clear = [&](int k, int parts) {
    const int64_t from = accumulate ? 0 : v->vocab * k / parts;
    const int64_t to = accumulate ? 0 : v->vocab * (k + 1) / parts;
    return Clear{table_grad,       (int64_t)(bytes / unit), from,
                 to - from,        (int)(used / unit),      unit};
  };
  if (!n) {
    e = lm_launch(clear_kernel, clear_ctas(clear(0, 1)), kSortThreads, 0, stream,
                  false, clear(0, 1));
    return e == cudaSuccess ? LAMB_OK : lm_cuda_fail(e, "clear launch");
  }
  // (4095 tokens: 31 us with a launch a pass, 29 with one in all)
  const bool small = n <= kSmallSort;
  if (small)
    e = lm_launch(sort_small_kernel, 1 + clear_ctas(clear(0, 1)),
                  kSmallThreads, 0, stream, false, ids, n, v->vocab,
                  v->sort_passes, v->keys[0], v->pos[0], v->status,
                  clear(0, 1));
  else
    e = lm_launch(digit_count_kernel, tiles, kSortThreads, 0, stream, false,
                  ids, n, v->vocab, rounds, v->sort_passes, v->hist, v->status);
  for (int pass = 0; e == cudaSuccess && !small && pass < v->sort_passes;
       ++pass) {
    int32_t* hist = v->hist + (int64_t)pass * kSortTiles * 256;
    const Clear c = clear(pass, v->sort_passes);
    e = lm_launch(digit_move_kernel, tiles + clear_ctas(c), kSortThreads, 0,
                  stream, true,
                  pass ? nullptr : ids, v->keys[in], pass ? v->pos[in] : nullptr,
                  n, v->vocab, rounds, 8 * pass, hist,
                  pass + 1 < v->sort_passes ? hist + kSortTiles * 256 : nullptr,
                  v->keys[in ^ 1], v->pos[in ^ 1], v->status, (int)tiles, c);
    in ^= 1;
  }
  if (e != cudaSuccess) return lm_cuda_fail(e, "sort launch");
  const int cols = grad_dtype == LAMB_F32 ? 4 : 8;       // 16 bytes
  const bool vec =
      vec_ok(grad_out, grad_dtype, grad_stride, v->width, cols) &&
      vec_ok(table_grad, table_dtype, table_stride, v->width);
  const float s = (float)scale;
  const bool add = accumulate != 0;
  typedef __nv_bfloat16 bf;
  if (grad_dtype == LAMB_F32 && table_dtype == LAMB_F32)
    e = launch_grad<float, float>(v, grad_out, grad_stride, n, in, s, add,
                                  table_grad, table_stride, vec, stream);
  else if (grad_dtype == LAMB_F32)
    e = launch_grad<float, bf>(v, grad_out, grad_stride, n, in, s, add,
                               table_grad, table_stride, vec, stream);
  else if (table_dtype == LAMB_F32)
    e = launch_grad<bf, float>(v, grad_out, grad_stride, n, in, s, add,
                               table_grad, table_stride, vec, stream);
  else
    e = launch_grad<bf, bf>(v, grad_out, grad_stride, n, in, s, add, table_grad,
                            table_stride, vec, stream);
  return e == cudaSuccess ? LAMB_OK : lm_cuda_fail(e, "embed gradient launch");
}
