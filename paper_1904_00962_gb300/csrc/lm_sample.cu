// Drawing a word from each row of logits.
//
//   p_i = exp((x_i - m) / T), m the largest;  the words in the order of falling x, ties
//   by index;  kept: the first top_k of them, of these the ones before which less than
//   top_p of their mass lies, of these the ones with p >= min_p; the first always.
//   With Z the mass of the kept words, the one drawn is the first, in the order of the
//   indices, up to and with which more than u Z lies.  log p(word) = (x - m) / T - log Z
//
// Masses are 64-bit integers (lm_exp.h): their sums do not depend on the order in
// which threads add, and equal values have equal masses.
//
// What is kept is a beginning of the order.  Words are counted in bins that fall with
// x (one atomic addition each, no exponential); a bin's count and middle say between
// which bins a limit lies.
//   Few words up to there: one CTA compares each with each.
//   Many: the cut is a value and a number of words that have that very value.  It is
//   found by adding up parts of the bins in question until one value is left: by one
//   CTA, which the others give their words of these bins, or by all where those are
//   too many.  Equal masses make the number of ties kept a division.
//
// In bf16 few values lie between m and the words that have no mass: 128 for each power
// of two.  There a table has the mass of each value and the bins are the values, so that
// a bin's mass is its count times one number and the cut needs no second look.
//
// A cluster of 1 to 8 CTAs has a row, a CTA a range of its columns, which it keeps in
// shared memory where that is large enough (else it reads them again, from L2 mostly).
// What CTAs tell one another they store into each other's shared memory.
//
// Bound by instructions and, with few rows, by the exchanges: reading the words is a tenth
// of it.  1,024 rows of 30,522 words in bf16 without a filter 53 us (81 without the
// table, 204 with the long form of each mass), 128 of 131,071 with top_p 62 (146, 186),
// 64 of 30,522 in fp32 with settings of their own 35, one with top_k and top_p 12.
// 1,024 rows of 30,522 in fp32: 48 greedy, 103 without a filter, 290 with top_p 0.9.  All
// forms are one kernel of 64 registers, which spills some 300 bytes.
// Among many words pairs are slow: a cut among 250 took 12 us more so than by parts.
// Tried and dropped: CTAs of 128 threads, eight on an SM, that read the row again (105
// and 194 us of the first two before the table); fp32 masses with a bound on their error,
// and the row again in full where the bound decides nothing (72 in the first, of which
// the few rows that go again are the end).
#include <cooperative_groups.h>
#include <cuda_bf16.h>

#include <algorithm>

#include "lm_exp.h"
#include "lm_rows.cuh"
#include "lm_vocab.h"

namespace cg = cooperative_groups;

namespace lamb {
namespace {

constexpr int kDrawThreads = 512;                  // of a CTA
constexpr int kDrawWarps = kDrawThreads / 32;
constexpr int kMostCtas = 8;                   // of a row
constexpr int kBins = 2048;                    // of all words
constexpr int kParts = 1024;                   // of a range of values
constexpr int kFew = 256;                      // words of which all that may be kept
constexpr int kPairs = 64;                     // words that are compared in pairs
constexpr int kHeld = 2048;                    // values of some bins that a CTA keeps
constexpr int kGather = 2048;                  // values that one CTA cuts alone
constexpr int kRoom = 220 * 1024;              // dynamic shared memory of a CTA
constexpr int kHalf = 110 * 1024;              // of one of two on an SM

__device__ const uint64_t kPowers[kExpTable] = LAMB_EXP_TABLE;

// A fraction: number * 2^-shift.
struct Ratio {
  uint64_t number;
  int shift;
};

struct DrawArgs {
  const void* logits;
  int64_t stride;
  int64_t rows;
  int vocab;
  int columns;                // of a CTA: a multiple of 8
  int bits;                   // a mass of 1 is 2^bits
  int cuts;                   // whether rows may have a top_k or a top_p
  const float* uniform;
  ExpRate rate;               // of all rows: where there is no d_ pointer
  Ratio top_p, min_p;
  int64_t top_k;
  int greedy, by_mass;        // temperature, top_p or min_p say so
  const float* d_temperature;       // NULL, or a row's own
  const float* d_top_p;
  const float* d_min_p;
  const int32_t* d_top_k;
  int64_t* ids;
  float* logprob;             // or NULL
};

// A row's settings.
struct Settings {
  ExpRate rate;
  Ratio top_p;
  uint64_t least;             // mass of a word that is kept
  uint32_t top_k;             // 0: all
  int greedy, by_mass;
  float uniform;
};

// Two numbers that the CTAs of a row add up.
struct Pair {
  uint32_t count;
  uint64_t mass;
};

struct Parts {
  uint32_t count[kParts], lo[kParts], hi[kParts];
};

// Where a limit lies: the bin, and the words in front of it and up to it.
struct Found {
  uint32_t bin, before, through;
  uint64_t mass;              // in front of it
};

struct Few {
  uint64_t word[kFew];        // key and complement of the index: falls in the order
  uint64_t mass[kFew], kept[kFew];
};
static_assert(sizeof(Parts) >= kGather * sizeof(float));

struct DrawShared {
  Settings set;
  uint32_t table_hi[kExpTable], table_lo[kExpTable], table_one[kExpTable];
  Pair slot[2][kMostCtas];    // what each CTA of the row tells, in turn
  uint64_t slot_front[kMostCtas];
  Found found[3];
  uint64_t warp_mass[kDrawWarps], scan_mass[kDrawWarps], base_mass[kDrawWarps];
  uint32_t warp_count[kDrawWarps], scan_count[kDrawWarps];
  uint64_t number;            // the mass of the first top_k
  uint32_t listed;            // words in `few` (the first CTA's), or in `held`
  uint32_t own;               // words of some bins: this CTA's
  uint32_t gathered, base;    // of all (the first CTA's); those in front of this one's
  struct { float x; uint32_t ties; } cut;
};

// Dynamic shared memory: the masses of bf16 values, in front of the rest; or words that
// the first CTA is given (where the bins are not values).
union DrawTable {
  uint64_t mass[kBins];
  float given[kGather];
};
// Its bytes: all of it for bf16, else what the given words take.
__host__ __device__ constexpr int table_bytes(int elem, bool cuts) {
  return elem == 2 ? (int)sizeof(DrawTable) : cuts ? kGather * (int)sizeof(float) : 0;
}
// In front of the columns, where rows may have a cut.
struct DrawCuts {
  uint32_t bins[kBins];
  union {
    Parts parts;
    Few few;
  };
  float held[kHeld];          // values of the CTA's words in some bins
};

// number * mass * 2^-shift, rounded down; or (up) to 53 bits and then up, so that 0.9 of
// 300 words is 270, whatever 0.9 is in fp64, and more than nothing is 1.
__device__ __forceinline__ uint64_t times(const Ratio& r, uint64_t mass, bool up) {
  const uint64_t hi = __umul64hi(r.number, mass), lo = r.number * mass;
  if (r.shift >= 128) return up && (hi | lo);
  uint64_t x = lo, rest = 0;            // rest: 2^-64 of one
  if (r.shift >= 64) {
    const int k = r.shift - 64;
    x = hi >> k;
    rest = k ? hi << (64 - k) | lo >> k : lo;
  } else if (r.shift) {
    x = hi << (64 - r.shift) | lo >> r.shift;
    rest = lo << (64 - r.shift);
  }
  if (!up) return x;
  const int extra = 11 - __clzll(x);    // bits beyond 53
  if (extra > 0) return ((x >> (extra - 1)) + 1) >> 1 << extra;
  return x ? x + (rest > x << 11) : (hi | lo) != 0;
}
// Of a number in (0, 1] (0 below it, all of it above).
__device__ __forceinline__ Ratio ratio_of(float x) {
  if (!(x > 0.f)) return {0, 1};
  if (x > 1.f) return {1, 0};
  const uint32_t b = __float_as_uint(x);
  const int e = b >> 23;
  return {(b & 0x7fffffu) | (e ? 0x800000u : 0u), 150 - max(e, 1)};
}

// Numbers in the order of logits; -0 is 0, and a NaN is beyond all others.  (From the bits
// alone: a NaN that a sum gives has no certain sign.)
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t bits = __float_as_uint(x);
  const uint32_t b = bits == 0x80000000u ? 0u : bits;
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float of_key(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
}
__device__ __forceinline__ uint64_t warp_sum(uint64_t x) {
#pragma unroll
  for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}

// 16 bytes of logits.
template <class T>
struct Vec;
template <>
struct Vec<float> {
  static constexpr int n = 4;
  __device__ static void get(const uint4& v, float (&x)[4]) {
    x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y);
    x[2] = __uint_as_float(v.z); x[3] = __uint_as_float(v.w);
  }
  __device__ static uint4 put(const float (&x)[4]) {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]),
                      __float_as_uint(x[2]), __float_as_uint(x[3]));
  }
  __device__ static float one(const float* p) { return *p; }
  // The largest (of those that are numbers).
  __device__ static float largest(const uint4& v) {
    return fmaxf(fmaxf(__uint_as_float(v.x), __uint_as_float(v.y)),
                 fmaxf(__uint_as_float(v.z), __uint_as_float(v.w)));
  }
  __device__ static uint4 none() {
    return make_uint4(0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u);
  }
  // Whether one is below `tiny` in size: none as a rule that is asked for.
  __device__ static bool has_tiny(const uint4&, float) { return false; }
  // Each at least `lower` (NaN, too).
  __device__ static uint4 raise(const uint4& v, float lower) {
    return make_uint4(__float_as_uint(fmaxf(__uint_as_float(v.x), lower)),
                      __float_as_uint(fmaxf(__uint_as_float(v.y), lower)),
                      __float_as_uint(fmaxf(__uint_as_float(v.z), lower)),
                      __float_as_uint(fmaxf(__uint_as_float(v.w), lower)));
  }
};
template <>
struct Vec<__nv_bfloat16> {
  static constexpr int n = 8;
  __device__ static void get(const uint4& v, float (&x)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  __device__ static uint4 put(const float (&x)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      w[i] = __float_as_uint(x[2 * i]) >> 16 |
             (__float_as_uint(x[2 * i + 1]) & 0xffff0000u);
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  __device__ static float one(const __nv_bfloat16* p) {
    return __bfloat162float(*p);
  }
  __device__ static uint4 none() {
    return make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u);
  }
  __device__ static uint32_t max2(uint32_t a, uint32_t b) {
    uint32_t m;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(m) : "r"(a), "r"(b));
    return m;
  }
  __device__ static uint32_t min2(uint32_t a, uint32_t b) {
    uint32_t m;
    asm("min.bf16x2 %0, %1, %2;" : "=r"(m) : "r"(a), "r"(b));
    return m;
  }
  __device__ static bool has_tiny(const uint4& v, float tiny) {
    constexpr uint32_t k = 0x7fff7fffu;
    const uint32_t m = min2(min2(v.x & k, v.y & k), min2(v.z & k, v.w & k));
    return fminf(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u)) < tiny;
  }
  // Of two logits' bits, numbers that fall as they rise (+0: 0x7fff, -0: 0x8000).
  __device__ static uint32_t falling(uint32_t w) {
    uint32_t negative;                  // 0xffff where one is
    asm("prmt.b32 %0, %1, 0, 0xbb99;" : "=r"(negative) : "r"(w));
    return w ^ (~negative & 0x7fff7fffu);
  }
  __device__ static float value_of(uint32_t falling) {
    return __uint_as_float(
        (falling & 0x8000u ? falling : falling ^ 0x7fffu) << 16);
  }
  __device__ static float largest(const uint4& v) {
    const uint32_t m = max2(max2(v.x, v.y), max2(v.z, v.w));
    return fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
  }
  __device__ static uint4 raise(const uint4& v, float lower) {
    const uint32_t b = __float_as_uint(lower);
    const uint32_t w = (b & 0xffff0000u) | b >> 16;
    return make_uint4(max2(v.x, w), max2(v.y, w), max2(v.z, w), max2(v.w, w));
  }
};

__device__ __forceinline__ uint32_t min_u16x2(uint32_t a, uint32_t b) {
  uint32_t m;
  asm("min.u16x2 %0, %1, %2;" : "=r"(m) : "r"(a), "r"(b));
  return m;
}
__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b) {
  uint32_t m;
  asm("max.u16x2 %0, %1, %2;" : "=r"(m) : "r"(a), "r"(b));
  return m;
}

// The values of bf16 logits from m down to `lower`, numbered from 0: falling() less its
// first, without those in [gap0, gap1] around zero, which are too many.  Those share
// the number gap0 - first; words among them are looked at one by one.
struct Values {
  uint32_t first, gap0, gap1;           // twice each, in both halves; first: and gap1
  uint32_t gap_number;                  // beyond kBins: there is no gap
  int last;                             // number of `lower`
  float gap;                            // size of the numbers in the gap: below this

  // Where there are more than kBins, as many around zero are left out.
  __device__ void set(float m, float lower) {
    uint32_t top = falling1(m), end = falling1(lower);
    if ((int)(end - top) >= kBins - 1) {
      // (of one sign, down to a very small one: all the small ones are left out)
      if (top > 0x8000u) top = 0x8000u;
      if (end < 0x7fffu) end = 0x7fffu;
    }
    const int range = (int)(end - top) + 1;
    const int above = top < 0x8000u ? (int)(0x8000u - top) : 0;
    const int below = end >= 0x8000u ? (int)(end - 0x7fffu) : 0;
    const int extra = range - (kBins - 1);
    const bool across = (above && below) || extra > 0;
    int half = across;                  // (the zeros are two, and equal)
    if (extra > 0) {
      const int less = min(above, below);
      half = max(half, 2 * less >= extra ? (extra + 1) / 2 : extra - less);
    }
    const uint32_t g0 = 0x8000u - min(above, half), g1 = 0x7fffu + min(below, half);
    gap0 = g0 * 0x10001u;
    gap1 = g1 * 0x10001u;
    first = (top + g1) * 0x10001u;
    gap_number = across ? g0 - top : 2 * kBins;
    last = (int)(min(end, g0) - top + max(end, g1) - g1);
    gap = across ? __uint_as_float((uint32_t)half << 16) : 0.f;
  }
  __device__ static uint32_t falling1(float x) {
    return Vec<__nv_bfloat16>::falling(__float_as_uint(x) >> 16) & 0xffffu;
  }
  // Of two logits that are not below `lower`.
  __device__ __forceinline__ uint32_t numbers(uint32_t w) const {
    const uint32_t f = Vec<__nv_bfloat16>::falling(w);
    return min_u16x2(f, gap0) + max_u16x2(f, gap1) - first;
  }
  __device__ float value(uint32_t number) const {
    const uint32_t g0 = gap0 & 0xffffu, g1 = gap1 & 0xffffu;
    const uint32_t top = (first - gap1) & 0xffffu;
    const int from_gap = (int)number - (int)(g0 - top);
    return Vec<__nv_bfloat16>::value_of(from_gap < 0 ? top + number : g1 + from_gap);
  }
};

// A CTA's columns of a row in units of 16 bytes; the first unit starts `shift` columns
// in front of them, on 16 bytes.
template <class T, bool kStaged>
struct Columns {
  static constexpr int n = Vec<T>::n;
  const T* row;               // at the CTA's first column
  uint4* kept;
  int shift, len, units;

  __device__ __forceinline__ bool whole(int u) const {
    return u * n >= shift && (u + 1) * n - shift <= len;
  }
  __device__ __forceinline__ uint4 load(int u) const {
    return *reinterpret_cast<const uint4*>(row + (u * n - shift));
  }
  __device__ __forceinline__ uint4 from_memory(int u) const {
    if (whole(u)) return load(u);
    const int at = u * n - shift;
    float x[n];
#pragma unroll
    for (int j = 0; j < n; ++j)
      x[j] = at + j >= 0 && at + j < len ? Vec<T>::one(row + at + j) : -INFINITY;
    return Vec<T>::put(x);
  }
  __device__ __forceinline__ uint4 raw(int u) const {
    return kStaged ? kept[u] : from_memory(u);
  }
  __device__ __forceinline__ void get(int u, float (&x)[n]) const {
    Vec<T>::get(raw(u), x);
  }
};

template <class T, bool kStaged>
struct Draw {
  static constexpr int n = Vec<T>::n;
  const DrawArgs& a;
  DrawShared& s;
  DrawCuts& k;
  DrawTable& table;           // (bf16)
  cg::cluster_group cluster;
  int rank, ctas;
  int turn;                   // of the slots
  float m;
  ExpRate rate;
  float scale;                // bins of a unit of exp_place
  float tiny;                 // logits below have no exact distance from m (bf16)
  float lower;                // logits below have no mass; m: not known
  bool tabled;
  Values values;
  uint64_t gap_mass;          // of the words in the values' gap
  Columns<T, kStaged> c;

  __device__ __forceinline__ Draw(const DrawArgs& args, DrawShared& shared,
                                  DrawTable& masses, DrawCuts& cuts)
      : a(args), s(shared), k(cuts), table(masses), cluster(cg::this_cluster()) {
    rank = cluster.block_rank();
    ctas = cluster.num_blocks();
    turn = 0;
  }

  // All threads of the row.
  __device__ __forceinline__ void sync() {
    if (ctas == 1) __syncthreads();
    else cluster.sync();
  }
  // Every CTA's pair, in s.slot[the turn returned]; `mine` is the CTA's in the first
  // threads, one for each CTA.
  __device__ __forceinline__ int tell(const Pair& mine) {
    const int t = turn;
    turn ^= 1;
    if (threadIdx.x < ctas)
      *cluster.map_shared_rank(&s.slot[t][rank], threadIdx.x) = mine;
    sync();
    return t;
  }
  // Of each warp in s.warp_..., and over the CTA in the first threads (as tell() takes
  // it).
  __device__ __forceinline__ Pair cta_sum(uint32_t count, uint64_t mass) {
    count = __reduce_add_sync(0xffffffffu, count);
    mass = warp_sum(mass);
    if ((threadIdx.x & 31) == 0) {
      s.warp_count[threadIdx.x >> 5] = count;
      s.warp_mass[threadIdx.x >> 5] = mass;
    }
    __syncthreads();
    Pair p = {0, 0};
    if (threadIdx.x < 32) {
      if (threadIdx.x < kDrawWarps) p = {s.warp_count[threadIdx.x], s.warp_mass[threadIdx.x]};
      p.count = __reduce_add_sync(0xffffffffu, p.count);
      p.mass = warp_sum(p.mass);
    }
    return p;
  }
  // Over the row, in every thread.
  __device__ __forceinline__ uint64_t row_sum(uint64_t mass) {
    const int t = tell(cta_sum(0, mass));
    mass = 0;
    for (int q = 0; q < ctas; ++q) mass += s.slot[t][q].mass;
    return mass;
  }
  // What is in front of each thread, and in all of the CTA.
  __device__ __forceinline__ Pair scan(const Pair& own, Pair& all) {
    Pair in = own;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t count = __shfl_up_sync(0xffffffffu, in.count, o);
      const uint64_t mass = __shfl_up_sync(0xffffffffu, in.mass, o);
      if (lane >= o) {
        in.count += count;
        in.mass += mass;
      }
    }
    __syncthreads();
    if (lane == 31) {
      s.scan_count[warp] = in.count;
      s.scan_mass[warp] = in.mass;
    }
    __syncthreads();
    Pair warps = {0, 0};                // up to and with warp `lane`
    if (lane < kDrawWarps) warps = {s.scan_count[lane], s.scan_mass[lane]};
    warps = lanes_scan(warps);
    all = of_lane(warps, kDrawWarps - 1);
    const Pair front = of_lane(warps, max(warp, 1) - 1);
    Pair before = {in.count - own.count, in.mass - own.mass};
    if (warp) {
      before.count += front.count;
      before.mass += front.mass;
    }
    return before;
  }
  // Sums up to and with each of the first kDrawWarps lanes.
  __device__ __forceinline__ static Pair lanes_scan(Pair p) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 1; o < kDrawWarps; o <<= 1) {
      const uint32_t count = __shfl_up_sync(0xffffffffu, p.count, o);
      const uint64_t mass = __shfl_up_sync(0xffffffffu, p.mass, o);
      if (lane >= o) {
        p.count += count;
        p.mass += mass;
      }
    }
    return p;
  }
  __device__ __forceinline__ static Pair of_lane(const Pair& p, int lane) {
    return {__shfl_sync(0xffffffffu, p.count, lane),
            __shfl_sync(0xffffffffu, p.mass, lane)};
  }
  // The CTA's largest and least.
  __device__ __forceinline__ void cta_extent(uint32_t& most, uint32_t& least) {
    most = __reduce_max_sync(0xffffffffu, most);
    least = __reduce_min_sync(0xffffffffu, least);
    if ((threadIdx.x & 31) == 0) {
      s.warp_count[threadIdx.x >> 5] = most;
      s.warp_mass[threadIdx.x >> 5] = least;
    }
    __syncthreads();
    const int lane = threadIdx.x & (kDrawWarps - 1);
    most = __reduce_max_sync(0xffffffffu, s.warp_count[lane]);
    least = __reduce_min_sync(0xffffffffu, (uint32_t)s.warp_mass[lane]);
  }
  // The row's.
  __device__ __forceinline__ void row_extent(uint32_t& most, uint32_t& least) {
    cta_extent(most, least);
    const int t = tell({most, least});
    for (int q = 0; q < ctas; ++q) {
      most = max(most, s.slot[t][q].count);
      least = min(least, (uint32_t)s.slot[t][q].mass);
    }
  }

  __device__ __forceinline__ uint64_t one() const { return 1ull << a.bits; }
  // Whether a word counts: its mass is about a unit at least.
  __device__ __forceinline__ bool counts(float x, float y) const {
    return x == m || y < (float)a.bits;
  }
  __device__ __forceinline__ float place(float x) const {
    return exp_place(x, m, rate);
  }
  __device__ __forceinline__ uint64_t mass(float x) const {
    const float y = place(x);
    if (!(y >= kExpFar) || (sizeof(T) == 2 && fabsf(x) < tiny)) {
      if (x == m) return one();
      if (!(y < (float)a.bits)) return 0;
      return fixed_exp(x, m, rate, y, a.bits, s.table_hi, s.table_lo);
    }
    if (!(y < (float)a.bits)) return 0;
    return fixed_exp_far<sizeof(T) == 2>(x, m, rate, y, a.bits, s.table_one);
  }
  // mass() of 16 bytes of logits, bit by bit: from the table, or two at a time by
  // fixed_exp_far's steps without a branch; those near m or of no exact distance (in the
  // table's gap) one by one.
  __device__ __forceinline__ void masses(const uint4& raw, uint64_t (&p)[n]) const {
    float x[n];
    if (sizeof(T) == 2 && tabled) {
      const uint4 v = Vec<T>::raise(raw, lower);
      const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int i = 0; i < n / 2; ++i) {
        const uint32_t two = values.numbers(w[i & 3]);
        p[2 * i] = table.mass[two & 0xffffu];
        p[2 * i + 1] = table.mass[two >> 16];
      }
      if (Vec<T>::has_tiny(raw, values.gap)) {
        Vec<T>::get(raw, x);
#pragma unroll
        for (int j = 0; j < n; ++j)
          if (fabsf(x[j]) < values.gap) p[j] = mass(x[j]);
      }
      return;
    }
    bool odd = !(lower < m) || Vec<T>::has_tiny(raw, tiny);
    if (!odd) {
      Vec<T>::get(Vec<T>::raise(raw, lower), x);
      constexpr float kK = 393216.f;                    // 1.5 2^23 / 32
      constexpr float L = 0.69314718055994531f, k37 = 0x1p37f;
      constexpr float c1 = L * k37, c2 = L * L / 2 * k37, c3 = L * L * L / 6 * k37,
                      c4 = L * L * L * L / 24 * k37;
      const Two minus = two(-1.f, -1.f);
#pragma unroll
      for (int j = 0; j < n; j += 2) {
        const Two x2 = two(x[j], x[j + 1]), m2 = two(m, m);
        const Two d = fma2(x2, minus, m2);
        const Two y = mul2(d, two(rate.hi, rate.hi));
        Two less = fma2(d, two(-rate.hi, -rate.hi), y);     // -y_lo
        less = fma2(d, two(-rate.lo, -rate.lo), less);
        if (sizeof(T) == 4) {
          const Two b = fma2(m2, minus, d);
          const Two e = fma2(fma2(b, minus, d), minus, m2);
          const Two f = fma2(add2(x2, b), minus, e);
          less = fma2(f, two(-rate.hi, -rate.hi), less);
        }
        const Two t = add2(y, two(kK, kK));
        const Two z = add2(fma2(y, minus, add2(t, two(-kK, -kK))), less);
        Two w = fma2(z, two(c4, c4), two(c3, c3));
        w = fma2(z, w, two(c2, c2));
        w = mul2(z, fma2(z, w, two(c1, c1)));
        float ws[2], ts[2], ys[2];
        apart(w, ws[0], ws[1]);
        apart(t, ts[0], ts[1]);
        apart(y, ys[0], ys[1]);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint32_t at = __float_as_uint(ts[i]);
          const uint32_t power = s.table_one[at & 31];
          const int32_t more =
              (__mulhi((int32_t)(power >> 1), __float2int_rn(ws[i])) + 8) >> 4;
          p[j + i] = (uint64_t)(power + (uint32_t)more) << (a.bits - 31) >>
                     (at >> 5 & 63);
          odd |= ys[i] < kExpFar;
        }
      }
    }
    if (odd) {
      Vec<T>::get(raw, x);
#pragma unroll
      for (int j = 0; j < n; ++j)
        if (!(lower < m) || !(place(x[j]) >= kExpFar) ||
            (sizeof(T) == 2 && Vec<T>::has_tiny(raw, tiny)))
          p[j] = mass(x[j]);
    }
  }
  // A bin's number, as long as it is not rounded down; 0 where x is m.
  __device__ __forceinline__ float bin_place(float x, float y) const {
    return x == m ? 0.f : y * scale;
  }
  __device__ __forceinline__ uint32_t bin_at(float x, float y) const {
    return min((uint32_t)bin_place(x, y), (uint32_t)kBins - 1);
  }

  // f(unit, its 16 bytes) from u0 in steps up to u1 (beyond the columns: any); two
  // units ahead are on their way where they come from memory.
  template <class F>
  __device__ __forceinline__ void walk(int u0, int u1, int step, const F& f) const {
    if (kStaged) {
#pragma unroll 1
      for (int u = u0; u < u1; u += step) f(u, c.raw(min(u, c.units - 1)));
      return;
    }
    uint4 now = {}, next = {};
    if (u0 < u1) now = c.raw(u0);
    if (u0 + step < u1) next = c.raw(u0 + step);
#pragma unroll 1
    for (int u = u0; u < u1; u += step) {
      const uint4 v = now;
      now = next;
      if (u + 2 * step < u1) next = c.raw(u + 2 * step);
      f(u, v);
    }
  }
  // f(x, index) of each of the CTA's columns (and of up to 15 of -inf beside them).
  template <class F>
  __device__ __forceinline__ void each(const F& f) const {
    walk(threadIdx.x, c.units, kDrawThreads, [&](int u, const uint4& v) {
      float x[n];
      Vec<T>::get(v, x);
#pragma unroll
      for (int j = 0; j < n; ++j)
        f(x[j], (uint32_t)(rank * a.columns + u * n - c.shift + j));
    });
  }
  // How many of some units, neighbours, a warp has: 32 at a time.
  __device__ __forceinline__ static int warp_units(int units) {
    return (units + kDrawThreads - 1) / kDrawThreads * 32;
  }

  // Bins are cut into a range for each thread of every CTA, parts into one for each
  // of the row.
  static constexpr int kOwnBins = kBins / kDrawThreads;
  struct Range {
    int first, bins;
    uint32_t of[kOwnBins];    // the row's, of each bin
    Pair before, own;         // in front of and in the thread's range
    Pair total;               // of all bins
  };
  // The mass of a bin's words, if all were in its middle: within 0.75% (of 44 / 2,048
  // in base 2) where the bin has a mass worth speaking of.
  __device__ __forceinline__ uint64_t bin_mass(int bin, uint32_t count) const {
    return (uint64_t)((float)count * exp2f((float)a.bits - (bin + 0.5f) / scale));
  }
  __device__ __forceinline__ uint64_t count_mass(int bin, uint32_t count) const {
    if (sizeof(T) == 2 && tabled)
      return bin == values.gap_number ? gap_mass : count * table.mass[bin];
    return bin_mass(bin, count);
  }
  // The row's bins, in every CTA: each adds up all, or, of eight CTAs, a part of them
  // for all (one row with top_k 50: 0.7 us less so).
  __device__ __forceinline__ Range gather_bins() {
    sync();
    Range r;
    r.bins = kOwnBins;
    r.first = threadIdx.x * kOwnBins;
    static_assert(kOwnBins == 4, "bins are read 16 bytes at a time");
    uint4 of = *reinterpret_cast<const uint4*>(k.bins + r.first);
    if (ctas <= 4) {
#pragma unroll
      for (int q = 1; q < 4; ++q) {
        if (q >= ctas) break;
        const uint32_t* other =
            cluster.map_shared_rank(k.bins, (q + rank) & (ctas - 1));
        const uint4 v = *reinterpret_cast<const uint4*>(other + r.first);
        of.x += v.x;
        of.y += v.y;
        of.z += v.z;
        of.w += v.w;
      }
    } else {
      const int of_cta = kBins / ctas;
      for (int i = rank * of_cta + threadIdx.x; i < (rank + 1) * of_cta;
           i += kDrawThreads) {
        uint32_t count = 0;
#pragma unroll
        for (int q = 0; q < kMostCtas; ++q)
          if (q < ctas) count += cluster.map_shared_rank(k.bins, q)[i];
        // (only this CTA reads these bins of the others)
        for (int q = 0; q < ctas; ++q) cluster.map_shared_rank(k.bins, q)[i] = count;
      }
      cluster.sync();
      of = *reinterpret_cast<const uint4*>(k.bins + r.first);
    }
    r.of[0] = of.x;
    r.of[1] = of.y;
    r.of[2] = of.z;
    r.of[3] = of.w;
    r.own = {0, 0};
#pragma unroll
    for (int i = 0; i < kOwnBins; ++i) {
      r.own.count += r.of[i];
      r.own.mass += count_mass(r.first + i, r.of[i]);
    }
    r.before = scan(r.own, r.total);
    return r;
  }
  __device__ __forceinline__ Range gather_parts() {
    sync();
    Range r;
    const int of_cta = kParts / ctas;
    r.bins = max(1, of_cta / kDrawThreads);
    r.first = rank * of_cta + threadIdx.x * r.bins;
    if (threadIdx.x * r.bins >= of_cta) r.bins = 0;
    r.own = {0, 0};
    for (int i = r.first; i < r.first + r.bins; ++i) {
      Pair p = {0, 0};
#pragma unroll
      for (int q = 0; q < kMostCtas; ++q) {
        if (q >= ctas) break;
        const Parts* o = cluster.map_shared_rank(&k.parts, q);
        p.count += o->count[i];
        p.mass += o->lo[i] + ((uint64_t)o->hi[i] << 32);
      }
      k.parts.count[i] = p.count;
      k.parts.lo[i] = (uint32_t)p.mass;
      k.parts.hi[i] = (uint32_t)(p.mass >> 32);
      r.own.count += p.count;
      r.own.mass += p.mass;
    }
    Pair cta;
    r.before = scan(r.own, cta);
    const int t = tell(cta);
    for (int q = 0; q < rank; ++q) {
      r.before.count += s.slot[t][q].count;
      r.before.mass += s.slot[t][q].mass;
    }
    return r;
  }
  // The bin in which the count, or the mass as count_mass has it, passes a target that
  // is not above the row's: in s.found[which] of every CTA.
  __device__ __forceinline__ void find_bin(const Range& r, int which, bool by_mass,
                                           uint64_t target) {
    const uint64_t lo = by_mass ? r.before.mass : r.before.count;
    const uint64_t hi = lo + (by_mass ? r.own.mass : r.own.count);
    if (!(lo < target && target <= hi)) return;
    Pair at = r.before;
    bool found = false;
#pragma unroll
    for (int i = 0; i < kOwnBins; ++i) {
      const uint32_t n_bin = r.of[i];
      const uint64_t p = count_mass(r.first + i, n_bin);
      if (!found && target <= (by_mass ? at.mass + p : (uint64_t)at.count + n_bin)) {
        s.found[which] = {(uint32_t)(r.first + i), at.count, at.count + n_bin, at.mass};
        found = true;
      }
      at.count += n_bin;
      at.mass += p;
    }
  }
  __device__ __forceinline__ void find_part(const Range& r, bool by_mass,
                                            uint64_t target, const Pair& base) {
    Pair at = {r.before.count + base.count, r.before.mass + base.mass};
    const uint64_t lo = by_mass ? at.mass : at.count;
    const uint64_t hi = lo + (by_mass ? r.own.mass : r.own.count);
    if (lo < target && target <= hi) {
      int i = r.first;
      for (;; ++i) {
        const uint64_t p = k.parts.lo[i] + ((uint64_t)k.parts.hi[i] << 32);
        if (target <=
            (by_mass ? at.mass + p : (uint64_t)at.count + k.parts.count[i]))
          break;
        at.count += k.parts.count[i];
        at.mass += p;
      }
      for (int q = 0; q < ctas; ++q)
        *cluster.map_shared_rank(&s.found[0], q) = {(uint32_t)i, at.count, 0,
                                                    at.mass};
    }
    sync();
  }

  __device__ __forceinline__ void add_to_part(uint32_t i, uint64_t p) {
    const uint32_t low = (uint32_t)p;
    const uint32_t old = atomicAdd(&k.parts.lo[i], low);
    const uint32_t high = (uint32_t)(p >> 32) + (old + low < old);
    if (high) atomicAdd(&k.parts.hi[i], high);
  }
  // The value among those with keys in [lo, hi] at which the count (or mass) passes the
  // target; `before`: what lies in front of hi, then of the value.
  __device__ __forceinline__ float cut(uint32_t lo, uint32_t hi, bool by_mass,
                                       uint64_t target, Pair& before) {
    while (lo < hi) {
      // parts of [lo, hi], from the top
      const int shift = max(0, 32 - __clz(hi - lo) - 10);
      for (int i = threadIdx.x; i < kParts; i += kDrawThreads)
        k.parts.count[i] = k.parts.lo[i] = k.parts.hi[i] = 0;
      __syncthreads();
      each([&](float x, uint32_t) {
        const uint32_t key = key_of(x);
        if (key < lo || key > hi) return;
        const uint32_t i = (hi - key) >> shift;
        if (!by_mass) {
          atomicAdd(&k.parts.count[i], 1u);
          return;
        }
        add_to_part(i, mass(x));
      });
      const Range r = gather_parts();
      find_part(r, by_mass, target, before);
      const uint32_t part = s.found[0].bin;
      before = {s.found[0].before, s.found[0].mass};
      uint32_t lo2 = 0xffffffffu, hi2 = 0;
      each([&](float x, uint32_t) {
        const uint32_t key = key_of(x);
        if (key < lo || key > hi || ((hi - key) >> shift) != part) return;
        lo2 = min(lo2, key);
        hi2 = max(hi2, key);
      });
      row_extent(hi2, lo2);
      lo = lo2;
      hi = hi2;
    }
    return of_key(lo);
  }

  // Puts a word into the first CTA's list.
  __device__ __forceinline__ void list(float x, uint32_t index) {
    Few& f = *cluster.map_shared_rank(&k.few, 0);
    f.word[atomicAdd(cluster.map_shared_rank(&s.listed, 0), 1u)] =
        (uint64_t)key_of(x) << 32 | (uint32_t)~index;
  }
  // f(x) of the words with bins in [first, last], of those that CTAs hold or of all.
  template <class F>
  __device__ __forceinline__ void in_bins(bool held, uint32_t first, uint32_t last,
                                          const F& f) const {
    const auto one = [&](float x) {
      const float y = place(x);
      if (!counts(x, y)) return;
      const uint32_t bin = bin_at(x, y);
      if (bin >= first && bin <= last) f(x);
    };
    if (held) {
      for (int i = threadIdx.x; i < s.listed; i += kDrawThreads) one(k.held[i]);
    } else {
      each([&](float x, uint32_t) { one(x); });
    }
  }
  // The value among the words of the bins [first, last] at which the count or mass passes
  // the target, and how many of it there are up to there; front: what lies in front of
  // the bins, exactly; held: CTAs hold their words of the bins.
  __device__ __forceinline__ float cut_bins(const Range& r, Found first, Found last,
                                            bool held, bool by_mass, uint64_t target,
                                            Pair front, uint32_t& ties) {
    // masses by bins are within 0.76% from the first bin on: narrower, twice at most
#pragma unroll 1
    for (int turns = 0;
         by_mass && turns < 2 && last.through - first.before > kGather; ++turns) {
      const uint64_t left = target - front.mass;
      find_bin(r, 1, true, first.mass + max((uint64_t)1, left - left / 62));
      find_bin(r, 2, true, min(first.mass + left + left / 62, r.total.mass));
      __syncthreads();
      const uint32_t begin = first.bin;
      first = s.found[1];
      if (s.found[2].bin < last.bin) last = s.found[2];
      uint64_t sum = 0;
      if (begin < first.bin)
        in_bins(held, begin, first.bin - 1, [&](float x) { sum += mass(x); });
      front = {first.before, front.mass + row_sum(sum)};
    }
    const int number = (int)(last.through - first.before);
    if (number > kGather) {
      uint32_t lo = 0xffffffffu, hi = 0;
      in_bins(held, first.bin, last.bin, [&](float x) {
        lo = min(lo, key_of(x));
        hi = max(hi, key_of(x));
      });
      row_extent(hi, lo);
      const float x = cut(lo, hi, by_mass, target, front);
      ties = by_mass ? ties_of(x, target - front.mass)
                     : (uint32_t)target - front.count;
      return x;
    }
    // to the first CTA: few in any order, more with each CTA's in one piece
    if (number <= kPairs) {
      float* given = cluster.map_shared_rank(table.given, 0);
      uint32_t* gathered = cluster.map_shared_rank(&s.gathered, 0);
      in_bins(held, first.bin, last.bin,
              [&](float x) { given[atomicAdd(gathered, 1u)] = x; });
      sync();
      if (rank == 0) {
        pair_given(number, by_mass, target, by_mass ? front.mass : front.count);
        if (threadIdx.x == 0) s.gathered = 0;
      }
      sync();
      ties = s.cut.ties;
      return s.cut.x;
    }
    float* own = reinterpret_cast<float*>(&k.parts);
    in_bins(held, first.bin, last.bin,
            [&](float x) { own[atomicAdd(&s.own, 1u)] = x; });
    __syncthreads();
    if (threadIdx.x == 0)
      s.base = atomicAdd(cluster.map_shared_rank(&s.gathered, 0), s.own);
    __syncthreads();
    float* given = cluster.map_shared_rank(table.given, 0) + s.base;
    for (int i = threadIdx.x; i < s.own; i += kDrawThreads) given[i] = own[i];
    sync();
    if (rank == 0) cut_given(number, by_mass, target, by_mass ? front.mass : front.count);
    if (threadIdx.x == 0) s.own = s.gathered = 0;
    sync();
    ties = s.cut.ties;
    return s.cut.x;
  }
  // The same of the words in table.given, by this CTA for all, into s.cut; before: the
  // mass (or count) in front of them.  Few of them: each compared with each, by a few
  // threads.
  __device__ __forceinline__ void pair_given(int number, bool by_mass, uint64_t target,
                                             uint64_t before) {
    int lanes = 32;                     // of a word
    while (lanes > 1 && number * lanes > kDrawThreads) lanes /= 2;
    if (by_mass) {
      for (int i = threadIdx.x; i < number; i += kDrawThreads)
        k.few.mass[i] = mass(table.given[i]);
      __syncthreads();
    }
    const int i = threadIdx.x / lanes, part = threadIdx.x & (lanes - 1);
    const bool has = i < number;
    const float x = has ? table.given[i] : INFINITY;
    uint64_t at = 0;
    uint32_t equal = 0;
    for (int j = part; j < number; j += lanes) {
      const float o = table.given[j];
      equal += o == x;
      if (o > x) at += by_mass ? k.few.mass[j] : 1;
    }
    for (int o = lanes / 2; o; o /= 2) {
      equal += __shfl_xor_sync(0xffffffffu, equal, o);
      at += __shfl_xor_sync(0xffffffffu, at, o);
    }
    at += before;
    const uint64_t own = !has ? 0 : by_mass ? k.few.mass[i] : 1;
    if (has && part == 0 && at < target && target <= at + equal * own) {
      // (several threads where values are equal, with one result)
      const uint32_t up_to = (uint32_t)((target - at + own - 1) / own);
      for (int q = 0; q < ctas; ++q)
        *cluster.map_shared_rank(&s.cut, q) = {x, up_to};
    }
  }
  // More of them: parts of their range, until one value is left.
  __device__ __forceinline__ void cut_given(int number, bool by_mass, uint64_t target,
                                            uint64_t before) {
    constexpr int kEach = kGather / kDrawThreads, kOwn = kParts / kDrawThreads;
    uint32_t key[kEach], lo = 0xffffffffu, hi = 0;
    uint64_t p[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int at = threadIdx.x + i * kDrawThreads;
      const float x = at < number ? table.given[at] : 0.f;
      key[i] = at < number ? key_of(x) : 0;             // (0: of no number)
      p[i] = by_mass && at < number ? mass(x) : 1;
      if (at < number) {
        lo = min(lo, key[i]);
        hi = max(hi, key[i]);
      }
    }
    cta_extent(hi, lo);
#pragma unroll 1
    while (lo < hi) {
      const int shift = max(0, 32 - __clz(hi - lo) - 10);
#pragma unroll
      for (int i = 0; i < kOwn; ++i)
        k.parts.lo[threadIdx.x * kOwn + i] = k.parts.hi[threadIdx.x * kOwn + i] = 0;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kEach; ++i)
        if (key[i] >= lo && key[i] <= hi) add_to_part((hi - key[i]) >> shift, p[i]);
      __syncthreads();
      Pair own = {0, 0}, all;
      uint64_t of[kOwn];
#pragma unroll
      for (int i = 0; i < kOwn; ++i) {
        const int at = threadIdx.x * kOwn + i;
        of[i] = k.parts.lo[at] + ((uint64_t)k.parts.hi[at] << 32);
        own.mass += of[i];
      }
      uint64_t at = before + scan(own, all).mass;
#pragma unroll
      for (int i = 0; i < kOwn; ++i) {
        if (at < target && target <= at + of[i])
          s.found[0] = {(uint32_t)(threadIdx.x * kOwn + i), 0, 0, at};
        at += of[i];
      }
      __syncthreads();
      const uint32_t part = s.found[0].bin;
      before = s.found[0].mass;
      uint32_t lo2 = 0xffffffffu, hi2 = 0;
#pragma unroll
      for (int i = 0; i < kEach; ++i)
        if (key[i] >= lo && key[i] <= hi && (hi - key[i]) >> shift == part) {
          lo2 = min(lo2, key[i]);
          hi2 = max(hi2, key[i]);
        }
      cta_extent(hi2, lo2);
      lo = lo2;
      hi = hi2;
    }
    const float x = of_key(lo);
    if (threadIdx.x < ctas)
      *cluster.map_shared_rank(&s.cut, threadIdx.x) = {
          x, by_mass ? ties_of(x, target - before) : (uint32_t)(target - before)};
  }
  // How many of one value have their words in front below `left`.
  __device__ __forceinline__ uint32_t ties_of(float x, uint64_t left) const {
    const uint64_t p = mass(x);
    return (uint32_t)((left + p - 1) / p);
  }
  // What is kept: the words above `above` and the first `ties` of value `tie`.  The
  // masses of those with bins below `summed` are in s.base_mass, for each warp of the
  // CTA.
  struct Kept {
    float above, tie;
    uint32_t ties;
    float summed;
  };

  // Writes the word drawn: x of index `at`, of a mass z in all.  Both terms of the
  // logarithm have one sign, so that fp32 keeps their digits: within 2^-22 of it.
  __device__ __forceinline__ void write(int64_t row, int64_t at, float x, uint64_t z) {
    a.ids[row] = at;
    if (!a.logprob) return;
    float log_p = 0.f;
    if (x != m) {
      const float d = m - x, b = d - m, y = d * rate.hi;
      const float d_lo = (m - (d - b)) - (x + b);
      log_p = -0.69314718055994531f *
              (y + fmaf(d_lo, rate.hi, fmaf(d, rate.lo, fmaf(d, rate.hi, -y))));
    }
    const float rest = (float)(z - one()) * __int_as_float((127 - a.bits) << 23);
    a.logprob[row] = log_p - log1pf(rest);
  }

  __device__ __forceinline__ void run(int64_t row);
  __device__ __forceinline__ void find_kept_tabled(Kept& kept);
  __device__ __forceinline__ bool find_kept(int64_t row, Kept& kept);
  __device__ __forceinline__ void first_largest(int64_t row);
  __device__ __forceinline__ void choose_listed(int64_t row, uint64_t whole);
  __device__ __forceinline__ void choose(int64_t row, Kept kept);
  // What the row's random number is of z.
  __device__ __forceinline__ uint64_t target_of(uint64_t z) const {
    const float u = s.set.uniform;
    return u >= 1.f ? z - 1 : min(times(ratio_of(u), z, false), z - 1);
  }
};

template <class T, bool kStaged>
__device__ __forceinline__ void Draw<T, kStaged>::first_largest(int64_t row) {
  uint32_t at = 0xffffffffu, none = 0;
  each([&](float x, uint32_t i) {
    if (x == m) at = min(at, i);
  });
  row_extent(none, at);
  if (rank == 0 && threadIdx.x == 0) {
    a.ids[row] = at;
    if (a.logprob) a.logprob[row] = 0.f;
  }
}

// Draws from the s.listed words of k.few, which are all that may be kept, in the first
// CTA; `whole`: the mass that top_p is of, 0: of the first top_k.  A few threads have a
// word and go over all of them twice: for what is in front of it in the order, and in
// front of it by index.
template <class T, bool kStaged>
__device__ __forceinline__ void Draw<T, kStaged>::choose_listed(int64_t row,
                                                                uint64_t whole) {
  const int number = s.listed;
  Few& f = k.few;
  for (int i = threadIdx.x; i < number; i += kDrawThreads)
    f.mass[i] = mass(of_key((uint32_t)(f.word[i] >> 32)));
  __syncthreads();
  int lanes = 32;                       // of a word
  while (lanes > 1 && number * lanes > kDrawThreads) lanes /= 2;
  const int i = threadIdx.x / lanes, part = threadIdx.x & (lanes - 1);
  const bool has = i < number;
  const uint64_t word = has ? f.word[i] : 0;
  uint64_t before = 0;
  uint32_t place = 0;
  for (int j = part; j < number; j += lanes)
    if (f.word[j] > word) {
      ++place;
      before += f.mass[j];
    }
  for (int o = lanes / 2; o; o /= 2) {
    place += __shfl_xor_sync(0xffffffffu, place, o);
    before += __shfl_xor_sync(0xffffffffu, before, o);
  }
  const uint64_t own = has ? f.mass[i] : 0;
  const int limit = s.set.top_k ? min(number, (int)s.set.top_k) : number;
  if (!whole) {
    if (has && part == 0 && place == limit - 1) s.number = before + own;
    __syncthreads();
    whole = s.number;
  }
  bool kept = has && place < limit;
  if (place) {
    kept &= own >= s.set.least;
    if (s.set.by_mass) kept &= before < times(s.set.top_p, whole, true);
  }
  if (has && part == 0) f.kept[i] = kept ? own : 0;
  __syncthreads();
  // up to and with the word, by index, and of all
  uint64_t to = 0, z = 0;
  for (int j = part; j < number; j += lanes) {
    z += f.kept[j];
    if ((uint32_t)f.word[j] >= (uint32_t)word) to += f.kept[j];
  }
  for (int o = lanes / 2; o; o /= 2) {
    to += __shfl_xor_sync(0xffffffffu, to, o);
    z += __shfl_xor_sync(0xffffffffu, z, o);
  }
  const uint64_t target = target_of(z);
  if (kept && part == 0 && target < to && target >= to - own)
    write(row, (uint32_t)~word, of_key((uint32_t)(word >> 32)), z);
}

// Draws from the words that are kept (of those, the ones of a mass s.set.least).
template <class T, bool kStaged>
__device__ __forceinline__ void Draw<T, kStaged>::choose(int64_t row, Kept kept) {
  const float above = kept.above, tie = kept.tie, summed = kept.summed;
  uint32_t ties = kept.ties;
  const uint64_t tie_mass = ties ? mass(tie) : 0;
  if (tie_mass < s.set.least) ties = 0;
  const auto kept_mass = [&](float x) -> uint64_t {
    if (!(x > above)) return 0;
    const uint64_t p = mass(x);
    return p >= s.set.least ? p : 0;
  };
  // the CTA's columns, then the part of them that has the target, are cut into one for
  // each warp, until every thread has 16 bytes
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int first = 0, end = c.units;
  uint64_t z = 0, before = 0, target = 0;
  uint32_t tied_before = 0;
  for (bool whole = true; whole || end - first > kDrawThreads; whole = false) {
    const int each_warp = warp_units(end - first);
    const int u0 = first + warp * each_warp, u1 = min(u0 + each_warp, end);
    uint64_t sum = 0;
    uint32_t tied = 0;
    const float begin = whole ? summed : 0.f;
    if (above == -INFINITY && !s.set.least) {
      walk(u0 + lane, u1, 32, [&](int, const uint4& v) {
        uint64_t p[n];
        masses(v, p);
#pragma unroll
        for (int j = 0; j < n; ++j) sum += p[j];
      });
    } else if (sizeof(T) == 2 && tabled) {
      walk(u0 + lane, u1, 32, [&](int, const uint4& v) {
        float x[n];
        uint64_t p[n];
        Vec<T>::get(v, x);
        masses(v, p);
#pragma unroll
        for (int j = 0; j < n; ++j) {
          if (ties && x[j] == tie) ++tied;
          if (x[j] > above && p[j] >= s.set.least) sum += p[j];
        }
      });
    } else {
      walk(u0 + lane, u1, 32, [&](int, const uint4& v) {
        float x[n];
        Vec<T>::get(v, x);
#pragma unroll
        for (int j = 0; j < n; ++j) {
          if (ties && x[j] == tie) ++tied;
          if (x[j] > above && !(bin_place(x[j], place(x[j])) < begin))
            sum += kept_mass(x[j]);
        }
      });
    }
    if (whole && summed > 0.f && lane == 0) sum += s.base_mass[warp];
    __syncthreads();
    const Pair cta = cta_sum(tied, sum);
    if (whole) {
      // Z, and what is in front of the CTA
      const int t = tell(cta);
      for (uint32_t q = 0, seen = 0; q < ctas; ++q) {
        const Pair o = s.slot[t][q];
        if (q == rank) {
          before = z;
          tied_before = seen;
        }
        z += o.mass + tie_mass * min(o.count, ties - min(ties, seen));
        seen += o.count;
      }
      target = target_of(z);
      if (target < before) return;
    }
    // each warp's own, the ties that are kept among it, and the one that has the target
    Pair own = {0, 0};
    if (lane < kDrawWarps) own = {s.warp_count[lane], s.warp_mass[lane]};
    if (ties) {
      const uint32_t seen = tied_before + lanes_scan(own).count - own.count;
      own.mass += tie_mass * min(own.count, ties - min(ties, seen));
    }
    const Pair to = lanes_scan(own);
    const uint32_t has = __ballot_sync(
        0xffffffffu, lane < kDrawWarps && target < before + to.mass);
    if (!has) return;
    const int owner = __ffs(has) - 1;
    const Pair front = of_lane({to.count - own.count, to.mass - own.mass}, owner);
    before += front.mass;
    tied_before += front.count;
    end = min(first + (owner + 1) * each_warp, end);
    first += owner * each_warp;
  }
  uint4 v = Vec<T>::none();
  if (first + threadIdx.x < end) v = c.raw(first + threadIdx.x);
  float x[n];
  uint64_t p[n], sum = 0;
  Vec<T>::get(v, x);
  masses(v, p);
  uint32_t left = 0;
  Pair all;
  if (ties) {
    uint32_t tied = 0;
#pragma unroll
    for (int j = 0; j < n; ++j) tied += x[j] == tie;
    left = tied_before + scan({tied, 0}, all).count;
    left = ties - min(ties, left);
  }
#pragma unroll
  for (int j = 0; j < n; ++j) {
    const bool is_tie = left && x[j] == tie;
    if (!is_tie && !(x[j] > above && p[j] >= s.set.least)) p[j] = 0;
    left -= is_tie;
    sum += p[j];
  }
  uint64_t at = before + scan({0, sum}, all).mass;
  if (target < at || target >= at + sum) return;
#pragma unroll
  for (int j = 0; j < n; ++j) {
    if (target >= at && target < at + p[j])
      write(row, (int64_t)rank * a.columns + (first + threadIdx.x) * n - c.shift + j,
            x[j], z);
    at += p[j];
  }
}

// Of a row whose bins are values.
template <class T, bool kStaged>
__device__ __forceinline__ void Draw<T, kStaged>::find_kept_tabled(Kept& kept) {
  for (int i = threadIdx.x; i < kBins; i += kDrawThreads)
    table.mass[i] = i <= values.last && i != values.gap_number
                        ? mass(values.value(i)) : 0;
  __syncthreads();
  const bool by_mass = s.set.by_mass;
  const uint32_t top_k = s.set.top_k;
  if (!top_k && !by_mass) return;
  uint64_t sum = 0;
  walk(threadIdx.x, c.units, kDrawThreads, [&](int, const uint4& raw) {
    const uint4 v = Vec<T>::raise(raw, lower);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t two = values.numbers(w[i]);
      atomicAdd(&k.bins[two & 0xffffu], 1u);
      atomicAdd(&k.bins[two >> 16], 1u);
    }
    if (by_mass && Vec<T>::has_tiny(raw, values.gap)) {
      float x[n];
      Vec<T>::get(raw, x);
#pragma unroll 1
      for (int j = 0; j < n; ++j)
        if (fabsf(x[j]) < values.gap) sum += mass(x[j]);
    }
  });
  gap_mass = by_mass ? row_sum(sum) : 0;
  const Range r = gather_bins();
  uint64_t whole = r.total.mass;
  // (columns beside the row count as words without a mass)
#pragma unroll 1
  for (int by = top_k && top_k < r.total.count ? 0 : 1; by <= by_mass; ++by) {
    const uint64_t target = by ? times(s.set.top_p, whole, true) : top_k;
    __syncthreads();
    find_bin(r, by, by, target);
    __syncthreads();
    const Found f = s.found[by];
    Pair before = {f.before, f.mass};
    if (f.bin != values.gap_number) {
      kept.tie = values.value(f.bin);
    } else {
      const float end = __uint_as_float(__float_as_uint(values.gap) - 1);
      if (!by && values.gap_number == values.last) {
        // (the words below `lower` were counted in the gap: they have no mass, and with
        // some of them among the first top_k all that have one are)
        sum = 0;
        each([&](float x, uint32_t) { sum += fabsf(x) < values.gap; });
        if (before.count + row_sum(sum) < top_k) continue;
      }
      kept.tie = cut(key_of(-end), key_of(end), by, target, before);
      if (!by && by_mass) {
        // (counting left no masses)
        sum = 0;
        each([&](float x, uint32_t) {
          if (x > kept.tie && fabsf(x) < values.gap) sum += mass(x);
        });
        before.mass = f.mass + row_sum(sum);
      }
    }
    kept.above = kept.tie;
    kept.ties = by ? ties_of(kept.tie, target - before.mass) : top_k - before.count;
    if (!by) whole = before.mass + kept.ties * mass(kept.tie);
  }
}

// False where the word is drawn already.
template <class T, bool kStaged>
__device__ __forceinline__ bool Draw<T, kStaged>::find_kept(int64_t row, Kept& kept) {
  const bool by_mass = s.set.by_mass;
  uint32_t top_k = s.set.top_k;
  if (!top_k && !by_mass) return true;
  each([&](float x, uint32_t) {
    const float y = place(x);
    if (counts(x, y)) atomicAdd(&k.bins[bin_at(x, y)], 1u);
  });
  const Range r = gather_bins();
  if (top_k >= r.total.count) top_k = 0;
  // the bins of the k-th word; without one, those in which top_p of the mass is
  // passed: masses by bins are within 0.76%, so of twice the ratio
  if (top_k) {
    find_bin(r, 0, false, top_k);
  } else if (by_mass) {
    const uint64_t about = times(s.set.top_p, r.total.mass, true);
    find_bin(r, 1, true, max((uint64_t)1, about - about / 62));
    find_bin(r, 2, true,
             max((uint64_t)1, min(about + about / 62, r.total.mass)));
  }
  if (!top_k && !by_mass) return true;
  __syncthreads();
  const Found from = s.found[top_k ? 0 : 1], to = s.found[top_k ? 0 : 2];
  const bool few = to.through <= kFew;
  // one look at all words: their mass, if top_p is of all; that of those in front of the
  // bins, for each warp; and a list of those that may be kept, or of those in the bins
  // (some CTA may have more of them than it can hold)
  bool held = !top_k && to.through - from.before <= kHeld * ctas;
  uint64_t whole = 0;
  Pair in_front = {from.before, 0};
  if (few || !top_k) {
    const float begin = (float)from.bin;
    const float end = to.bin == kBins - 1 ? INFINITY : (float)(to.bin + 1);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int each_warp = warp_units(c.units);
    const int u1 = min((warp + 1) * each_warp, c.units);
    const uint64_t least = s.set.least;
    uint64_t sum = 0, front = 0, front_kept = 0;
    walk(warp * each_warp + lane, u1, 32, [&](int u, const uint4& v) {
      float x[n];
      uint64_t p[n];
      Vec<T>::get(v, x);
      if (!top_k) {
        masses(v, p);
#pragma unroll
        for (int j = 0; j < n; ++j) sum += p[j];
      }
      uint32_t to_hold = 0;
#pragma unroll
      for (int j = 0; j < n; ++j) {
        const float y = place(x[j]), b = bin_place(x[j], y);
        if (!few) {
          const uint64_t q = b < begin ? p[j] : 0;
          front += q;
          if (least) front_kept += q >= least ? q : 0;
        }
        if (b < end && (few || (held && b >= begin)) && counts(x[j], y)) {
          if (few) list(x[j], (uint32_t)(rank * a.columns + u * n - c.shift + j));
          else to_hold |= 1u << j;
        }
      }
      if (to_hold) {
        uint32_t at = atomicAdd(&s.listed, (uint32_t)__popc(to_hold));
#pragma unroll
        for (int j = 0; j < n; ++j)
          if (to_hold >> j & 1) {
            if (at < kHeld) k.held[at] = x[j];
            ++at;
          }
      }
    });
    if (!few) {
      front = warp_sum(front);
      front_kept = least ? warp_sum(front_kept) : front;
      if (lane == 0) {
        s.scan_mass[warp] = front;
        s.base_mass[warp] = front_kept;
      }
    }
    Pair cta = cta_sum(0, sum);
    if (!few && warp == 0) {
      front = warp_sum(lane < kDrawWarps ? s.scan_mass[lane] : 0);
      if (lane < ctas)
        *cluster.map_shared_rank(&s.slot_front[rank], lane) = front;
      cta.count = s.listed > kHeld;
    }
    const int t = tell(cta);
    for (int q = 0; q < ctas; ++q) {
      whole += s.slot[t][q].mass;
      held &= !s.slot[t][q].count;
    }
    if (few) {
      if (rank == 0) choose_listed(row, whole);
      return false;
    }
    for (int q = 0; q < ctas; ++q) in_front.mass += s.slot_front[q];
  }
  Found first = from, last = to;
#pragma unroll 1
  for (int by = top_k ? 0 : 1; by <= by_mass; ++by) {
    uint64_t target = top_k;
    if (by && top_k) {
      // top_p of the first top_k, of all bins
      uint64_t sum = 0;
      each([&](float x, uint32_t) { sum += x > kept.tie ? mass(x) : 0; });
      whole = row_sum(sum) + kept.ties * mass(kept.tie);
      first = {0, 0, 0, 0};             // (up to the k-th word's)
      in_front = {0, 0};
    }
    if (by) target = times(s.set.top_p, whole, true);
    kept.tie = cut_bins(r, first, last, held && by, by, target, in_front, kept.ties);
  }
  kept.above = kept.tie;
  kept.summed = top_k ? 0.f : (float)from.bin;
  return true;
}

template <class T, bool kStaged>
__device__ __forceinline__ void Draw<T, kStaged>::run(int64_t row) {
  // (waited for in front of the first tell(): what a CTA stores into another's shared memory comes
  // after that one has started)
  if (ctas > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
  // (on their way while the row's are)
  float uniform = 0.f, row_temperature = 0.f, row_top_p = 0.f, row_min_p = 0.f;
  int32_t row_top_k = 0;
  if (threadIdx.x == 0) {
    uniform = a.uniform[row];
    if (a.d_temperature) row_temperature = a.d_temperature[row];
    if (a.d_top_p) row_top_p = a.d_top_p[row];
    if (a.d_min_p) row_min_p = a.d_min_p[row];
    if (a.d_top_k) row_top_k = a.d_top_k[row];
  }
  const uint64_t power = threadIdx.x < kExpTable ? kPowers[threadIdx.x] : 0;
  if (a.cuts)
    for (int i = threadIdx.x; i < kBins; i += kDrawThreads) k.bins[i] = 0;
  const int64_t col0 = (int64_t)rank * a.columns;
  c.len = (int)max((int64_t)0, min((int64_t)a.columns, a.vocab - col0));
  c.row = static_cast<const T*>(a.logits) + row * a.stride + (c.len ? col0 : 0);
  c.shift = (int)(((uintptr_t)c.row & 15) / sizeof(T));
  c.units = c.len ? (c.shift + c.len + n - 1) / n : 0;
  float largest = -INFINITY;
  constexpr int kAhead = 4;             // loads of a thread in flight
  for (int u0 = threadIdx.x; u0 < c.units; u0 += kAhead * kDrawThreads) {
    uint4 v[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (c.whole(u0 + i * kDrawThreads)) v[i] = c.load(u0 + i * kDrawThreads);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int u = u0 + i * kDrawThreads;
      if (u >= c.units) break;
      if (!c.whole(u)) v[i] = c.from_memory(u);
      if (kStaged) c.kept[u] = v[i];
      largest = fmaxf(largest, Vec<T>::largest(v[i]));
    }
  }
  if (threadIdx.x == 0) {
    Settings& t = s.set;
    t.rate = a.rate;
    t.greedy = a.greedy;
    if (a.d_temperature) {
      // log2(e) as an fp32 pair over an fp32 number
      constexpr float hi = 1.44269502f, lo = 1.92596299e-8f;
      const float temperature = fminf(row_temperature, 3e38f);
      t.greedy |= !(row_temperature > 0.f);
      t.rate.hi = hi / temperature;
      t.rate.lo = (fmaf(-t.rate.hi, temperature, hi) + lo) / temperature;
    }
    t.top_p = a.top_p;
    t.by_mass = a.by_mass;
    if (a.d_top_p) {
      t.greedy |= !(row_top_p > 0.f);
      t.by_mass = row_top_p < 1.f;
      t.top_p = ratio_of(row_top_p);
    }
    Ratio min_p = a.min_p;
    if (a.d_min_p) {
      t.greedy |= !(row_min_p <= 1.f);
      min_p = ratio_of(row_min_p);
    }
    t.least = times(min_p, one(), true);
    const int64_t top_k = a.d_top_k ? (int64_t)row_top_k : a.top_k;
    t.top_k = top_k > 0 && top_k < a.vocab ? (uint32_t)top_k : 0;
    t.greedy |= t.top_k == 1;
    t.uniform = uniform;
    s.listed = s.own = s.gathered = 0;
  }
  if (threadIdx.x < kExpTable) {
    s.table_hi[threadIdx.x] = (uint32_t)(power >> 32);
    s.table_lo[threadIdx.x] = (uint32_t)power;
    s.table_one[threadIdx.x] =
        (uint32_t)((power + (1u << 30)) >> 31);
  }
  if (ctas > 1) {
    __syncwarp();
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  }
  uint32_t most = key_of(largest), none = 0;
  row_extent(most, none);
  m = of_key(most);
  rate = s.set.rate;
  scale = (float)kBins / (float)a.bits;
  // (numbers of 8 bits, of which none is 2^-14 of the distance or smaller, but 0)
  tiny = (float)a.bits / rate.hi * 0x1p-14f;
  if (m != 0.f && fabsf(m) < tiny) tiny = INFINITY;
  // (towards -inf in T)
  const uint32_t below = __float_as_uint(m - 50.f / rate.hi);
  lower = __uint_as_float(sizeof(T) == 4 ? below
                                         : (below + (below >> 31) * 0xffffu) &
                                               0xffff0000u);
  const float far = (m - lower) * rate.hi;
  if (!(lower > -1e38f && m < 1e38f && far > 46.f && far < 63.f)) lower = m;
  if (m == -INFINITY) {
    if (rank == 0 && threadIdx.x == 0) {
      a.ids[row] = -1;
      if (a.logprob) a.logprob[row] = -INFINITY;
    }
    return;
  }
  if (s.set.greedy) {
    first_largest(row);
    return;
  }
  tabled = sizeof(T) == 2 && lower < m;
  if (tabled) values.set(m, lower);
  Kept kept = {-INFINITY, 0.f, 0, 0.f};
  if (sizeof(T) == 2 && tabled) find_kept_tabled(kept);
  else if (!find_kept(row, kept)) return;
  choose(row, kept);
}

template <class T, bool kStaged>
__global__ void __launch_bounds__(kDrawThreads, 2) draw_kernel(const DrawArgs a) {
  __shared__ DrawShared shared;
  extern __shared__ uint4 dynamic[];
  const int table = table_bytes(sizeof(T), a.cuts) / 16;
  Draw<T, kStaged> d(a, shared, *reinterpret_cast<DrawTable*>(dynamic),
                     *reinterpret_cast<DrawCuts*>(dynamic + table));
  d.c.kept = dynamic + table + (a.cuts ? sizeof(DrawCuts) / 16 : 0);
  d.run(blockIdx.x / d.ctas);
}

Ratio ratio_of(double x) {
  int e;
  const double f = frexp(x, &e);
  return {(uint64_t)ldexp(f, 53), 53 - e};
}

}  // namespace

cudaError_t lm_sample_setup() {
  cudaError_t e = cudaFuncSetAttribute(
      draw_kernel<float, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kRoom);
  if (e == cudaSuccess)
    e = cudaFuncSetAttribute(draw_kernel<__nv_bfloat16, true>,
                             cudaFuncAttributeMaxDynamicSharedMemorySize, kRoom);
  return e;
}

}  // namespace lamb

using namespace lamb;

extern "C" lamb_status_t lamb_vocab_sample(
    struct lamb_vocab* v, const void* logits, int32_t dtype, int64_t stride,
    int64_t n_rows, const float* uniform, double temperature,
    const float* d_temperature, int64_t top_k, const int32_t* d_top_k, double top_p,
    const float* d_top_p, double min_p, const float* d_min_p, int64_t* ids,
    float* logprob, cudaStream_t stream) {
  if (!v) return lm_fail(LAMB_ERR_INVALID_ARG, "plan is NULL");
  if (dtype != LAMB_F32 && dtype != LAMB_BF16)
    return lm_fail(LAMB_ERR_UNSUPPORTED_DTYPE, "logits: dtype %d unsupported",
                   dtype);
  if (n_rows < 0 || n_rows > v->max_tokens)
    return lm_fail(LAMB_ERR_INVALID_ARG, "n_rows %lld is not in [0, %lld]",
                   (long long)n_rows, (long long)v->max_tokens);
  if (!d_temperature && !(temperature >= 0. && temperature < INFINITY))
    return lm_fail(LAMB_ERR_INVALID_ARG, "temperature is not in [0, inf)");
  if (!d_top_k && top_k < 0)
    return lm_fail(LAMB_ERR_INVALID_ARG, "top_k is below 0");
  if (!d_top_p && !(top_p >= 0. && top_p <= 1.))
    return lm_fail(LAMB_ERR_INVALID_ARG, "top_p is not in [0, 1]");
  if (!d_min_p && !(min_p >= 0. && min_p <= 1.))
    return lm_fail(LAMB_ERR_INVALID_ARG, "min_p is not in [0, 1]");
  if (v->vocab > (1 << 24))
    return lm_fail(LAMB_ERR_INVALID_ARG, "vocab is above 2^24");
  if (!n_rows) return LAMB_OK;
  if (!logits || !uniform || !ids)
    return lm_fail(LAMB_ERR_INVALID_ARG, "logits, uniform and ids are required");
  if (stride < v->vocab)
    return lm_fail(LAMB_ERR_INVALID_ARG, "logits: row stride below the vocabulary");
  if ((uintptr_t)logits % lm_elem_size(dtype) || (uintptr_t)uniform % 4 ||
      (uintptr_t)ids % 8 || (uintptr_t)logprob % 4 ||
      (uintptr_t)d_temperature % 4 || (uintptr_t)d_top_k % 4 ||
      (uintptr_t)d_top_p % 4 || (uintptr_t)d_min_p % 4)
    return lm_fail(LAMB_ERR_INVALID_ARG, "a pointer is not aligned");
  LmDevice dev(v->device);
  if (dev.err != cudaSuccess) return lm_cuda_fail(dev.err, "cudaSetDevice");
  DrawArgs a = {};
  a.logits = logits;
  a.stride = stride;
  a.rows = n_rows;
  a.vocab = (int)v->vocab;
  // masses of a vocabulary add up below 2^63
  a.bits = 44;
  while (v->vocab >> (63 - a.bits)) --a.bits;
  a.uniform = uniform;
  if (!d_temperature && temperature > 0.) a.rate = exp_rate(temperature);
  a.top_k = top_k;
  if (!d_top_p) a.top_p = ratio_of(top_p);
  if (!d_min_p) a.min_p = ratio_of(min_p);
  a.greedy = (!d_temperature && temperature == 0.) || (!d_top_p && top_p == 0.);
  a.by_mass = !d_top_p && top_p < 1.;
  a.d_temperature = d_temperature;
  a.d_top_k = d_top_k;
  a.d_top_p = d_top_p;
  a.d_min_p = d_min_p;
  a.ids = ids;
  a.logprob = logprob;
  a.cuts = d_top_k || d_top_p || (top_k > 0 && top_k < v->vocab) ||
           a.by_mass;
  const int bins = (a.cuts ? sizeof(DrawCuts) : 0) +
                   table_bytes(lm_elem_size(dtype), a.cuts);
  // CTAs of a row: while two of all of them fit on each SM, and until two of one row
  // do; of 4,096 columns at least.  (Before the table, 1,024 rows of 30,522 by one CTA 81 us, by two 101;
  // 64 by two 43, four 41, eight 46; 128 rows of 131,071 in bf16 by two, which are alone
  // on their SMs, 209, by four 146, eight 194.)
  const int size = lm_elem_size(dtype);
  int ctas = 1;
  while (ctas < kMostCtas && v->vocab / ctas > 4096 &&
         (n_rows * ctas * 2 <= 2 * v->sms ||
          bins + v->vocab / ctas * size + 64 > kHalf))
    ctas *= 2;
  a.columns = (int)lm_round_up(lm_ceil_div(v->vocab, ctas), 8);
  const int64_t whole = bins + (int64_t)a.columns * size + 32;
  const bool staged = whole <= kRoom;
  const size_t smem = staged ? whole : bins;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(n_rows * ctas));
  cfg.blockDim = dim3(kDrawThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = ctas;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  typedef __nv_bfloat16 bf;
  const cudaError_t e = cudaLaunchKernelEx(
      &cfg,
      dtype == LAMB_F32 ? (staged ? draw_kernel<float, true>
                                  : draw_kernel<float, false>)
                        : (staged ? draw_kernel<bf, true> : draw_kernel<bf, false>),
      a);
  return e == cudaSuccess ? LAMB_OK : lm_cuda_fail(e, "sampling launch");
}
