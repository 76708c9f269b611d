// The Muon plan's device tables, and the launch of its product steps.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stddef.h>

#include "lm_host.h"

namespace lamb {

constexpr float kScaleD = 1024.f;            // D is stored times this
constexpr float kScaleE = 256.f;             // and E times this
constexpr float kScaleLo = 2048.f;           // lo: the rest of hi, times this

constexpr int kMuonMaps = 13;

struct MuonMatrix {               // the maps first
  // the products' operands, 128 rows by 64 of K in one copy: K-major (_k),
  // MN-major (_mn); hi has two buffers, taken in turn
  CUtensorMap x_k[2], x_mn[2], d, e;
  // the epilogues' blocks: 128 rows of 32 columns (64-byte swizzle), and
  // mirrored ones of 32 rows by 64 columns
  CUtensorMap x_c[2], lo_c, d_c, e_c, d_t, e_t;
  __half* hi[2];
  __half* lo;
  __half* D;
  __half* E;
  float* diag;                   // l
  float* beta;
  float scale;                   // hi + lo = X scale
  int rows, cols, m, n;          // m = min, n = max
  int tall;                      // rows > cols
  int pitch, pitch_m;            // of X, of D and E
  int first_chunk, n_chunks;
  int sym, app;                  // CTAs' tiles of a Gram matrix, of X
  float decay;
};

static_assert(offsetof(MuonMatrix, hi) == kMuonMaps * sizeof(CUtensorMap),
              "kMuonMaps");

struct MuonPtrs {
  float* w;
  const void* g;                 // or the direction's input
  float* m;
  __nv_bfloat16* out;            // copy of w, or the direction
};

struct MuonChunk {
  int matrix;
  int len;
  int64_t offset;
};

enum { kGram = 0, kSquare = 1, kApply = 2, kNoTile = 3 };

// A tile of one product of one matrix, two CTAs' work, with what they need of the
// matrix: one load when the tile is taken.
struct __align__(16) MuonTile {
  int matrix, i, j, phase;
  int height, width;     // of the product
  int kn;                // blocks of K
  int tall;
  int sym, app;          // the matrix'
  float scale, decay;
  const MuonMatrix* x;
  float *diag, *beta;
  int rows, cols;
};
struct MuonConsts {
  float a, b, c;
  float beta, omb;               // momentum
  float eps;
  float wd, size;                // lambda, s without its shape's part
  int nesterov, scale_kind;
};

struct MuonParams {
  const MuonMatrix* mats;
  const MuonPtrs* ptrs;
  const MuonTile* tiles;         // of one step
  uint32_t* done;                // CTAs' tiles of each matrix finished
  const float* d_lr;             // NULL: the direction alone
  uint32_t* status;
  MuonConsts k;
  int n_mats, steps;
  int step_tiles, total;         // tiles of one step, of all
};

// s of a matrix.
__device__ __forceinline__ float muon_size(const MuonConsts& k, int rows,
                                           int cols) {
  if (k.scale_kind == LAMB_MUON_SCALE_RMS)
    return k.size * 0.2f * sqrtf((float)(rows > cols ? rows : cols));
  if (k.scale_kind == LAMB_MUON_SCALE_SPECTRAL)
    return k.size * sqrtf(fmaxf(1.f, (float)rows / (float)cols));
  return k.size;
}
__device__ __forceinline__ uint32_t pack_half2(float x, float y) {
  const __half2 h = __floats2half2_rn(x, y);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float2 half2_at(uint32_t w) {
  return __half22float2(*reinterpret_cast<const __half2*>(&w));
}
__device__ __forceinline__ uint16_t half_bits(uint32_t w, int i) {
  return (uint16_t)(i ? w >> 16 : w & 0xffffu);
}

constexpr int kMuonRows = 128;        // rows of a tile that a CTA has
constexpr int kMuonCols = 32;                       // columns of a block

// lm_muon_steps.cu: tiles of 128 x 128 by single CTAs, or of 256 x 256 by pairs.
// Setup: how many of either the current device holds at a time.
cudaError_t muon_steps_setup(int sms, int* ctas, int* pairs);
cudaError_t muon_launch_steps(const MuonParams& p, bool pair, int units,
                              cudaStream_t stream);

}  // namespace lamb
