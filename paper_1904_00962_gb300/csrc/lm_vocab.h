// The vocabulary plan: workspaces of the word table's lookup, its gradient and
// the head's loss (lm_embed.cu, lm_head.cu).
#pragma once
#include <cuda_bf16.h>

#include "lm_host.h"

struct lamb_vocab {
  int device = 0, sms = 0;
  int64_t vocab = 0, max_tokens = 0;
  int width = 0;
  lamb::EncodeTiled encode = nullptr;
  void* arena = nullptr;
  uint32_t* status = nullptr;

  // lookup gradient: sort buffers, and the sums that chunks leave
  int sort_passes = 0;          // of 8 bits each
  uint32_t* keys[2] = {nullptr, nullptr};
  int32_t* pos[2] = {nullptr, nullptr};
  int32_t* hist = nullptr;      // [pass][tile][256]
  float* part = nullptr;        // [chunks][2][width]

  // head: the rows that have a label, and what is known of each
  __nv_bfloat16* rows = nullptr;
  int32_t* row_label = nullptr;
  int32_t* row_token = nullptr;
  int32_t* n_rows = nullptr;
  int32_t* counts = nullptr;    // labels in runs of tokens
  float2* stats = nullptr;      // [vocab tiles][max_tokens]
  float* label_logit = nullptr;
  float4* row_lse = nullptr;
  double* block_sums = nullptr;
  uint32_t* ticket = nullptr;
  float* coef = nullptr;        // scale / number of labels
  __nv_bfloat16* dlogits = nullptr;
  int64_t dlogits_elems = 0;
  float* slabs = nullptr;       // grad_hidden's partial sums
  __nv_bfloat16* weight_copy = nullptr;   // W on 16-byte boundaries
};

namespace lamb {
// Sizes the head's and the lookup gradient's workspaces (base NULL: counts).
void lm_head_carve(lamb_vocab* v, LmArena* a);
void lm_embed_carve(lamb_vocab* v, LmArena* a);
// Shared-memory limits of the head's kernels on the current device.
int lm_head_setup();
}  // namespace lamb
