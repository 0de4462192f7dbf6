// Declarations shared by the attention and page operators' host API and kernels.
#pragma once

#include <stdint.h>

#include <hip/hip_runtime.h>

#include "../skv_internal.h"

namespace skv {

constexpr int kMaxPromptBatch = 48;  // requests per launch (descriptors travel as kernel arguments)

// One request of a prompt attention launch.  Strides in elements.
struct PromptDesc {
  const uint16_t* q;
  const uint16_t* k;
  const uint16_t* v;
  uint16_t* out;
  float* lse;  // [num_queries][Hq], may be null
  int64_t kv_token, kv_head;
  int32_t nq, nk;
  int32_t splits;    // parts of the key range, joined by a second launch where > 1
  uint32_t begin;    // the request's first workgroup
  uint32_t rows_at;  // splits > 1: the request's first row in the partial results
};

struct PromptArgs {
  int32_t count, H, G, causal;
  int32_t key_streams;  // 1: a workgroup's waves take 32 rows each; 2: pairs of waves share rows, each half the keys
  int32_t row_tiles;    // 32-row tiles per workgroup
  float alpha;          // scale * log2(e)
  uint32_t blocks;      // workgroups
  int64_t q_token, q_head, out_token, out_head;
  float* part_o;        // partial results: binary32 [rows][d], unnormalized
  float* part_ml;       // [rows][2]: reference and sum
  PromptDesc r[kMaxPromptBatch];
};
static_assert(sizeof(PromptArgs) <= 4000, "kernel arguments");

hipError_t launch_attn_prompt(const PromptArgs& a, int32_t dtype, int32_t d, hipStream_t stream);

}  // namespace skv
