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
  int64_t kv_head;
  int32_t kv_token;
  int32_t nq, nk;
  int32_t splits;    // parts of the key range, joined by a second launch where > 1
  int32_t row_blocks;
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
  Divider by_H, by_G;
  uint32_t begin[kMaxPromptBatch];  // the requests' first workgroups; past the last, 2^32 - 1
  PromptDesc r[kMaxPromptBatch];
};
static_assert(sizeof(PromptArgs) <= 4000, "kernel arguments");

hipError_t launch_attn_prompt(const PromptArgs& a, int32_t dtype, int32_t d, hipStream_t stream);

// Attention of a batch's newest tokens over the paged cache.  The launch's
// workgroups are first those of the shared prefix (row blocks x KV heads x
// parts, over the rows of every request), then those of the rest ("tail") of each
// request (parts x row blocks x KV heads): with tail_parts == 0 a part is a request;
// else the device cuts the tails of at most kCutRequests requests into at most
// tail_parts parts, as short as that allows.
constexpr int kCutRequests = 256;
struct DecodeArgs {
  const uint16_t* q;
  const uint16_t* k;
  const uint16_t* v;
  uint16_t* out;
  float* lse;             // [B][Lq][Hq], may be null
  const int32_t* tables;  // [B][table_stride]
  const int32_t* lens;
  const uint8_t* tiers;   // may be null
  uint32_t* status;       // may be null
  // partial results, unnormalized sums and (reference, sum): prefix rows [parts][H]
  // [B Lq G], then tail rows [part][H][Lq G]
  float* part_o;
  float* part_ml;
  int32_t* first_part;  // [B]: a request's first tail part, and how many it has
  int32_t* part_count;
  int64_t q_request, q_token, q_head, out_request, out_token, out_head, table_stride, tier_request, tier_head;
  int64_t tail_at;       // first tail row of the partial results
  int32_t B, Lq, H, G, num_blocks, block_size, width, prefix, tier_len;
  int32_t prefix_parts, prefix_blocks, prefix_tiles, prefix_chunk;  // row blocks, 32-row tiles of one, tokens of a part
  int32_t tail_parts, tail_blocks, tail_tiles, tail_least;  // the last: 64-token tiles of a part, at least
  int32_t direct;                  // no parts: results are written at once
  uint32_t prefix_groups, groups;  // workgroups of the prefix, of the launch
  float alpha;
  Divider by_block, by_G, by_Lq;
};
hipError_t launch_attn_decode(const DecodeArgs& a, int32_t dtype, int32_t d, hipStream_t stream);

// Page operators.  op kPagesReserve: tables grow in place (out_tables are the
// tables, lens the old lengths); kPagesFork and kPagesCompact: out rows from
// source rows (parents; null: row c from row c).
enum { kPagesReserve = 0, kPagesFork = 1, kPagesCompact = 2 };
struct PageArgs {
  uint8_t* k;
  uint8_t* v;
  int32_t* refs;
  const int32_t* tables;   // [sources][width]
  const int32_t* lens;     // [sources]
  const int32_t* new_lens; // reserve
  const int32_t* parents;  // fork
  const uint8_t* tiers;    // compact
  int32_t* out_tables;     // [rows][out_width]
  int32_t* out_lens;
  uint32_t* status;
  // workspace
  uint32_t* ws_status;
  int32_t* ws_bad;
  int32_t* ws_off;
  int32_t* ws_need;
  int32_t* ws_shared;
  int32_t* ws_total;
  int32_t* ws_list;   // [num_blocks]
  int32_t* ws_kept;   // [rows][chunks]: kept tokens of a chunk, then before it
  int32_t* ws_first;  // [rows][chunks]: first dropped token
  int64_t tier_stride, row_bytes, plane_bytes;
  int32_t op, rows, sources, width, out_width, num_blocks, block_size, num_layers, tier_len;
  int32_t chunks, plane_groups, checked;
  uint32_t copy_groups;
  Divider by_block, by_units, by_width;
};
hipError_t launch_pages(const PageArgs& a, hipStream_t stream);
hipError_t launch_pages_free(const PageArgs& a, hipStream_t stream);

struct PageCopyArgs {
  const uint8_t* src_k;
  const uint8_t* src_v;
  uint8_t* dst_k;
  uint8_t* dst_v;
  const int32_t* src_pages;
  const int32_t* dst_pages;
  uint32_t* status;
  int64_t page_bytes, src_plane_bytes, dst_plane_bytes;
  int32_t count, src_blocks, dst_blocks;
  uint32_t planes, pieces;
  uint64_t units;
};
hipError_t launch_pages_copy(PageCopyArgs a, hipStream_t stream);

}  // namespace skv
