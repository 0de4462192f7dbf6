// Host side of the attention and page operators of include/skv.h: argument
// checks, the rules that size launches, and workspace layouts.
#include <algorithm>
#include <cmath>
#include <cstring>

#include "serving_internal.h"

namespace skv {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int32_t kCus = 256;  // compute units of an MI355X

bool aligned(const void* p, uintptr_t to) { return p != nullptr && reinterpret_cast<uintptr_t>(p) % to == 0; }

bool shape_ok(int32_t dtype, int32_t Hq, int32_t H, int32_t d, float scale) {
  return (dtype == SKV_DTYPE_F16 || dtype == SKV_DTYPE_BF16) && H >= 1 && Hq >= H && Hq <= 65536 && Hq % H == 0 &&
         (d == 32 || d == 64 || d == 128 || d == 256) && std::isfinite(scale * kLog2e) && scale > 0.0f;
}

bool stride_ok(int64_t s) { return s > 0 && s % 8 == 0 && s < (int64_t{1} << 40); }

// Queries, keys and rows of a request: packed rows and tokens are 32-bit indexes in the kernels.
bool lengths_ok(const skv_attn_config* c, const skv_attn_request& r) {
  return r.num_queries >= 0 && r.num_keys >= 0 && r.num_keys <= (1 << 30) && r.num_queries <= (1 << 30) &&
         static_cast<int64_t>(r.num_queries) * (c->num_q_heads / c->num_kv_heads) <= (1 << 30);
}

skv_status check_prompt(const skv_attn_config* c, const skv_attn_request* reqs, int32_t count, bool pointers) {
  if (c == nullptr || count < 0 || (count > 0 && reqs == nullptr)) return SKV_ERR_INVALID_ARG;
  if (!shape_ok(c->dtype, c->num_q_heads, c->num_kv_heads, c->head_dim, c->scale)) return SKV_ERR_INVALID_ARG;
  if (c->causal != 0 && c->causal != 1) return SKV_ERR_INVALID_ARG;
  if (pointers && (!stride_ok(c->q_token_stride) || !stride_ok(c->q_head_stride) || !stride_ok(c->out_token_stride) ||
                   !stride_ok(c->out_head_stride)))
    return SKV_ERR_INVALID_ARG;
  for (int32_t i = 0; i < count; ++i) {
    const skv_attn_request& r = reqs[i];
    if (!lengths_ok(c, r)) return SKV_ERR_INVALID_ARG;
    if (!pointers || r.num_queries == 0) continue;
    if (!aligned(r.q, 16) || !aligned(r.out, 16)) return SKV_ERR_INVALID_ARG;
    if (r.lse != nullptr && !aligned(r.lse, 4)) return SKV_ERR_INVALID_ARG;
    if (r.num_keys == 0) continue;
    if (!aligned(r.k, 16) || !aligned(r.v, 16)) return SKV_ERR_INVALID_ARG;
    if (!stride_ok(r.kv_token_stride) || r.kv_token_stride >= (1 << 25) || !stride_ok(r.kv_head_stride))
      return SKV_ERR_INVALID_ARG;
  }
  return SKV_OK;
}

// 32-row tiles of a workgroup for this many rows.
int32_t row_tiles(int64_t rows) { return rows <= 32 ? 1 : rows <= 64 ? 2 : 4; }

// The requests of a launch, longest first (the heaviest workgroups start first).
struct PromptBatch {
  const skv_attn_request* r[kMaxPromptBatch];
  int32_t n;
  const skv_attn_request* const* begin() const { return r; }
  const skv_attn_request* const* end() const { return r + n; }
};

// How a launch runs.
struct PromptPlan {
  int32_t key_streams, row_tiles;
  int32_t splits[kMaxPromptBatch];
  uint64_t rows;    // partial rows
  uint64_t blocks;  // workgroups of an unsplit launch
};

int64_t prompt_blocks(const skv_attn_config* c, const skv_attn_request& r, int32_t per) {
  const int64_t rows = static_cast<int64_t>(r.num_queries) * (c->num_q_heads / c->num_kv_heads);
  return (rows + per - 1) / per * c->num_kv_heads;
}

PromptPlan plan_prompt(const skv_attn_config* c, const PromptBatch& reqs) {
  PromptPlan p{1, 4, {}, 0, 0};
  const int64_t room = c->head_dim >= 256 ? kCus : 2 * kCus;  // workgroups that the GPU holds at once
  auto blocks = [&](int32_t tiles) {
    int64_t n = 0;
    for (const skv_attn_request* r : reqs) n += prompt_blocks(c, *r, 32 * tiles);
    return n;
  };
  int32_t most_keys = 0;
  int64_t most_rows = 0;
  for (const skv_attn_request* r : reqs) {
    most_keys = std::max(most_keys, r->num_keys);
    most_rows = std::max(most_rows, static_cast<int64_t>(r->num_queries) * (c->num_q_heads / c->num_kv_heads));
  }
  // Workgroups of 128 rows, the most work per byte staged, where they fill three
  // quarters of the room or their keys will be split; otherwise of 64 or 32 rows with
  // two waves per row tile.  128 against 64 rows: 1000 queries of 32 x 128 on 8 KV heads
  // (half of the room) 24.1 us and 21.0, 6 x 250 (three quarters) 15.2 and 18.2, 2 x 900
  // (nine tenths) 30.5 and 28.4; 1000 of 16 x 256 (half) 37.4 and 29.3, 4 x 360 (three
  // quarters) 21.2 and 27.7.
  const bool splits = most_keys > 1024;
  if (blocks(4) * 4 < room * 3 && !(splits && most_rows >= 128)) {
    p.key_streams = 2;
    p.row_tiles = row_tiles(std::min<int64_t>(most_rows, 64));
  }
  // Parts of at least 256 keys that fill the room (100 queries of 32 x 128 over 30000
  // keys: 474 us in one part, 77 in 16); a second launch and its traffic cost about
  // 10 us, so short keys are left whole.  Of at least 512: one query of 32 x 128 over
  // 2048 keys 13.2 us against 10.5; of 128: 9.3, but 30 queries 15.0 against 14.4.
  const int64_t all = std::max<int64_t>(1, blocks(p.row_tiles));
  p.blocks = static_cast<uint64_t>(all);
  for (int32_t i = 0; i < reqs.n; ++i) {
    const int64_t rows = static_cast<int64_t>(reqs.r[i]->num_queries) * c->num_q_heads;
    int64_t s = 1;
    if (splits && 2 * all <= room) s = std::max<int64_t>(1, std::min<int64_t>({room / all, reqs.r[i]->num_keys / 256, 64}));
    p.splits[i] = static_cast<int32_t>(s);
    if (s > 1) p.rows += static_cast<uint64_t>(rows * s);
  }
  return p;
}

// The launches of a call: its requests with queries in their order, kMaxPromptBatch
// at a time, sorted within one.  Nothing here allocates.
template <class F>
skv_status prompt_launches(const skv_attn_config* c, const skv_attn_request* reqs, int32_t count, F each) {
  for (int32_t at = 0; at < count;) {
    PromptBatch some;
    for (some.n = 0; at < count && some.n < kMaxPromptBatch; ++at) {
      if (reqs[at].num_queries == 0) continue;
      int32_t i = some.n++;
      for (; i > 0 && some.r[i - 1]->num_keys < reqs[at].num_keys; --i) some.r[i] = some.r[i - 1];
      some.r[i] = &reqs[at];
    }
    if (some.n == 0) break;
    const skv_status st = each(some, plan_prompt(c, some));
    if (st != SKV_OK) return st;
  }
  return SKV_OK;
}

// How skv_attn_decode cuts its work (the counts, lengths and dimensions of c are
// valid).
struct DecodePlan {
  int32_t prefix_parts, prefix_blocks, prefix_tiles, prefix_chunk, tail_parts, tail_blocks, tail_tiles, tail_least;
  uint64_t prefix_groups, groups, prefix_rows, part_rows, bytes;  // (bytes 0: no parts)
};

DecodePlan plan_decode(const skv_decode_config* c) {
  DecodePlan p{};
  if (c->num_requests == 0 || c->num_queries == 0) return p;
  const int64_t H = c->num_kv_heads, G = c->num_q_heads / H, own = c->num_queries * G, all = own * c->num_requests;
  const int64_t tail = std::max(0, c->max_len - c->prefix_len);
  const int64_t room = c->head_dim >= 256 ? kCus : 2 * kCus;  // workgroups that the GPU holds at once
  auto up = [](int64_t x, int64_t to) { return (x + to - 1) / to; };
  p.tail_tiles = row_tiles(own);
  p.tail_blocks = static_cast<int32_t>(up(own, 32 * p.tail_tiles));
  // The prefix gets the share of the room that its tiles are of all (one of many rows
  // counted twice, the tails taken to be half as long as the longest), at most half:
  // more parts are more partial results to write and join (64 requests behind 16384
  // tokens of 8 x 128, 0.4 of them dropped: 45 us with all of the room at most, 38 with
  // half, 47 with a quarter), of 128 tokens at least (4 requests behind 512 of 8 x 128:
  // 11.8 us, by 64 11.2, by 256 13.6; 40 behind 1024: 17.3, 24.8 and 18.5).  By its share
  // against always half: 64 behind 2048 with up to 3800 of their own, 123 us against 139;
  // 12 behind 2048 of 8 x 256, 5 queries each, with up to 1450, 34 against 47.
  if (c->prefix_len > 0) {
    p.prefix_tiles = row_tiles(all);
    p.prefix_blocks = static_cast<int32_t>(up(all, 32 * p.prefix_tiles));
    const int64_t here = 2 * p.prefix_blocks * up(c->prefix_len, 64);
    const int64_t there = c->num_requests * p.tail_blocks * up(tail / 2, 64);
    const int64_t share = std::min(room / 2, room * here / (here + there));
    const int64_t parts = std::max<int64_t>(1, std::min(share / (H * p.prefix_blocks), up(c->prefix_len, 128)));
    p.prefix_chunk = static_cast<int32_t>(up(up(c->prefix_len, parts), 64) * 64);
    p.prefix_parts = static_cast<int32_t>(up(c->prefix_len, p.prefix_chunk));
    p.prefix_groups = static_cast<uint64_t>(H * p.prefix_blocks * p.prefix_parts);
    p.prefix_rows = static_cast<uint64_t>(p.prefix_parts * H * all);
  }
  // The tails in as many parts as fill the rest of the room, two per request at least
  // where they may be long and uneven, of 128 tokens at least (as far as max_len says);
  // of 64 where so few fill at most half the room and a request has 32 at most, which
  // its join reads at once (one request of 500 tokens of 8 x 128: 11.9 us against
  // 12.8; of 8192 of 4 x 128: 16.6 against 14.4); whole where that fills the room with
  // short ones (64 requests of up to 400 tokens: 14 us whole, 20 with a second launch
  // for the parts).  Whole up to 256 tokens (8 requests of 250 tokens of 8 x 128: 10.0
  // us, cut 11.8; of 500: 14.0 whole, 12.7 cut).  Two parts from 2048 (64 requests of 100
  // to 4000 tokens: 127 us, in one 141; all of 4000: 202 and 196; of 100 to 1500: 50 in
  // two, 44 whole).
  const int64_t groups = H * p.tail_blocks, left = room - static_cast<int64_t>(p.prefix_groups);
  p.tail_least = tail <= 2048 && 2 * groups * c->num_requests * up(tail, 64) <= room ? 1 : 2;
  int64_t parts = std::max(left / groups, c->num_requests * static_cast<int64_t>(tail >= 2048 ? 2 : 1));
  parts = std::min(parts, c->num_requests * up(tail, 64 * p.tail_least));
  const bool whole = tail <= 256 || (tail < 2048 && c->num_requests * groups >= left);
  if (c->num_requests <= kCutRequests && !whole && parts > 1) p.tail_parts = static_cast<int32_t>(parts);
  const int64_t runs = p.tail_parts > 0 ? p.tail_parts : c->num_requests;
  p.groups = p.prefix_groups + static_cast<uint64_t>(groups * runs);
  if (p.prefix_parts == 0 && p.tail_parts == 0) return p;
  p.part_rows = p.prefix_rows + static_cast<uint64_t>(runs * H * own);
  p.bytes = p.part_rows * static_cast<uint64_t>(c->head_dim + 2) * 4u + 8u * static_cast<uint64_t>(c->num_requests);
  return p;
}

skv_status check_decode_sizes(const skv_decode_config* c) {
  if (c == nullptr || !shape_ok(SKV_DTYPE_F16, c->num_q_heads, c->num_kv_heads, c->head_dim, 1.0f))
    return SKV_ERR_INVALID_ARG;
  if (c->num_requests < 0 || c->num_queries < 0 || c->max_len < 0 || c->prefix_len < 0) return SKV_ERR_INVALID_ARG;
  // (a join of 2^26 - 3 rows or more, a wave each, would be a grid of 2^32 threads, which no launch takes)
  if (static_cast<int64_t>(c->num_requests) * c->num_queries > (1 << 20) ||
      static_cast<int64_t>(c->num_requests) * c->num_queries * c->num_q_heads > (1 << 26) - 4)
    return SKV_ERR_INVALID_ARG;
  return SKV_OK;
}

uint64_t up256(uint64_t x) { return (x + 255) / 256 * 256; }

// Workspace of the page operators: the status, five words per output row, the free
// pages' list, two words per chunk of 256 tokens.
struct PageLayout {
  uint64_t rows, list, kept, first, total;
  PageLayout(int64_t requests, int64_t blocks, int64_t chunks) {
    rows = 256;
    list = rows + 5 * up256(4u * static_cast<uint64_t>(requests));
    kept = list + up256(4u * static_cast<uint64_t>(blocks));
    first = kept + up256(4u * static_cast<uint64_t>(requests * chunks));
    total = first + up256(4u * static_cast<uint64_t>(requests * chunks));
  }
};

bool pool_ok(const skv_page_pool* p, bool caches, bool refs) {
  return p != nullptr && p->num_layers >= 1 && p->num_layers <= 65536 && p->num_blocks >= 1 && p->block_size >= 1 &&
         static_cast<int64_t>(p->num_blocks) * p->block_size <= INT32_MAX && p->row_bytes >= 16 &&
         p->row_bytes % 16 == 0 && p->row_bytes <= (1 << 24) &&
         (!caches || (aligned(p->k_cache, 16) && aligned(p->v_cache, 16))) && (!refs || aligned(p->refs, 16));
}

bool tables_ok(const skv_page_pool* p, const void* tables, int32_t width, const void* lens, int32_t requests) {
  if (requests < 0 || requests > (1 << 24) || width < 0 || static_cast<int64_t>(width) * p->block_size > (1 << 30) ||
      static_cast<int64_t>(requests) * width > INT32_MAX)
    return false;
  return requests == 0 || (aligned(lens, 4) && (width == 0 || aligned(tables, 4)));
}

PageArgs page_args(const skv_page_pool* p, const int32_t* tables, int32_t width, const int32_t* lens, int32_t rows,
                   uint32_t* status) {
  PageArgs a;
  std::memset(&a, 0, sizeof(a));
  a.k = static_cast<uint8_t*>(p->k_cache);
  a.v = static_cast<uint8_t*>(p->v_cache);
  a.refs = p->refs;
  a.tables = tables;
  a.lens = lens;
  a.status = status;
  a.rows = rows;
  a.sources = rows;
  a.width = width;
  a.num_blocks = p->num_blocks;
  a.block_size = p->block_size;
  a.num_layers = p->num_layers;
  a.row_bytes = p->row_bytes;
  a.plane_bytes = static_cast<int64_t>(p->num_blocks) * p->block_size * p->row_bytes;
  a.chunks = 1;
  a.plane_groups = 1;
  a.by_block = make_divider(static_cast<uint32_t>(p->block_size));
  a.by_units = make_divider(static_cast<uint32_t>(p->row_bytes / 16));
  a.by_width = make_divider(static_cast<uint32_t>(std::max(1, width)));
  return a;
}

skv_status page_workspace(PageArgs* a, int64_t chunks, void* ws, uint64_t ws_bytes) {
  const PageLayout lay(a->rows, a->num_blocks, chunks);
  if (!aligned(ws, 16)) return SKV_ERR_INVALID_ARG;
  if (ws_bytes < lay.total) return SKV_ERR_CAPACITY;
  uint8_t* base = static_cast<uint8_t*>(ws);
  const uint64_t row_area = up256(4u * static_cast<uint64_t>(a->rows));
  auto at = [&](uint64_t off) { return reinterpret_cast<int32_t*>(base + off); };
  a->ws_status = reinterpret_cast<uint32_t*>(base);
  a->ws_bad = at(lay.rows);
  a->ws_off = at(lay.rows + row_area);
  a->ws_need = at(lay.rows + 2 * row_area);
  a->ws_shared = at(lay.rows + 3 * row_area);
  a->ws_total = at(lay.rows + 4 * row_area);
  a->ws_list = at(lay.list);
  a->ws_kept = at(lay.kept);
  a->ws_first = at(lay.first);
  return SKV_OK;
}

// Whether an output of fork or compact lies on one of their inputs, which the last
// launch still reads.
struct Span {
  const void* p;
  uint64_t n;  // int32 entries
};
bool overlap(const Span& x, const Span& y) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(x.p), b = reinterpret_cast<uintptr_t>(y.p);
  return x.n > 0 && y.n > 0 && a < b + 4 * y.n && b < a + 4 * x.n;
}
bool outputs_apart(const PageArgs& a) {
  const uint64_t rows = static_cast<uint64_t>(a.rows), sources = static_cast<uint64_t>(a.sources);
  const Span in[3] = {{a.tables, sources * static_cast<uint64_t>(a.width)}, {a.lens, sources}, {a.parents, a.parents ? rows : 0}};
  const Span out[2] = {{a.out_tables, rows * static_cast<uint64_t>(a.out_width)}, {a.out_lens, rows}};
  bool apart = !overlap(out[0], out[1]);
  for (const Span& x : in) apart = apart && !overlap(x, out[0]) && !overlap(x, out[1]);
  return apart;
}

// Workgroups of the row copies: the planes are spread until the launch has about
// `want` workgroups.
skv_status spread_planes(PageArgs* a, int64_t pieces, int64_t want) {
  const int64_t planes = 2 * static_cast<int64_t>(a->num_layers);
  a->plane_groups = static_cast<int32_t>(std::max<int64_t>(1, std::min(planes, (want + pieces - 1) / pieces)));
  const int64_t groups = pieces * a->plane_groups;
  // (a table's entries, at most 2^31, take 2^21 workgroups more)
  if (groups > static_cast<int64_t>(kMaxGridThreads / 512)) return SKV_ERR_CAPACITY;
  a->copy_groups = static_cast<uint32_t>(groups);
  return SKV_OK;
}

}  // namespace
}  // namespace skv

using namespace skv;

extern "C" {

skv_status skv_attn_prompt_workspace_size(const skv_attn_config* cfg, const skv_attn_request* reqs, int32_t count,
                                          uint64_t* bytes) {
  if (bytes == nullptr) return SKV_ERR_INVALID_ARG;
  const skv_status st = check_prompt(cfg, reqs, count, false);
  if (st != SKV_OK) return st;
  uint64_t most = 0;
  prompt_launches(cfg, reqs, count, [&](const PromptBatch&, const PromptPlan& p) {
    most = std::max(most, p.rows * static_cast<uint64_t>(cfg->head_dim + 2) * 4u);
    return SKV_OK;
  });
  *bytes = most;
  return SKV_OK;
}

skv_status skv_attn_prompt(const skv_attn_config* cfg, const skv_attn_request* reqs, int32_t count, void* ws,
                           uint64_t ws_bytes, hipStream_t stream) {
  skv_status st = check_prompt(cfg, reqs, count, true);
  if (st != SKV_OK) return st;
  if (ws != nullptr && !aligned(ws, 16)) return SKV_ERR_INVALID_ARG;
  // (split launches are small ones: this bounds them too)
  st = prompt_launches(cfg, reqs, count, [](const PromptBatch&, const PromptPlan& p) {
    return p.blocks > kMaxGridThreads / 512 ? SKV_ERR_CAPACITY : SKV_OK;
  });
  if (st != SKV_OK) return st;
  return prompt_launches(cfg, reqs, count, [&](const PromptBatch& some, const PromptPlan& p) {
    PromptArgs a;
    std::memset(&a, 0, sizeof(a));
    a.count = some.n;
    a.H = cfg->num_kv_heads;
    a.G = cfg->num_q_heads / cfg->num_kv_heads;
    a.causal = cfg->causal;
    a.key_streams = p.key_streams;
    a.row_tiles = p.row_tiles;
    a.alpha = cfg->scale * kLog2e;
    a.q_token = cfg->q_token_stride;
    a.q_head = cfg->q_head_stride;
    a.out_token = cfg->out_token_stride;
    a.out_head = cfg->out_head_stride;
    const bool split = ws != nullptr && ws_bytes >= p.rows * static_cast<uint64_t>(cfg->head_dim + 2) * 4u;
    a.part_o = static_cast<float*>(ws);
    a.part_ml = split ? a.part_o + p.rows * static_cast<uint64_t>(cfg->head_dim) : nullptr;
    a.by_H = make_divider(static_cast<uint32_t>(a.H));
    a.by_G = make_divider(static_cast<uint32_t>(a.G));
    std::fill(a.begin, a.begin + kMaxPromptBatch, UINT32_MAX);
    uint64_t begin = 0, rows_at = 0;
    for (int32_t i = 0; i < a.count; ++i) {
      const skv_attn_request& q = *some.r[i];
      PromptDesc& r = a.r[i];
      r.q = static_cast<const uint16_t*>(q.q);
      r.k = static_cast<const uint16_t*>(q.k);
      r.v = static_cast<const uint16_t*>(q.v);
      r.out = static_cast<uint16_t*>(q.out);
      r.lse = q.lse;
      r.kv_token = static_cast<int32_t>(q.kv_token_stride);
      r.kv_head = q.kv_head_stride;
      r.nq = q.num_queries;
      r.nk = q.num_keys;
      r.splits = split ? p.splits[i] : 1;
      r.row_blocks = static_cast<int32_t>(prompt_blocks(cfg, q, 32 * a.row_tiles) / a.H);
      r.rows_at = static_cast<uint32_t>(rows_at);
      a.begin[i] = static_cast<uint32_t>(begin);
      begin += static_cast<uint64_t>(r.row_blocks) * static_cast<uint64_t>(a.H) * static_cast<uint64_t>(r.splits);
      if (r.splits > 1) rows_at += static_cast<uint64_t>(q.num_queries) * cfg->num_q_heads * r.splits;
    }
    a.blocks = static_cast<uint32_t>(begin);
    return launch_attn_prompt(a, cfg->dtype, cfg->head_dim, stream) == hipSuccess ? SKV_OK : SKV_ERR_DEVICE;
  });
}

skv_status skv_attn_decode_workspace_size(const skv_decode_config* cfg, uint64_t* bytes) {
  if (bytes == nullptr) return SKV_ERR_INVALID_ARG;
  const skv_status st = check_decode_sizes(cfg);
  if (st == SKV_OK) *bytes = plan_decode(cfg).bytes;
  return st;
}

skv_status skv_attn_decode(const skv_decode_config* cfg, const void* q, const void* k_cache, const void* v_cache,
                           const int32_t* tables, const int32_t* lens, const uint8_t* tiers, void* out, float* lse,
                           uint32_t* dev_status, void* ws, uint64_t ws_bytes, hipStream_t stream) {
  skv_status st = check_decode_sizes(cfg);
  if (st != SKV_OK) return st;
  const skv_decode_config& c = *cfg;
  if (!shape_ok(c.dtype, c.num_q_heads, c.num_kv_heads, c.head_dim, c.scale)) return SKV_ERR_INVALID_ARG;
  if (c.num_blocks < 1 || c.block_size < 1 || static_cast<int64_t>(c.num_blocks) * c.block_size > INT32_MAX ||
      c.table_width < 0 || static_cast<int64_t>(c.table_width) * c.block_size > (1 << 30) ||
      c.table_stride < c.table_width)
    return SKV_ERR_INVALID_ARG;
  if (c.prefix_len % c.block_size != 0 || c.prefix_len > c.table_width * c.block_size) return SKV_ERR_INVALID_ARG;
  if (!stride_ok(c.q_request_stride) || !stride_ok(c.q_token_stride) || !stride_ok(c.q_head_stride) ||
      !stride_ok(c.out_request_stride) || !stride_ok(c.out_token_stride) || !stride_ok(c.out_head_stride))
    return SKV_ERR_INVALID_ARG;
  if (tiers != nullptr && (c.tier_len < 0 || c.tier_request_stride < 0 || c.tier_head_stride < 0)) return SKV_ERR_INVALID_ARG;
  if (c.num_requests == 0 || c.num_queries == 0) return SKV_OK;
  if (!aligned(q, 16) || !aligned(k_cache, 16) || !aligned(v_cache, 16) || !aligned(out, 16) || !aligned(lens, 4) ||
      (c.table_width > 0 && !aligned(tables, 4)) || (lse != nullptr && !aligned(lse, 4)) || (dev_status != nullptr && !aligned(dev_status, 4)))
    return SKV_ERR_INVALID_ARG;
  const DecodePlan p = plan_decode(cfg);
  if (p.bytes > 0 && !aligned(ws, 16)) return SKV_ERR_INVALID_ARG;
  if (ws_bytes < p.bytes || p.groups > kMaxGridThreads / 512) return SKV_ERR_CAPACITY;
  const int32_t H = c.num_kv_heads, G = c.num_q_heads / H;
  DecodeArgs a;
  std::memset(&a, 0, sizeof(a));
  a.q = static_cast<const uint16_t*>(q);
  a.k = static_cast<const uint16_t*>(k_cache);
  a.v = static_cast<const uint16_t*>(v_cache);
  a.out = static_cast<uint16_t*>(out);
  a.lse = lse;
  a.tables = tables;
  a.lens = lens;
  a.tiers = tiers;
  a.status = dev_status;
  a.part_o = static_cast<float*>(ws);
  a.direct = p.bytes == 0;
  if (!a.direct) {
    a.part_ml = a.part_o + p.part_rows * static_cast<uint64_t>(c.head_dim);
    a.first_part = reinterpret_cast<int32_t*>(a.part_ml + 2 * p.part_rows);
    a.part_count = a.first_part + c.num_requests;
  }
  a.tail_at = static_cast<int64_t>(p.prefix_rows);
  a.q_request = c.q_request_stride;
  a.q_token = c.q_token_stride;
  a.q_head = c.q_head_stride;
  a.out_request = c.out_request_stride;
  a.out_token = c.out_token_stride;
  a.out_head = c.out_head_stride;
  a.table_stride = c.table_stride;
  a.tier_request = c.tier_request_stride;
  a.tier_head = c.tier_head_stride;
  a.B = c.num_requests;
  a.Lq = c.num_queries;
  a.H = H;
  a.G = G;
  a.num_blocks = c.num_blocks;
  a.block_size = c.block_size;
  a.width = c.table_width;
  a.prefix = c.prefix_len;
  a.tier_len = c.tier_len;
  a.prefix_parts = p.prefix_parts;
  a.prefix_blocks = p.prefix_blocks;
  a.prefix_tiles = p.prefix_tiles;
  a.prefix_chunk = p.prefix_chunk;
  a.tail_parts = p.tail_parts;
  a.tail_blocks = p.tail_blocks;
  a.tail_tiles = p.tail_tiles;
  a.tail_least = p.tail_least;
  a.prefix_groups = static_cast<uint32_t>(p.prefix_groups);
  a.groups = static_cast<uint32_t>(p.groups);
  a.alpha = c.scale * kLog2e;
  a.by_block = make_divider(static_cast<uint32_t>(c.block_size));
  a.by_G = make_divider(static_cast<uint32_t>(G));
  a.by_Lq = make_divider(static_cast<uint32_t>(c.num_queries));
  return launch_attn_decode(a, c.dtype, c.head_dim, stream) == hipSuccess ? SKV_OK : SKV_ERR_DEVICE;
}

skv_status skv_pages_workspace_size(int32_t num_requests, int32_t num_blocks, int32_t max_len, uint64_t* bytes) {
  if (bytes == nullptr || num_requests < 0 || num_blocks < 1 || max_len < 0 || max_len > (1 << 30)) return SKV_ERR_INVALID_ARG;
  // (four chunks to spare: a table's last page may reach past max_len)
  *bytes = PageLayout(num_requests, num_blocks, (static_cast<int64_t>(max_len) + 255) / 256 + 4).total;
  return SKV_OK;
}

skv_status skv_pages_reserve(const skv_page_pool* pool, int32_t* tables, int32_t table_width, const int32_t* lens,
                             const int32_t* new_lens, int32_t num_requests, uint32_t* dev_status, void* ws,
                             uint64_t ws_bytes, hipStream_t stream) {
  if (!pool_ok(pool, false, true) || !tables_ok(pool, tables, table_width, lens, num_requests) || !aligned(dev_status, 4) ||
      (num_requests > 0 && !aligned(new_lens, 4)))
    return SKV_ERR_INVALID_ARG;
  PageArgs a = page_args(pool, tables, table_width, lens, num_requests, dev_status);
  a.op = kPagesReserve;
  a.new_lens = new_lens;
  a.out_tables = tables;
  a.out_width = table_width;
  const skv_status st = page_workspace(&a, 0, ws, ws_bytes);
  if (st != SKV_OK) return st;
  return launch_pages(a, stream) == hipSuccess ? SKV_OK : SKV_ERR_DEVICE;
}

skv_status skv_pages_fork(const skv_page_pool* pool, const int32_t* tables, int32_t table_width, const int32_t* lens,
                          int32_t num_requests, const int32_t* parents, int32_t num_children, int32_t* out_tables,
                          int32_t out_width, int32_t* out_lens, uint32_t* dev_status, void* ws, uint64_t ws_bytes,
                          hipStream_t stream) {
  if (!pool_ok(pool, true, true) || !tables_ok(pool, tables, table_width, lens, num_requests) ||
      !tables_ok(pool, out_tables, out_width, out_lens, num_children) || !aligned(dev_status, 4) ||
      (num_children > 0 && !aligned(parents, 4)))
    return SKV_ERR_INVALID_ARG;
  PageArgs a = page_args(pool, tables, table_width, lens, num_children, dev_status);
  a.op = kPagesFork;
  a.sources = num_requests;
  a.parents = parents;
  a.out_tables = out_tables;
  a.out_width = out_width;
  a.out_lens = out_lens;
  // one workgroup looks over 2000 entries faster than a launch more costs (8 children of
  // 4001 tokens forked, grown and released: 17.8 us against 19.5), 8000 as fast (25.1,
  // 24.6), 16000 slower (29.4, 24.9)
  a.checked = static_cast<int64_t>(num_children) * table_width > 8192;
  skv_status st = page_workspace(&a, 0, ws, ws_bytes);
  if (st == SKV_OK && !outputs_apart(a)) st = SKV_ERR_INVALID_ARG;
  if (st == SKV_OK) st = spread_planes(&a, std::max(1, num_children), 1024);
  if (st != SKV_OK) return st;
  if (num_children == 0) a.copy_groups = 0;
  return launch_pages(a, stream) == hipSuccess ? SKV_OK : SKV_ERR_DEVICE;
}

skv_status skv_pages_compact(const skv_page_pool* pool, const int32_t* tables, int32_t table_width, const int32_t* lens,
                             int32_t num_requests, const uint8_t* tiers, int32_t tier_len, int64_t tier_stride,
                             int32_t* out_tables, int32_t out_width, int32_t* out_lens, uint32_t* dev_status, void* ws,
                             uint64_t ws_bytes, hipStream_t stream) {
  if (!pool_ok(pool, true, true) || !tables_ok(pool, tables, table_width, lens, num_requests) ||
      !tables_ok(pool, out_tables, out_width, out_lens, num_requests) || !aligned(dev_status, 4) || tier_len < 0 ||
      tier_stride < 0 || (num_requests > 0 && tier_len > 0 && tiers == nullptr))
    return SKV_ERR_INVALID_ARG;
  PageArgs a = page_args(pool, tables, table_width, lens, num_requests, dev_status);
  a.op = kPagesCompact;
  a.tiers = tiers;
  a.tier_len = tier_len;
  a.tier_stride = tier_stride;
  a.out_tables = out_tables;
  a.out_width = out_width;
  a.out_lens = out_lens;
  a.chunks = static_cast<int32_t>(std::max<int64_t>(1, (static_cast<int64_t>(table_width) * pool->block_size + 255) / 256));
  skv_status st = page_workspace(&a, a.chunks, ws, ws_bytes);
  if (st == SKV_OK && !outputs_apart(a)) st = SKV_ERR_INVALID_ARG;
  if (st == SKV_OK) st = spread_planes(&a, std::max<int64_t>(1, static_cast<int64_t>(num_requests) * a.chunks), 4096);
  if (st != SKV_OK) return st;
  if (num_requests == 0) a.copy_groups = 0;
  return launch_pages(a, stream) == hipSuccess ? SKV_OK : SKV_ERR_DEVICE;
}

skv_status skv_pages_free(const skv_page_pool* pool, const int32_t* tables, int32_t table_width, const int32_t* lens,
                          int32_t num_requests, uint32_t* dev_status, hipStream_t stream) {
  if (!pool_ok(pool, false, true) || !tables_ok(pool, tables, table_width, lens, num_requests) || !aligned(dev_status, 4))
    return SKV_ERR_INVALID_ARG;
  const PageArgs a = page_args(pool, tables, table_width, lens, num_requests, dev_status);
  return launch_pages_free(a, stream) == hipSuccess ? SKV_OK : SKV_ERR_DEVICE;
}

skv_status skv_pages_copy(const skv_page_pool* src, const skv_page_pool* dst, const int32_t* src_pages,
                          const int32_t* dst_pages, int32_t count, uint32_t* dev_status, hipStream_t stream) {
  if (!pool_ok(src, true, false) || !pool_ok(dst, true, false) || src->num_layers != dst->num_layers ||
      src->block_size != dst->block_size || src->row_bytes != dst->row_bytes || count < 0 || !aligned(dev_status, 4) ||
      (count > 0 && (!aligned(src_pages, 4) || !aligned(dst_pages, 4))))
    return SKV_ERR_INVALID_ARG;
  PageCopyArgs a;
  std::memset(&a, 0, sizeof(a));
  a.src_k = static_cast<const uint8_t*>(src->k_cache);
  a.src_v = static_cast<const uint8_t*>(src->v_cache);
  a.dst_k = static_cast<uint8_t*>(dst->k_cache);
  a.dst_v = static_cast<uint8_t*>(dst->v_cache);
  a.src_pages = src_pages;
  a.dst_pages = dst_pages;
  a.status = dev_status;
  a.page_bytes = static_cast<int64_t>(src->block_size) * src->row_bytes;
  a.src_plane_bytes = a.page_bytes * src->num_blocks;
  a.dst_plane_bytes = a.page_bytes * dst->num_blocks;
  a.count = count;
  a.src_blocks = src->num_blocks;
  a.dst_blocks = dst->num_blocks;
  a.planes = 2u * static_cast<uint32_t>(src->num_layers);
  // units of 32 KB, numbered in 32 bits
  if (static_cast<uint64_t>(count) * a.planes > UINT32_MAX / static_cast<uint64_t>((a.page_bytes + 32767) / 32768))
    return SKV_ERR_CAPACITY;
  return launch_pages_copy(a, stream) == hipSuccess ? SKV_OK : SKV_ERR_DEVICE;
}

}  // extern "C"
