// Host side of the attention and page operators of include/skv.h: argument
// checks, the rules that size launches, and workspace layouts.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <numeric>
#include <vector>

#include "serving_internal.h"

namespace skv {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int32_t kCus = 256;  // compute units of an MI355X

bool aligned(const void* p, uintptr_t to) { return p != nullptr && reinterpret_cast<uintptr_t>(p) % to == 0; }

bool shape_ok(int32_t dtype, int32_t Hq, int32_t H, int32_t d, float scale) {
  return (dtype == SKV_DTYPE_F16 || dtype == SKV_DTYPE_BF16) && H >= 1 && Hq >= H && Hq <= 65536 && Hq % H == 0 &&
         (d == 32 || d == 64 || d == 128 || d == 256) && std::isfinite(scale) && scale > 0.0f;
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

// How a launch of requests [0, n) (already ordered) runs.
struct PromptPlan {
  int32_t key_streams, row_tiles;
  std::vector<int32_t> splits;
  uint64_t rows;  // partial rows
};

int64_t prompt_blocks(const skv_attn_config* c, const skv_attn_request& r, int32_t per) {
  const int64_t rows = static_cast<int64_t>(r.num_queries) * (c->num_q_heads / c->num_kv_heads);
  return (rows + per - 1) / per * c->num_kv_heads;
}

PromptPlan plan_prompt(const skv_attn_config* c, const std::vector<const skv_attn_request*>& reqs) {
  PromptPlan p{1, 4, {}, 0};
  auto blocks = [&](int32_t tiles) {
    int64_t n = 0;
    for (const skv_attn_request* r : reqs) n += prompt_blocks(c, *r, 32 * tiles);
    return n;
  };
  if (blocks(4) < 2 * kCus) {
    p.key_streams = 2;
    p.row_tiles = blocks(2) < kCus ? 1 : 2;
  }
  const int64_t all = blocks(p.row_tiles);
  for (const skv_attn_request* r : reqs) {
    const int64_t rows = static_cast<int64_t>(r->num_queries) * c->num_q_heads;
    int64_t s = 1;
    if (all < kCus) s = std::min<int64_t>(2 * kCus / std::max<int64_t>(all, 1), r->num_keys / 512);
    s = std::max<int64_t>(1, std::min<int64_t>(s, 64));
    p.splits.push_back(static_cast<int32_t>(s));
    if (s > 1) p.rows += static_cast<uint64_t>(rows * s);
  }
  return p;
}

// The requests with queries, longest first (the heaviest workgroups start first).
std::vector<const skv_attn_request*> prompt_order(const skv_attn_request* reqs, int32_t count) {
  std::vector<const skv_attn_request*> order;
  for (int32_t i = 0; i < count; ++i)
    if (reqs[i].num_queries > 0) order.push_back(&reqs[i]);
  std::stable_sort(order.begin(), order.end(),
                   [](const skv_attn_request* x, const skv_attn_request* y) { return x->num_keys > y->num_keys; });
  return order;
}

template <class F>
skv_status prompt_launches(const skv_attn_config* c, const skv_attn_request* reqs, int32_t count, F each) {
  const std::vector<const skv_attn_request*> order = prompt_order(reqs, count);
  for (size_t first = 0; first < order.size(); first += kMaxPromptBatch) {
    const size_t n = std::min<size_t>(kMaxPromptBatch, order.size() - first);
    const std::vector<const skv_attn_request*> some(order.begin() + first, order.begin() + first + n);
    const skv_status st = each(some, plan_prompt(c, some));
    if (st != SKV_OK) return st;
  }
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
  prompt_launches(cfg, reqs, count, [&](const std::vector<const skv_attn_request*>&, const PromptPlan& p) {
    most = std::max(most, p.rows * static_cast<uint64_t>(cfg->head_dim + 2) * 4u);
    return SKV_OK;
  });
  *bytes = most;
  return SKV_OK;
}

skv_status skv_attn_prompt(const skv_attn_config* cfg, const skv_attn_request* reqs, int32_t count, void* ws,
                           uint64_t ws_bytes, hipStream_t stream) {
  const skv_status st = check_prompt(cfg, reqs, count, true);
  if (st != SKV_OK) return st;
  if (ws != nullptr && !aligned(ws, 16)) return SKV_ERR_INVALID_ARG;
  return prompt_launches(cfg, reqs, count, [&](const std::vector<const skv_attn_request*>& some, const PromptPlan& p) {
    PromptArgs a;
    std::memset(&a, 0, sizeof(a));
    a.count = static_cast<int32_t>(some.size());
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
    uint64_t begin = 0, rows_at = 0;
    for (int32_t i = 0; i < a.count; ++i) {
      const skv_attn_request& q = *some[i];
      PromptDesc& r = a.r[i];
      r.q = static_cast<const uint16_t*>(q.q);
      r.k = static_cast<const uint16_t*>(q.k);
      r.v = static_cast<const uint16_t*>(q.v);
      r.out = static_cast<uint16_t*>(q.out);
      r.lse = q.lse;
      r.kv_token = q.kv_token_stride;
      r.kv_head = q.kv_head_stride;
      r.nq = q.num_queries;
      r.nk = q.num_keys;
      r.splits = split ? p.splits[i] : 1;
      r.begin = static_cast<uint32_t>(begin);
      r.rows_at = static_cast<uint32_t>(rows_at);
      begin += static_cast<uint64_t>(prompt_blocks(cfg, q, 32 * a.row_tiles)) * static_cast<uint64_t>(r.splits);
      if (r.splits > 1) rows_at += static_cast<uint64_t>(q.num_queries) * cfg->num_q_heads * r.splits;
      if (begin > kMaxGridThreads / 256 || rows_at > UINT32_MAX) return SKV_ERR_CAPACITY;
    }
    a.blocks = static_cast<uint32_t>(begin);
    return launch_attn_prompt(a, cfg->dtype, cfg->head_dim, stream) == hipSuccess ? SKV_OK : SKV_ERR_DEVICE;
  });
}

}  // extern "C"
