// Drives the host side of the attention and page calls without a device, under the
// host sanitizers: the HIP launch entry points are replaced here, and what each call
// would launch is checked against what its kernels assume -- grids below 2^32
// threads, every row block and key range of a request covered, parts and lists inside
// the workspace that the size calls ask for -- over small, odd and largest sizes.
#include <stdint.h>
#include <stdio.h>

#include <algorithm>
#include <vector>

#include <hip/hip_runtime.h>

#include "../../paper_2606_08635_amd/csrc/serving/serving_internal.h"

namespace {

struct Launch {
  uint64_t blocks, threads;
  std::vector<uint8_t> arg;  // the first argument
};
std::vector<Launch> launches;
size_t arg_bytes = 0;
hipError_t last = hipSuccess;
int failures = 0, refused = 0, done = 0;

uint64_t state = 88172645463325252ull;
uint64_t next() {
  state ^= state << 13;
  state ^= state >> 7;
  state ^= state << 17;
  return state;
}
// 1..most, spread over its logarithm
int64_t spread(int64_t most) {
  int bits = 0;
  while ((int64_t{1} << bits) <= most) ++bits;
  return std::max<int64_t>(1, std::min<int64_t>(most, static_cast<int64_t>(next() >> (64 - 1 - next() % static_cast<uint64_t>(bits)))));
}
template <class T>
T pick(std::initializer_list<T> of) {
  return *(of.begin() + next() % of.size());
}

#define EXPECT(c)                                                       \
  do {                                                                  \
    if (!(c)) {                                                         \
      if (++failures < 20) printf("%s:%d: %s\n", __func__, __LINE__, #c); \
    }                                                                   \
  } while (0)

uint8_t* const kDev = reinterpret_cast<uint8_t*>(uintptr_t{1} << 40);  // never read on the host
uint8_t* const kWs = reinterpret_cast<uint8_t*>(uintptr_t{1} << 44);

template <class T>
void expect_args() {
  launches.clear();
  arg_bytes = sizeof(T);
}
template <class T>
const T& args_of(const Launch& l) {
  return *reinterpret_cast<const T*>(l.arg.data());
}
bool inside(const void* p, uint64_t bytes, uint64_t size) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(p), w = reinterpret_cast<uintptr_t>(kWs);
  return a >= w && a + bytes <= w + size;
}

void prompt(int32_t d, int32_t H, int32_t G, const std::vector<std::pair<int32_t, int32_t>>& lens, bool causal, int room) {
  skv_attn_config c = {SKV_DTYPE_F16, H * G, H, d, causal, 0.1f, H * G * d, d, H * G * d, d};
  std::vector<skv_attn_request> r;
  for (const auto& n : lens) r.push_back({n.first, n.second, kDev, kDev, kDev, kDev, nullptr, d, int64_t{d} * std::max(1, n.second)});
  uint64_t size = 0;
  EXPECT(skv_attn_prompt_workspace_size(&c, r.data(), static_cast<int32_t>(r.size()), &size) == SKV_OK);
  const uint64_t given = room == 0 ? 0 : room == 1 ? size : size / 2 / 16 * 16;
  expect_args<skv::PromptArgs>();
  const skv_status st = skv_attn_prompt(&c, r.data(), static_cast<int32_t>(r.size()), given ? kWs : nullptr, given, nullptr);
  if (st == SKV_ERR_CAPACITY) {
    EXPECT(launches.empty());
    ++refused;
    return;
  }
  EXPECT(st == SKV_OK);
  size_t at = 0, request = 0;
  while (at < launches.size()) {
    const skv::PromptArgs& a = args_of<skv::PromptArgs>(launches[at]);
    EXPECT(launches[at].blocks == a.blocks && a.count >= 1 && a.count <= skv::kMaxPromptBatch);
    EXPECT(a.row_tiles == 1 || a.row_tiles == 2 || a.row_tiles == 4);
    EXPECT(a.key_streams == 1 ? a.row_tiles == 4 : a.key_streams == 2 && a.row_tiles <= 2);
    uint64_t begin = 0, rows = 0, joins = 0;
    for (int i = 0; i < a.count; ++i, ++request) {
      const skv::PromptDesc& q = a.r[i];
      EXPECT(a.begin[i] == begin && q.nq > 0 && q.splits >= 1);
      EXPECT(static_cast<int64_t>(q.row_blocks) * a.row_tiles * 32 >= static_cast<int64_t>(q.nq) * a.G);
      EXPECT(static_cast<int64_t>(q.row_blocks - 1) * a.row_tiles * 32 < static_cast<int64_t>(q.nq) * a.G);
      begin += static_cast<uint64_t>(q.row_blocks) * a.H * q.splits;
      if (q.splits > 1) {
        EXPECT(q.rows_at == rows);
        rows += static_cast<uint64_t>(q.nq) * a.G * a.H * q.splits;
        ++joins;
      }
    }
    EXPECT(begin == a.blocks);
    for (int i = a.count; i < skv::kMaxPromptBatch; ++i) EXPECT(a.begin[i] == UINT32_MAX);
    if (rows > 0) {
      EXPECT(a.part_o == reinterpret_cast<float*>(kWs) && a.part_ml >= a.part_o + rows * d);
      EXPECT(inside(a.part_ml, 8 * rows, given));
    }
    at += 1 + joins;
  }
  size_t with_queries = 0;
  for (const auto& n : lens) with_queries += n.first > 0;
  EXPECT(request == with_queries && at == launches.size());
  ++done;
}

void decode(int32_t d, int32_t H, int32_t G, int32_t B, int32_t Lq, int32_t block, int32_t width, int32_t max_len, int32_t prefix) {
  const int64_t row = int64_t{H} * G * d;
  skv_decode_config c = {SKV_DTYPE_BF16, B, Lq, H * G, H, d, 1000, block, width, max_len, prefix, 0, 0.1f,
                         row * Lq, row, d, row * Lq, row, d, width, 0, 0};
  uint64_t size = 0;
  const skv_status sizes = skv_attn_decode_workspace_size(&c, &size);
  expect_args<skv::DecodeArgs>();
  int32_t* const ints = reinterpret_cast<int32_t*>(kDev);
  const skv_status st = skv_attn_decode(&c, kDev, kDev, kDev, ints, ints, nullptr, kDev, nullptr, nullptr, kWs, size, nullptr);
  if (sizes != SKV_OK || st != SKV_OK) {
    EXPECT(launches.empty() && (st == SKV_ERR_INVALID_ARG || st == SKV_ERR_CAPACITY) && (sizes == SKV_OK || sizes == st));
    ++refused;
    return;
  }
  ++done;
  if (B == 0 || Lq == 0) {
    EXPECT(launches.empty());
    return;
  }
  EXPECT(launches.size() >= 1);
  const skv::DecodeArgs& a = args_of<skv::DecodeArgs>(launches[0]);
  const int64_t own = int64_t{Lq} * G, all = own * B;
  EXPECT(launches[0].blocks == a.groups && launches.size() == (a.direct ? 1u : 2u));
  EXPECT(a.tail_tiles * 32 * int64_t{a.tail_blocks} >= own && a.tail_tiles * 32 * int64_t{a.tail_blocks - 1} < own);
  if (prefix > 0) {
    EXPECT(a.prefix_chunk % 64 == 0 && int64_t{a.prefix_chunk} * a.prefix_parts >= prefix &&
           int64_t{a.prefix_chunk} * (a.prefix_parts - 1) < prefix);
    EXPECT(a.prefix_tiles * 32 * int64_t{a.prefix_blocks} >= all && a.prefix_tiles * 32 * int64_t{a.prefix_blocks - 1} < all);
  }
  EXPECT(a.prefix_groups == static_cast<uint64_t>(H) * a.prefix_blocks * a.prefix_parts);
  EXPECT(a.tail_parts == 0 || (B <= skv::kCutRequests && a.tail_parts >= B && a.tail_least >= 1));
  const int64_t runs = a.tail_parts > 0 ? a.tail_parts : B;
  EXPECT(a.groups == a.prefix_groups + static_cast<uint64_t>(runs * a.tail_blocks * H));
  if (a.direct) {
    EXPECT(size == 0 && prefix == 0 && a.tail_parts == 0);
    return;
  }
  const uint64_t rows = static_cast<uint64_t>(a.prefix_parts * H * all + runs * H * own);
  EXPECT(a.tail_at == a.prefix_parts * H * all);
  EXPECT(inside(a.part_o, 4 * rows * d, size) && reinterpret_cast<const float*>(a.part_ml) >= a.part_o + rows * d);
  EXPECT(inside(a.part_ml, 8 * rows, size) && reinterpret_cast<float*>(a.first_part) >= a.part_ml + 2 * rows);
  EXPECT(a.part_count >= a.first_part + B && inside(a.part_count, 4u * B, size));
}

void pages(int32_t requests, int32_t children, int32_t blocks, int32_t block, int32_t width, int32_t out_width, int32_t layers,
           int32_t row_bytes) {
  int32_t* const ints = reinterpret_cast<int32_t*>(kDev);
  auto at = [&](uint64_t i) { return ints + (i << 34); };
  const skv_page_pool pool = {layers, blocks, block, row_bytes, kDev, kDev, ints};
  uint32_t* const status = reinterpret_cast<uint32_t*>(kDev);
  for (int op = 0; op < 4; ++op) {
    uint64_t size = 0;
    const int32_t rows = op == 1 ? children : requests;
    const int64_t longest = int64_t{width} * block;
    if (longest > (1 << 30) || skv_pages_workspace_size(rows, blocks, static_cast<int32_t>(longest), &size) != SKV_OK) {
      ++refused;
      continue;
    }
    expect_args<skv::PageArgs>();
    skv_status st = SKV_OK;
    if (op == 0) st = skv_pages_reserve(&pool, at(1), width, at(2), at(3), requests, status, kWs, size, nullptr);
    if (op == 1)
      st = skv_pages_fork(&pool, at(1), width, at(2), requests, at(3), children, at(4), out_width, at(5), status, kWs, size, nullptr);
    if (op == 2)
      st = skv_pages_compact(&pool, at(1), width, at(2), requests, kDev, 100, 100, at(4), out_width, at(5), status, kWs, size, nullptr);
    if (op == 3) st = skv_pages_free(&pool, at(1), width, at(2), requests, status, nullptr);
    if (st != SKV_OK) {
      EXPECT(launches.empty());
      ++refused;
      continue;
    }
    ++done;
    EXPECT(!launches.empty());
    if (op == 3) continue;  // no workspace; its first launch may be the status's alone
    for (const Launch& l : launches) {
      const skv::PageArgs& a = args_of<skv::PageArgs>(l);
      const uint64_t r = 4u * static_cast<uint64_t>(rows), c = r * static_cast<uint64_t>(op == 2 ? a.chunks : 0);
      EXPECT(a.rows == rows && a.sources == requests);
      const int32_t* const lists[] = {a.ws_bad, a.ws_off, a.ws_need, a.ws_shared, a.ws_total, a.ws_list, a.ws_kept, a.ws_first};
      const uint64_t bytes[] = {r, r, r, r, r, 4u * static_cast<uint64_t>(blocks), c, c};
      EXPECT(inside(a.ws_status, 4, size));
      const uint8_t* end = kWs + 4;
      for (int i = 0; i < 8; ++i) {
        EXPECT(inside(lists[i], bytes[i], size) && reinterpret_cast<const uint8_t*>(lists[i]) >= end);
        end = reinterpret_cast<const uint8_t*>(lists[i]) + bytes[i];
      }
      EXPECT(op != 2 || int64_t{a.chunks} * 256 >= longest);
    }
  }
  const skv_page_pool other = {layers, blocks / 2 + 1, block, row_bytes, kDev, kDev, ints};
  expect_args<skv::PageCopyArgs>();
  const skv_status st = skv_pages_copy(&pool, &other, ints, ints, children, status, nullptr);
  EXPECT(st == SKV_OK ? !launches.empty() : launches.empty());
}

}  // namespace

extern "C" hipError_t hipLaunchKernel(const void*, dim3 grid, dim3 block, void** args, size_t, hipStream_t) {
  const uint64_t threads = static_cast<uint64_t>(grid.x) * block.x;
  if (threads >= 1ull << 32 || grid.x == 0) {
    ++failures;
    printf("a grid of %u x %u threads\n", grid.x, block.x);
  }
  Launch l{grid.x, block.x, {}};
  // (the status alone: one pointer)
  if (grid.x > 1 || block.x > 1) l.arg.assign(static_cast<uint8_t*>(args[0]), static_cast<uint8_t*>(args[0]) + arg_bytes);
  launches.push_back(std::move(l));
  return last = hipSuccess;
}
static dim3 cfg_grid, cfg_block;
extern "C" hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t, hipStream_t) {
  cfg_grid = grid;
  cfg_block = block;
  return hipSuccess;
}
extern "C" hipError_t __hipPopCallConfiguration(dim3* grid, dim3* block, size_t* shared, hipStream_t* stream) {
  *grid = cfg_grid;
  *block = cfg_block;
  *shared = 0;
  *stream = nullptr;
  return hipSuccess;
}
extern "C" hipError_t hipGetLastError() { return last; }

int main() {
  for (int i = 0; i < 20000; ++i) {
    const int32_t d = pick({32, 64, 128, 256}), H = static_cast<int32_t>(spread(64)), G = static_cast<int32_t>(spread(16));
    std::vector<std::pair<int32_t, int32_t>> lens;
    const int64_t count = i % 50 ? spread(60) - 1 : 150;
    for (int64_t j = 0; j < count; ++j)
      lens.emplace_back(static_cast<int32_t>(spread(1 << (i % 21)) - 1), static_cast<int32_t>(spread(1 << 20) - 1));
    prompt(d, H, G, lens, next() & 1, static_cast<int>(next() % 3));
    const int32_t block = static_cast<int32_t>(spread(300)), width = static_cast<int32_t>(spread(4000)) - 1;
    const int32_t prefix = pick({0, 0, static_cast<int32_t>(spread(width + 1) - 1) * block});
    decode(d, H, G, static_cast<int32_t>(spread(2000) - 1), static_cast<int32_t>(spread(100) - 1), block, width,
           static_cast<int32_t>(spread(1 << 24) - 1), prefix);
    pages(static_cast<int32_t>(spread(3000) - 1), static_cast<int32_t>(spread(3000) - 1), static_cast<int32_t>(spread(1 << 20)), block,
          width, static_cast<int32_t>(spread(4000)) - 1, static_cast<int32_t>(spread(128)), 16 * static_cast<int32_t>(spread(512)));
  }
  // the largest of everything
  for (int32_t d : {32, 64, 128, 256}) {
    prompt(d, 1, 1, {{1 << 28, 1 << 30}}, true, 1);
    prompt(d, 65536, 1, {{4096, 1 << 30}, {1, 5}}, false, 1);
    prompt(d, 1, 65536, {{1 << 14, 7}}, true, 1);
    prompt(d, 1, 2, {{(1 << 28) + 1, 3}}, true, 1);
    for (int32_t B : {1, 255, 256, 257, 1 << 20})
      for (int32_t prefix : {0, 1 << 29, 1 << 30}) {
        decode(d, 1, 1, B, 1, 1, 1 << 30, INT32_MAX, prefix);
        decode(d, 1, 63, B, 1, 1 << 15, 1 << 15, INT32_MAX, prefix);
        decode(d, 8, 8, B, 2, 16, 1 << 26, 1 << 30, prefix);
        decode(d, 1, 65536, B, 1, 16, 1 << 26, 1 << 30, prefix);
        decode(d, 65536, 1, B, 1, 16, 1 << 26, 1 << 30, prefix);
        decode(d, 1, 1020, ((1 << 26) - 4) / 1020, 1, 16, 100, 1600, 16);
      }
  }
  pages(1 << 24, 1 << 21, 1 << 20, 1, 0, 1, 65536, 1 << 24);
  pages(1 << 20, 1 << 20, INT32_MAX, 1, 1024, 1024, 1, 16);
  pages(1, 1, INT32_MAX, 1, 1 << 30, 1 << 30, 1, 16);
  pages(1, 1, 1, 1 << 30, 1, 1, 1, 16);
  pages(1, INT32_MAX, 1 << 10, 16, 1 << 26, 1, 65536, 16);
  if (failures) {
    printf("%d failures\n", failures);
    return 1;
  }
  printf("ok %d calls, %d refused\n", done, refused);
  return 0;
}
