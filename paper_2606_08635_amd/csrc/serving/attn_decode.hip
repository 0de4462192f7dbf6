// Attention of a batch's newest tokens over the paged cache, a prefix that the
// batch shares read once for all of it.
//
// Every part of the work is a run of rows against a range of token positions:
//   prefix  all B Lq G rows of a KV head (128 per workgroup) against the shared
//           positions, so a key is loaded once per row block and not per request;
//   rest    the Lq G rows of one request against its own positions.
// Ranges are cut into parts that fill the GPU; a second launch joins a row's
// parts.  A workgroup turns its range into a list of cache rows in shared memory
// first (up to kList positions at a time): positions past the request's end and
// DROP tokens are left out, so the tiles that follow hold kept tokens only and a
// dropped token costs neither bandwidth nor a product.  The tiles gather the
// listed rows by direct global-to-LDS loads.
#include "attn_core.h"
#include "serving_internal.h"

namespace skv {
namespace {

constexpr int kList = 1024;  // positions listed at a time

template <int THREADS>
struct Lists {
  int32_t rows[kList];  // row of the cache: page * block_size + slot
  int32_t pos[kList];   // token position; past the list's end, to the end of its last tile, one that nothing sees
  uint32_t scan[THREADS / 64];
};

// The kept positions of [p0, p1), p1 - p0 <= kList, in order.  The caller's
// barrier before the call has ended every use of the previous list.
template <int THREADS>
__device__ __forceinline__ int build_list(const DecodeArgs& a, Lists<THREADS>& s, const int32_t* table, const uint8_t* tier,
                                          int p0, int p1) {
  constexpr int kPer = kList / THREADS;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int32_t row[kPer], n = 0;
  const int first = p0 + kPer * static_cast<int>(threadIdx.x);
  bool bad = false;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int p = first + i;
    row[i] = -1;
    if (p >= p1) continue;
    const int at = static_cast<int>(a.by_block.div(static_cast<uint32_t>(p)));
    const int page = table[at];
    const bool kept = tier == nullptr || p >= a.tier_len || tier[p] != kDROP;
    if (static_cast<uint32_t>(page) >= static_cast<uint32_t>(a.num_blocks)) bad = true;
    else if (kept) row[i] = page * a.block_size + (p - at * a.block_size);
    n += row[i] >= 0;
  }
  if (bad && a.status != nullptr) *a.status = SKV_ERR_FORMAT;
  const uint32_t inc = wave_inclusive_scan(static_cast<uint32_t>(n));
  if (lane == 63) s.scan[wave] = inc;
  __syncthreads();
  int to = static_cast<int>(inc) - n, count = 0;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) {
    if (w < wave) to += static_cast<int>(s.scan[w]);
    count += static_cast<int>(s.scan[w]);
  }
#pragma unroll
  for (int i = 0; i < kPer; ++i)
    if (row[i] >= 0) {
      s.rows[to] = row[i];
      s.pos[to] = first + i;
      ++to;
    }
  const int past = count + static_cast<int>(threadIdx.x);
  if (past < (count + 63) / 64 * 64) s.pos[past] = INT32_MAX;
  __syncthreads();
  return __builtin_amdgcn_readfirstlane(count);
}

// Rows [row0, row0 + rows) of the launch's B Lq G (row = (request * Lq + query) *
// G + head of the group) against positions [p0, p1) of `table`.
template <class E, int D, Form F>
__device__ __forceinline__ void attend(const DecodeArgs& a, uint8_t* stage, typename WaveAttention<E, D, F>::AreaType& area,
                                       Lists<Stage<D>::kThreads>& lists, int h, int row0, int rows, int tiles, const int32_t* table,
                                       const uint8_t* tier, int p0, int p1, int part, bool only) {
  typedef Stage<D> S;
  typedef WaveAttention<E, D, F> Wave;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  Wave w;
  w.init(stage, tiles, tiles == 4 ? 1 : 2);
  const bool active = w.rt * 32 < rows;
  const int mine = w.rt * 32 + (lane & 31);
  const uint32_t row = static_cast<uint32_t>(row0 + min(mine, rows - 1));
  const uint32_t token = a.by_G.div(row), g = row - token * a.G;
  const uint32_t b = a.by_Lq.div(token), i = token - b * a.Lq;
  const int head = h * a.G + static_cast<int>(g);
  const int len = min(max(a.lens[b], 0), a.width * a.block_size);
  const int limit = len - a.Lq + static_cast<int>(i);  // the row's last visible position
  int wave_min = limit;
#pragma unroll
  for (int x = 16; x > 0; x >>= 1) wave_min = min(wave_min, __shfl_xor(wave_min, x));
  wave_min = __builtin_amdgcn_readfirstlane(wave_min);

  w.load_q(a.q + b * a.q_request + i * a.q_token + head * a.q_head);
  const int prow = static_cast<int>(threadIdx.x) / S::kCpr, place = static_cast<int>(threadIdx.x) % S::kCpr;
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane(lds_address(stage) + static_cast<uint32_t>(wave * 1024));
  const int64_t cache_row = static_cast<int64_t>(a.H) * D;
  const uint16_t* kbase = a.k + h * D;
  const uint16_t* vbase = a.v + h * D;
  walk_tiles(w, area, [&](auto second) {
    for (int q0 = p0; q0 < p1; q0 += kList) {
      const int q1 = min(p1, q0 + kList);
      const int count = build_list(a, lists, table, tier, q0, q1);
      const int nt = (count + S::kKeys - 1) / S::kKeys;
      const bool cut = q1 - 1 > wave_min;  // some row ends before the list does
      auto issue = [&](int t, int buffer) {
#pragma unroll
        for (int u = 0; u < S::kPieces; ++u) {
          const int rr = prow + u * S::kRowStep;
          // rows past the list's end repeat its last one: hidden from every row
          const int64_t off = lists.rows[min(t * S::kKeys + rr, count - 1)] * cache_row + 8 * (place ^ S::swz(rr));
          const uint32_t to = lds0 + static_cast<uint32_t>(buffer * S::kBytes + u * S::kThreads * 16);
          direct_load(kbase + off, to);
          direct_load(vbase + off, to + S::kHalf);
        }
      };
      auto masked = [&](int key, int keys) {
        if (key + keys > count) return true;
        return cut && __builtin_amdgcn_readfirstlane(lists.pos[key + keys - 1]) > wave_min;
      };
      auto shown = [&](int key) { return lists.pos[key] <= limit; };
      auto tile = [&](int t, auto offset, auto again) {
        w.template tile<decltype(offset)::value, decltype(again)::value>(area, a.alpha, t * S::kKeys, active, true, masked,
                                                                          shown);
      };
      walk_once<D, decltype(second)::value>(w, 0, nt, issue, tile);
      if (q1 < p1) __syncthreads();  // the next list
    }
  });
  const bool writes = w.finish(stage, area, active);
  if (!writes || mine >= rows) return;
  if (only) {
    w.write_out(a.out + b * a.out_request + i * a.out_token + head * a.out_head, inverse_or_zero(w.l));
    if (a.lse != nullptr && w.writes_sum()) a.lse[static_cast<int64_t>(token) * a.H * a.G + head] = log_sum(w.m, w.l);
    return;
  }
  const int64_t at = (static_cast<int64_t>(part) * a.H + h) * (static_cast<int64_t>(a.B) * a.Lq * a.G) + row;
  if (p0 < p1) w.write_partial(a.part_o + at * D);
  if (w.writes_sum()) *reinterpret_cast<floatx2*>(a.part_ml + 2 * at) = floatx2{w.m, w.l};
}

template <class E, int D>
__global__ __launch_bounds__(Stage<D>::kThreads, Stage<D>::kWavesPerSimd) void attn_decode(const DecodeArgs a) {
  constexpr Form F = D >= 256 ? kPair : kOne;
  __shared__ __align__(1024) uint8_t stage[2 * Stage<D>::kBytes];
  __shared__ typename WaveAttention<E, D, F>::AreaType area;
  __shared__ Lists<Stage<D>::kThreads> lists;
  uint32_t at = blockIdx.x;
  const uint32_t H = static_cast<uint32_t>(a.H);
  int h, row0, rows, tiles, p0, p1, part;
  const int32_t* table;
  const uint8_t* tier;
  if (at < a.prefix_groups) {
    h = static_cast<int>(at % H);
    at /= H;
    const int blk = static_cast<int>(at % static_cast<uint32_t>(a.prefix_blocks));
    part = static_cast<int>(at / static_cast<uint32_t>(a.prefix_blocks));
    tiles = a.prefix_tiles;
    row0 = blk * tiles * 32;
    rows = min(tiles * 32, a.B * a.Lq * a.G - row0);
    p0 = part * a.prefix_chunk;
    p1 = min(a.prefix, p0 + a.prefix_chunk);
    table = a.tables;
    tier = a.tiers == nullptr ? nullptr : a.tiers + h * a.tier_head;
  } else {
    at -= a.prefix_groups;
    h = static_cast<int>(at % H);
    at /= H;
    const int blk = static_cast<int>(at % static_cast<uint32_t>(a.tail_blocks));
    at /= static_cast<uint32_t>(a.tail_blocks);
    part = static_cast<int>(at % static_cast<uint32_t>(a.tail_parts));
    const int b = static_cast<int>(at / static_cast<uint32_t>(a.tail_parts));
    tiles = a.tail_tiles;
    row0 = b * a.Lq * a.G + blk * tiles * 32;
    rows = min(tiles * 32, a.Lq * a.G - blk * tiles * 32);
    const int given = a.lens[b], most = a.width * a.block_size, len = min(max(given, 0), most);
    if (given != len && a.status != nullptr) *a.status = SKV_ERR_FORMAT;
    // whole tiles to each part
    const int n = max(len - a.prefix, 0), tilesn = (n + 63) / 64, chunk = (tilesn + a.tail_parts - 1) / a.tail_parts * 64;
    p0 = a.prefix + min(n, part * chunk);
    p1 = a.prefix + min(n, part * chunk + chunk);
    part += a.prefix_parts;
    table = a.tables + b * a.table_stride;
    tier = a.tiers == nullptr ? nullptr : a.tiers + b * a.tier_request + h * a.tier_head;
  }
  const bool only = a.prefix_parts + a.tail_parts == 1;
  attend<E, D, F>(a, stage, area, lists, h, row0, rows, tiles, table, tier, p0, p1, part, only);
}

// Joins the parts of each row: one wave per (KV head, row).
template <class E, int D>
__global__ __launch_bounds__(256) void attn_decode_join(const DecodeArgs a) {
  const int64_t rows = static_cast<int64_t>(a.B) * a.Lq * a.G;
  const int64_t at = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6);  // h * rows + row
  if (at >= rows * a.H) return;
  const JoinedRow<D> j(a.part_o, a.part_ml, at, rows * a.H, a.prefix_parts + a.tail_parts);
  const int h = static_cast<int>(at / rows);
  const uint32_t row = static_cast<uint32_t>(at - h * rows);
  const uint32_t token = a.by_G.div(row), g = row - token * a.G;
  const uint32_t b = a.by_Lq.div(token), i = token - b * a.Lq;
  const int head = h * a.G + static_cast<int>(g);
  j.template write<E>(reinterpret_cast<typename E::elem*>(a.out + b * a.out_request + i * a.out_token + head * a.out_head));
  if (a.lse != nullptr && (threadIdx.x & 63) == 0)
    a.lse[static_cast<int64_t>(token) * a.H * a.G + head] = log_sum(j.m, j.l);
}

template <class E, int D>
hipError_t launch(const DecodeArgs& a, hipStream_t stream) {
  attn_decode<E, D><<<a.groups, Stage<D>::kThreads, 0, stream>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.prefix_parts + a.tail_parts == 1) return e;
  const uint64_t rows = static_cast<uint64_t>(a.B) * a.Lq * a.G * a.H;
  attn_decode_join<E, D><<<static_cast<uint32_t>((rows + 3) / 4), 256, 0, stream>>>(a);
  return hipGetLastError();
}

template <class E>
hipError_t launch_d(const DecodeArgs& a, int32_t d, hipStream_t stream) {
  switch (d) {
    case 32: return launch<E, 32>(a, stream);
    case 64: return launch<E, 64>(a, stream);
    case 128: return launch<E, 128>(a, stream);
    default: return launch<E, 256>(a, stream);
  }
}

}  // namespace

hipError_t launch_attn_decode(const DecodeArgs& a, int32_t dtype, int32_t d, hipStream_t stream) {
  return dtype == SKV_DTYPE_F16 ? launch_d<TypeF16>(a, d, stream) : launch_d<TypeBF16>(a, d, stream);
}

}  // namespace skv
