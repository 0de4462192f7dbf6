// Attention of a batch's newest tokens over the paged cache, a prefix that the
// batch shares read once for all of it.
//
// Every part of the work is a run of rows against a range of token positions:
//   prefix  all B Lq G rows of a KV head (128 per workgroup) against the shared
//           positions, so a key is loaded once per row block and not per request;
//   rest    the Lq G rows of one request against its own positions.
// The prefix is cut into equal parts, the requests' rests into parts of one length
// that the device finds from their lengths; a second launch joins a row's parts.  A
// workgroup turns its range into a list of cache rows in shared memory first (up to
// kList positions at a time): positions past the request's end and DROP tokens are
// left out, so the tiles that follow hold kept tokens only and a dropped token costs
// neither bandwidth nor a product.  The tiles gather the
// listed rows by direct global-to-LDS loads.
//
// What bounds it: reading each kept row of K and V once (4 requests of up to 32768
// tokens of 8 x 128, a fifth dropped: 59 us for 257 MB, 4.3 TB/s with the join, and 52
// where the same input again is partly in cache); for few tokens the latencies in turn
// (one request of 4096 tokens of 4 x 128: 13 us, of them 1.2 to find the part, 1.9 for
// the list, 0.8 for the first tile, 2 for two tiles, 1.2 for the end, 3.5 for the join,
// and the launches); for a prefix
// under many requests its partial results (64 requests behind 16384 tokens, 0.4 of
// them dropped: 31 us and 18 MB of sums, which the join reads in 6.5).
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

// The next positions' pages and tiers: loaded while the tiles before them are
// multiplied, turned into a list afterwards.
template <int THREADS>
struct Upcoming {
  static constexpr int kPer = kList / THREADS;
  int32_t page[kPer];
  uint32_t tier[kPer];
  int first;

  // positions [p0, p1), p1 - p0 <= kList
  __device__ __forceinline__ void load(const DecodeArgs& a, const int32_t* table, const uint8_t* tiers, int p0, int p1) {
    first = p0 + kPer * static_cast<int>(threadIdx.x);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int p = first + i;
      page[i] = 0;
      tier[i] = kDROP;
      if (p >= p1) continue;
      page[i] = table[a.by_block.div(static_cast<uint32_t>(p))];
      tier[i] = kFP16;
      if (tiers != nullptr && p < a.tier_len) tier[i] = tiers[p];
    }
  }
  // Lists the kept positions in order and returns how many; before the call a
  // barrier has ended every use of the previous list.
  __device__ __forceinline__ int list(const DecodeArgs& a, Lists<THREADS>& s) const {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int32_t row[kPer], n = 0;
    bool bad = false;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int p = first + i;
      const bool inside = static_cast<uint32_t>(page[i]) < static_cast<uint32_t>(a.num_blocks);
      bad |= !inside;
      row[i] = -1;
      if (inside && tier[i] != kDROP)
        row[i] = page[i] * a.block_size + (p - static_cast<int>(a.by_block.div(static_cast<uint32_t>(p))) * a.block_size);
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
};

// Rows [row0, row0 + rows) of the launch's B Lq G (row = (request * Lq + query) *
// G + head of the group) against positions [p0, p1) of `table`.  part_row: the
// first row's place in the partial results; -1: results are written at once.
template <class E, int D, Form F>
__device__ __forceinline__ void attend(const DecodeArgs& a, uint8_t* stage, typename WaveAttention<E, D, F>::AreaType& area,
                                       Lists<Stage<D>::kThreads>& lists, int h, int row0, int rows, int tiles,
                                       const int32_t* table, const uint8_t* tiers, int p0, int p1, int64_t part_row) {
  typedef Stage<D> S;
  typedef WaveAttention<E, D, F> Wave;
  Upcoming<S::kThreads> next;
  next.load(a, table, tiers, p0, min(p1, p0 + kList));
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  Wave w;
  w.init(stage, tiles, tiles == 4 ? 1 : 2);
  const bool active = w.rt * 32 < rows;
  const int mine = w.rt * 32 + (lane & 31);
  const uint32_t row = static_cast<uint32_t>(row0 + min(mine, rows - 1));
  const uint32_t token = a.by_G.div(row), g = row - token * a.G;
  const uint32_t b = a.by_Lq.div(token), i = token - b * a.Lq;
  const int head = h * a.G + static_cast<int>(g);
  // (with one row tile most waves only load: without their queries 16 x 256, one
  // request of 1000 tokens: 13.3 -> 12.8 us)
  if (w.multiplies()) w.load_q(a.q + b * a.q_request + i * a.q_token + head * a.q_head);
  const int len = min(max(a.lens[b], 0), a.width * a.block_size);
  const int limit = len - a.Lq + static_cast<int>(i);  // the row's last visible position
  int wave_min = limit;
#pragma unroll
  for (int x = 16; x > 0; x >>= 1) wave_min = min(wave_min, __shfl_xor(wave_min, x));
  wave_min = __builtin_amdgcn_readfirstlane(wave_min);

  const int prow = static_cast<int>(threadIdx.x) / S::kCpr, place = static_cast<int>(threadIdx.x) % S::kCpr;
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane(lds_address(stage) + static_cast<uint32_t>(wave * 1024));
  const int64_t cache_row = static_cast<int64_t>(a.H) * D;
  const uint16_t* kbase = a.k + h * D;
  const uint16_t* vbase = a.v + h * D;
  int first_kept = INT32_MAX;  // position
  walk_tiles(w, area, [&](auto second) {
    if (decltype(second)::value) next.load(a, table, tiers, p0, min(p1, p0 + kList));
    for (int q0 = p0; q0 < p1; q0 += kList) {
      const int q1 = min(p1, q0 + kList);
      const int count = next.list(a, lists);
      if (count > 0) first_kept = min(first_kept, lists.pos[0]);
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
        // (rows of one request are a bandwidth-bound product: two terms cost nothing there)
        w.template tile<decltype(offset)::value, decltype(again)::value>(area, a.alpha, t * S::kKeys, active, tiles < 4,
                                                                          masked, shown);
      };
      if (q1 < p1) next.load(a, table, tiers, q1, min(p1, q1 + kList));
      walk_once<D, decltype(second)::value>(w, 0, nt, issue, tile);
      if (q1 < p1) __syncthreads();  // the next list
    }
  });
  const bool writes = w.finish(stage, area, active);
  if (!writes || mine >= rows) return;
  const bool saw = first_kept <= limit;
  if (part_row < 0) {
    w.write_out(a.out + b * a.out_request + i * a.out_token + head * a.out_head, inverse_sum(w.l, saw));
    if (a.lse != nullptr && w.writes_sum()) a.lse[static_cast<int64_t>(token) * a.H * a.G + head] = log_sum(w.m, w.l);
    return;
  }
  w.write_partial(a.part_o + (part_row + mine) * D);
  if (w.writes_sum()) *reinterpret_cast<floatx2*>(a.part_ml + 2 * (part_row + mine)) = floatx2{w.m, part_sum(w.l, saw)};
}

// Tokens of request b past the prefix.
__device__ __forceinline__ int tail_tokens(const DecodeArgs& a, int b) {
  const int given = a.lens[b], len = min(max(given, 0), a.width * a.block_size);
  if (given != len && a.status != nullptr) *a.status = SKV_ERR_FORMAT;
  return max(len - a.prefix, 0);
}

// Workgroup i of runs x row blocks x heads.  Consecutive workgroups go to the 8 XCDs
// in turn.  A head's row of D = 32 is half a 128-byte line, which two XCDs would both
// fetch: there the runs go fastest, so that the heads of a run share an XCD (32
// requests of 4000 tokens, 8 heads: 35 us against 50).  From D = 64 on the heads go
// fastest (64 x up to 4000 tokens of 8 x 128: 119 us against 123).
struct Place {
  uint32_t run, blk, h;
};
template <int D>
__device__ __forceinline__ Place place(uint32_t i, uint32_t runs, uint32_t blocks, uint32_t H) {
  Place p;
  if constexpr (2 * D < 128) {
    p.run = i % runs;
    i /= runs;
    p.blk = i % blocks;
    p.h = i / blocks;
  } else {
    p.h = i % H;
    i /= H;
    p.blk = i % blocks;
    p.run = i / blocks;
  }
  return p;
}

// Where a tail workgroup's part lies: request, and tokens of its tail.
struct TailPart {
  int request, first, last;
};
__device__ __forceinline__ uint32_t wave_sum(uint32_t x) {
  return static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(wave_inclusive_scan(x)), 63));
}
// Cuts the tails into parts of c tiles, c the smallest (from a.tail_least on) that
// gives at most a.tail_parts parts, and finds part `at`; false past the last.  (With
// N tiles of B requests, c >= N / parts, and c >= N / (parts - B) always gives few
// enough.)  Every wave does it for itself, a lane holding four requests, so nothing
// waits for another wave.  `tell`: write the requests' first parts and counts for
// the join.
__device__ __forceinline__ bool find_part(const DecodeArgs& a, int at, bool tell, TailPart& part) {
  const int lane = threadIdx.x & 63;
  uint32_t tokens[4], n[4], all = 0, most = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    tokens[i] = 4 * lane + i < a.B ? static_cast<uint32_t>(tail_tokens(a, 4 * lane + i)) : 0;
    n[i] = (tokens[i] + 63) / 64;
    all += n[i];
    most = max(most, n[i]);
  }
  all = wave_sum(all);
  most = wave_max(most);
  const uint32_t limit = static_cast<uint32_t>(a.tail_parts);
  uint32_t lo = max(static_cast<uint32_t>(a.tail_least), (all + limit - 1) / limit), hi = max(lo, most);  // (most: one part per request)
  const uint32_t spare = limit - static_cast<uint32_t>(a.B);
  if (spare > 0) hi = min(hi, max(lo, (all + spare - 1) / spare));
  while (lo < hi) {
    const uint32_t c = (lo + hi) >> 1;
    uint32_t parts = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) parts += (n[i] + c - 1) / c;
    if (wave_sum(parts) <= limit) hi = c;
    else lo = c + 1;
  }
  uint32_t mine = 0, count[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    count[i] = (n[i] + lo - 1) / lo;
    mine += count[i];
  }
  uint32_t begin = wave_inclusive_scan(mine) - mine;
  int request = -1;
  uint32_t first = 0, end = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t u = static_cast<uint32_t>(at) - begin;  // (wraps where the part lies before)
    if (u < count[i]) {
      request = 4 * lane + i;
      first = 64 * u * lo;
      end = tokens[i];
    }
    if (tell && 4 * lane + i < a.B) {
      a.first_part[4 * lane + i] = static_cast<int32_t>(begin);
      a.part_count[4 * lane + i] = static_cast<int32_t>(count[i]);
    }
    begin += count[i];
  }
  const uint64_t has = __ballot(request >= 0);
  if (has == 0) return false;
  const int from = __builtin_ctzll(has);
  part.request = __builtin_amdgcn_readlane(request, from);
  part.first = __builtin_amdgcn_readlane(static_cast<int>(first), from);
  part.last = min(part.first + static_cast<int>(64 * lo), __builtin_amdgcn_readlane(static_cast<int>(end), from));
  return true;
}

template <class E, int D>
__global__ __launch_bounds__(Stage<D>::kThreads, Stage<D>::kWavesPerSimd) void attn_decode(const DecodeArgs a) {
  constexpr Form F = D >= 256 ? kPair : kOne;
  __shared__ __align__(1024) uint8_t stage[2 * Stage<D>::kBytes];
  __shared__ typename WaveAttention<E, D, F>::AreaType area;
  __shared__ Lists<Stage<D>::kThreads> lists;
  const uint32_t H = static_cast<uint32_t>(a.H);
  const int own = a.Lq * a.G, rows_all = a.B * own;
  int h, row0, rows, tiles, p0, p1, b = 0;
  int64_t part_row;
  if (blockIdx.x < a.prefix_groups) {
    const Place p = place<D>(blockIdx.x, static_cast<uint32_t>(a.prefix_parts), static_cast<uint32_t>(a.prefix_blocks), H);
    h = static_cast<int>(p.h);
    tiles = a.prefix_tiles;
    row0 = static_cast<int>(p.blk) * tiles * 32;
    rows = min(tiles * 32, rows_all - row0);
    p0 = static_cast<int>(p.run) * a.prefix_chunk;
    p1 = min(a.prefix, p0 + a.prefix_chunk);
    part_row = (static_cast<int64_t>(p.run) * a.H + h) * rows_all + row0;
  } else {
    const uint32_t runs = static_cast<uint32_t>(a.tail_parts == 0 ? a.B : a.tail_parts);
    const Place p = place<D>(blockIdx.x - a.prefix_groups, runs, static_cast<uint32_t>(a.tail_blocks), H);
    h = static_cast<int>(p.h);
    tiles = a.tail_tiles;
    p0 = a.prefix;
    if (a.tail_parts == 0) {
      b = static_cast<int>(p.run);
      p1 = a.prefix + tail_tokens(a, b);
    } else {
      TailPart part;
      if (!find_part(a, static_cast<int>(p.run), blockIdx.x == a.prefix_groups && threadIdx.x < 64, part)) return;
      b = part.request;
      p1 = a.prefix + part.last;
      p0 += part.first;
    }
    row0 = b * own + static_cast<int>(p.blk) * tiles * 32;
    rows = min(tiles * 32, own - static_cast<int>(p.blk) * tiles * 32);
    part_row = a.direct ? -1 : a.tail_at + (static_cast<int64_t>(p.run) * a.H + h) * own + static_cast<int>(p.blk) * tiles * 32;
  }
  const int32_t* table = a.tables + b * a.table_stride;
  const uint8_t* tiers = a.tiers == nullptr ? nullptr : a.tiers + b * a.tier_request + h * a.tier_head;
  attend<E, D, F>(a, stage, area, lists, h, row0, rows, tiles, table, tiers, p0, p1, part_row);
}

// Joins the parts of each row: WAVES waves per (KV head, row).
template <class E, int D, int WAVES>
__global__ __launch_bounds__(256) void attn_decode_join(const DecodeArgs a) {
  __shared__ typename JoinedRow<D, WAVES>::Shared shared;
  const int own = a.Lq * a.G;
  const int64_t rows = static_cast<int64_t>(a.B) * own;
  const int64_t at = (static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6)) / WAVES;  // h * rows + row
  if (at >= rows * a.H) return;
  const int h = static_cast<int>(at / rows);
  const uint32_t row = static_cast<uint32_t>(at - h * rows);
  const uint32_t token = a.by_G.div(row), g = row - token * a.G;
  const uint32_t b = a.by_Lq.div(token), i = token - b * a.Lq;
  JoinedRow<D, WAVES> j;
  j.add(a.part_o, a.part_ml, at, rows * a.H, a.prefix_parts);
  const int64_t stride = static_cast<int64_t>(a.H) * own;
  const int64_t first = a.tail_parts == 0 ? b : a.first_part[b];
  j.add(a.part_o, a.part_ml, a.tail_at + first * stride + static_cast<int64_t>(h) * own + (row - b * own), stride,
        a.tail_parts == 0 ? 1 : a.part_count[b]);
  if (!j.together(shared)) return;
  const int head = h * a.G + static_cast<int>(g);
  j.template write<E>(reinterpret_cast<typename E::elem*>(a.out + b * a.out_request + i * a.out_token + head * a.out_head));
  if (a.lse != nullptr && (threadIdx.x & 63) == 0)
    a.lse[static_cast<int64_t>(token) * a.H * a.G + head] = log_sum(j.m, j.l);
}

template <class E, int D>
hipError_t launch(const DecodeArgs& a, hipStream_t stream) {
  attn_decode<E, D><<<a.groups, Stage<D>::kThreads, 0, stream>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.direct) return e;
  const uint64_t rows = static_cast<uint64_t>(a.B) * a.Lq * a.G * a.H;
  if (rows <= kFewRows) attn_decode_join<E, D, 4><<<static_cast<uint32_t>(rows), 256, 0, stream>>>(a);
  else attn_decode_join<E, D, 1><<<static_cast<uint32_t>((rows + 3) / 4), 256, 0, stream>>>(a);
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
