// Pages of the cache: allocation by reference counts, forks, compaction, copies.
//
// refs[p] counts the block tables that hold page p; p is free when it is 0.  New
// pages are the lowest free ones, in (request, page) order, so results do not
// depend on the order in which anything runs.  Each call is
//   pages_check    (fork with large tables, compact) entries of the source tables
//                  looked over by the whole GPU; compact: kept tokens per chunk
//   pages_plan     one workgroup: what each request needs, prefix sums, whether
//                  the pool has it, the free pages, the status
//   pages_apply    tables and counts written and rows copied, unless the status
//                  says otherwise: a refused call changes nothing but the status
// Rows are copied in every layer of K and V; that traffic bounds fork, compact
// and copy (2 x row bytes x rows x 2 L), so a workgroup keeps 8 16-byte loads per
// thread in flight and the planes (a layer of K or of V) are spread over
// workgroups until the launch fills the GPU.  4 requests of up to 16384 tokens of 32
// x 8 x 128, two fifths dropped, compacted: 1.24 ms for 3.0 GB read and 3.0 written,
// 4.9 TB/s (5.0 in pages_apply); 1 GiB copied to another pool: 0.43 ms, 5.0 TB/s (a
// large copy of the library's: 4.8-4.9).  Small calls are launches: the plan 3-6 us,
// the copies of 8 forks' last pages 6 us, a release 3-4 us.
#include <algorithm>

#include "../device_util.h"
#include "serving_internal.h"

namespace skv {
namespace {

constexpr int kPlanThreads = 1024;
constexpr int kPlanWaves = kPlanThreads / 64;
constexpr int kChunk = 256;  // tokens of a chunk of compact: a wave's, 4 per lane

__device__ __forceinline__ int pages_of(int tokens, const Divider& by_block, int block_size) {
  return static_cast<int>(by_block.div(static_cast<uint32_t>(tokens + block_size - 1)));
}
__device__ __forceinline__ bool held(const PageArgs& a, int page) {
  return static_cast<uint32_t>(page) < static_cast<uint32_t>(a.num_blocks) && a.refs[page] > 0;
}
__device__ __forceinline__ bool length_ok(const PageArgs& a, int n) { return n >= 0 && n <= a.width * a.block_size; }

// The source request of output row c.
__device__ __forceinline__ int source_of(const PageArgs& a, int c) { return a.parents == nullptr ? c : a.parents[c]; }

// grid: fork, one workgroup per child; compact, one per 1024 tokens of a request.
__global__ __launch_bounds__(256) void pages_check(const PageArgs a) {
  if (a.op == kPagesFork) {
    const int c = blockIdx.x, src = source_of(a, c);
    bool bad = static_cast<uint32_t>(src) >= static_cast<uint32_t>(a.sources);
    if (!bad) {
      const int n = a.lens[src];
      bad = !length_ok(a, n);
      const int pages = bad ? 0 : pages_of(n, a.by_block, a.block_size);
      for (int j = threadIdx.x; j < pages; j += 256) bad |= !held(a, a.tables[static_cast<int64_t>(src) * a.width + j]);
    }
    const int any = __syncthreads_or(bad);
    if (threadIdx.x == 0) a.ws_bad[c] = any;
    return;
  }
  const int groups = (a.chunks + 3) / 4;
  const int b = blockIdx.x / groups, chunk = blockIdx.x % groups * 4 + static_cast<int>(threadIdx.x >> 6);
  if (chunk >= a.chunks) return;
  const int lane = threadIdx.x & 63;
  const int n = a.lens[b];
  int kept = 0, first = INT32_MAX;
  bool bad = !length_ok(a, n);
  if (!bad) {
    const uint8_t* tier = a.tiers + static_cast<int64_t>(b) * a.tier_stride;
    const int32_t* table = a.tables + static_cast<int64_t>(b) * a.width;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int t = chunk * kChunk + 4 * lane + i;
      if (t >= n) break;
      const int j = static_cast<int>(a.by_block.div(static_cast<uint32_t>(t)));
      if (j * a.block_size == t || i == 0) bad |= !held(a, table[j]);
      if (t >= a.tier_len || tier[t] != kDROP) ++kept;
      else first = min(first, t);
    }
  }
#pragma unroll
  for (int x = 32; x > 0; x >>= 1) {
    kept += __shfl_xor(kept, x);
    first = min(first, __shfl_xor(first, x));
  }
  if (__any(bad)) kept = -1;
  if (lane == 0) {
    a.ws_kept[static_cast<int64_t>(b) * a.chunks + chunk] = kept;
    a.ws_first[static_cast<int64_t>(b) * a.chunks + chunk] = first;
  }
}

struct PlanShared {
  uint32_t sums[4][kPlanWaves];
  int32_t bad, total;
};

// Exclusive prefix sum over the workgroup; *all: the sum.  Ends with a barrier.
__device__ __forceinline__ uint32_t plan_scan(uint32_t x, uint32_t (&sums)[kPlanWaves], uint32_t* all) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const uint32_t inc = wave_inclusive_scan(x);
  if (lane == 63) sums[wave] = inc;
  __syncthreads();
  uint32_t base = 0, total = 0;
#pragma unroll
  for (int w = 0; w < kPlanWaves; ++w) {
    if (w < wave) base += sums[w];
    total += sums[w];
  }
  *all = total;
  __syncthreads();
  return base + inc - x;
}

// One workgroup.  ws_off[c], ws_shared[c]: where row c's new pages begin in the
// list of free ones, and how many pages of its source it shares.
__global__ __launch_bounds__(kPlanThreads) void pages_plan(const PageArgs a) {
  __shared__ PlanShared s;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (tid == 0) s.bad = 0;
  __syncthreads();
  uint32_t bad = 0;  // 1: a bad entry; 2: a table too narrow
  if (a.op == kPagesCompact) {
    // a wave per request: kept tokens before each chunk, the first dropped token
    for (int b = wave; b < a.rows; b += kPlanWaves) {
      int kept = 0, first = INT32_MAX;
      for (int c0 = 0; c0 < a.chunks; c0 += 64) {
        const int64_t at = static_cast<int64_t>(b) * a.chunks + c0 + lane;
        const bool in = c0 + lane < a.chunks;
        int k = in ? a.ws_kept[at] : 0;
        if (k < 0) bad |= 1, k = 0;
        if (in) first = min(first, a.ws_first[at]);
        const uint32_t inc = wave_inclusive_scan(static_cast<uint32_t>(k));
        if (in) a.ws_kept[at] = kept + static_cast<int>(inc) - k;
        kept += __shfl(static_cast<int>(inc), 63);
      }
#pragma unroll
      for (int x = 32; x > 0; x >>= 1) first = min(first, __shfl_xor(first, x));
      const int n = a.lens[b];
      if (lane == 0) {
        a.ws_shared[b] = static_cast<int>(a.by_block.div(static_cast<uint32_t>(max(0, min(first, n)))));
        a.ws_total[b] = kept;
      }
    }
  } else if (a.op == kPagesFork && a.checked) {
    for (int c = tid; c < a.rows; c += kPlanThreads) bad |= a.ws_bad[c] != 0;
  } else if (a.op == kPagesFork) {  // small tables: looked over here
    const uint32_t entries = static_cast<uint32_t>(a.rows) * static_cast<uint32_t>(max(1, a.width));
#pragma unroll 4
    for (uint32_t e = tid; e < entries; e += kPlanThreads) {
      const uint32_t c = a.by_width.div(e), j = e - c * static_cast<uint32_t>(max(1, a.width));
      const int src = source_of(a, static_cast<int>(c));
      const bool there = static_cast<uint32_t>(src) < static_cast<uint32_t>(a.sources);
      const int n = there ? a.lens[src] : -1;
      if (!length_ok(a, n)) bad |= 1;
      else if (j < static_cast<uint32_t>(pages_of(n, a.by_block, a.block_size))) bad |= !held(a, a.tables[static_cast<int64_t>(src) * a.width + j]);
    }
  } else {
    for (int c = tid; c < a.rows; c += kPlanThreads) bad |= !length_ok(a, a.lens[c]) || !length_ok(a, a.new_lens[c]);
  }
  if (bad) atomicOr(&s.bad, static_cast<int>(bad));
  __syncthreads();
  const bool sound = s.bad == 0;
  __syncthreads();  // every wave has read it before one sets it again below
  uint32_t total = 0;
  bool too_many = false;
  if (sound) {
    for (int c0 = 0; c0 < a.rows; c0 += kPlanThreads) {
      const int c = c0 + tid;
      int need = 0;
      if (c < a.rows) {
        if (a.op == kPagesReserve) {
          const int old = pages_of(a.lens[c], a.by_block, a.block_size);
          need = max(0, pages_of(a.new_lens[c], a.by_block, a.block_size) - old);
          a.ws_shared[c] = old;
        } else {
          const int n = a.op == kPagesFork ? a.lens[source_of(a, c)] : a.ws_total[c];
          const int shared = a.op == kPagesFork ? static_cast<int>(a.by_block.div(static_cast<uint32_t>(n))) : a.ws_shared[c];
          const int pages = pages_of(n, a.by_block, a.block_size);
          if (pages > a.out_width) atomicOr(&s.bad, 2);
          a.ws_shared[c] = shared;
          a.ws_total[c] = n;
          need = pages - shared;
        }
      }
      uint32_t all;
      const uint32_t off = plan_scan(static_cast<uint32_t>(need), s.sums[0], &all);
      if (c < a.rows) {
        a.ws_off[c] = static_cast<int32_t>(total + off);
        a.ws_need[c] = need;
      }
      // one chunk of rows adds less than 2^31: no overflow before this is seen
      if (total + all > static_cast<uint32_t>(a.num_blocks)) {
        too_many = true;
        break;
      }
      total += all;
    }
  }
  // the lowest `total` free pages: 16 counts per thread at a time, pages in (i, thread, j) order
  uint32_t found = 0;
  const bool fits = s.bad == 0 && !too_many;
  if (fits && total > 0) {
    for (int p0 = 0; p0 < a.num_blocks && found < total; p0 += 16 * kPlanThreads) {
      u32x4 r[4];
      uint32_t mine[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int p = p0 + i * 4 * kPlanThreads + 4 * tid;
        r[i] = u32x4{1, 1, 1, 1};
        if (p + 3 < a.num_blocks) r[i] = *reinterpret_cast<const u32x4*>(a.refs + p);
        else
          for (int j = 0; j < 4; ++j)
            if (p + j < a.num_blocks) r[i][j] = static_cast<uint32_t>(a.refs[p + j]);
      }
      uint32_t inc[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        mine[i] = (r[i].x == 0) + (r[i].y == 0) + (r[i].z == 0) + (r[i].w == 0);
        inc[i] = wave_inclusive_scan(mine[i]);
        if (lane == 63) s.sums[i][wave] = inc[i];
      }
      __syncthreads();
      uint32_t before = found;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t at = before + inc[i] - mine[i];
#pragma unroll
        for (int w = 0; w < kPlanWaves; ++w) {
          if (w < wave) at += s.sums[i][w];
          before += s.sums[i][w];
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (r[i][j] == 0) {
            if (at < total) a.ws_list[at] = p0 + i * 4 * kPlanThreads + 4 * tid + j;
            ++at;
          }
      }
      found = before;
      __syncthreads();
    }
  }
  uint32_t status = SKV_OK;
  if (s.bad & 1) status = SKV_ERR_FORMAT;
  else if ((s.bad & 2) || too_many || found < total) status = SKV_ERR_CAPACITY;
  if (tid == 0) *a.ws_status = *a.status = status;
  if (status != SKV_OK) return;
  if (a.op == kPagesReserve) {  // few entries: written here (the list is this workgroup's own: a barrier orders it)
    __syncthreads();
    for (int c = wave; c < a.rows; c += kPlanWaves) {
      const int need = a.ws_need[c], off = a.ws_off[c], old = a.ws_shared[c];
      for (int j = lane; j < need; j += 64) {
        const int page = a.ws_list[off + j];
        a.out_tables[static_cast<int64_t>(c) * a.out_width + old + j] = page;
        a.refs[page] = 1;
      }
    }
    return;
  }
  for (int c = tid; c < a.rows; c += kPlanThreads) a.out_lens[c] = a.ws_total[c];
}

struct RowList {
  int64_t src[kChunk], dst[kChunk];  // byte offsets in a plane
  uint32_t scan[4];
  int32_t count;
};

// Copies rows list.src -> list.dst in planes [plane0, plane1): thread units of 16
// bytes, eight in flight.
__device__ __forceinline__ void copy_rows(const PageArgs& a, const RowList& list, int count, int plane0, int plane1) {
  const uint32_t units = static_cast<uint32_t>(a.row_bytes >> 4), all = units * static_cast<uint32_t>(count);
  for (int plane = plane0; plane < plane1; ++plane) {
    uint8_t* base = (plane & 1 ? a.v : a.k) + static_cast<int64_t>(plane >> 1) * a.plane_bytes;
    for (uint32_t u0 = threadIdx.x; u0 < all; u0 += 8 * 256) {
      u32x4 x[8];
      int64_t to[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t u = u0 + 256 * i;
        if (u >= all) continue;
        const uint32_t row = a.by_units.div(u), part = (u - row * units) << 4;
        to[i] = list.dst[row] + part;
        x[i] = ld_nt16(base + list.src[row] + part);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (u0 + 256 * i < all) st_nt16(base + to[i], x[i]);
    }
  }
}

// grid: the row copies (output row, chunk, planes), then the table entries (1024
// per workgroup).
__global__ __launch_bounds__(256) void pages_apply(const PageArgs a) {
  __shared__ RowList list;
  if (*a.ws_status != SKV_OK) return;
  uint32_t at = blockIdx.x;
  if (at >= a.copy_groups) {
    const int64_t e0 = static_cast<int64_t>(at - a.copy_groups) * 1024 + threadIdx.x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t e = e0 + 256 * i;
      if (e >= static_cast<int64_t>(a.rows) * a.out_width) break;
      const int c = static_cast<int>(e / a.out_width), j = static_cast<int>(e % a.out_width);
      const int shared = a.ws_shared[c];
      if (j < shared) {
        const int page = a.tables[static_cast<int64_t>(source_of(a, c)) * a.width + j];
        a.out_tables[e] = page;
        atomicAdd(a.refs + page, 1);
      } else if (j < shared + a.ws_need[c]) {
        const int page = a.ws_list[a.ws_off[c] + j - shared];
        a.out_tables[e] = page;
        a.refs[page] = 1;
      }
    }
    return;
  }
  const int group = static_cast<int>(at % static_cast<uint32_t>(a.plane_groups));
  at /= static_cast<uint32_t>(a.plane_groups);
  const int chunk = static_cast<int>(at % static_cast<uint32_t>(a.chunks)), c = static_cast<int>(at / static_cast<uint32_t>(a.chunks));
  const int planes = 2 * a.num_layers;
  const int plane0 = static_cast<int>(static_cast<int64_t>(planes) * group / a.plane_groups);
  const int plane1 = static_cast<int>(static_cast<int64_t>(planes) * (group + 1) / a.plane_groups);
  const int src = source_of(a, c), n = a.lens[src], shared = a.ws_shared[c];
  const int begin = shared * a.block_size;  // tokens before it stay where they are
  const int32_t* table = a.tables + static_cast<int64_t>(src) * a.width;
  const int32_t* pages = a.ws_list + a.ws_off[c];
  // fork: the tokens of the last, partly filled page, all of them kept; compact: the chunk
  const bool fork = a.op == kPagesFork;
  const int t0 = fork ? begin : chunk * kChunk, t1 = fork ? n : min(n, t0 + kChunk);
  if (t1 <= begin) return;
  const uint8_t* tier = fork ? nullptr : a.tiers + static_cast<int64_t>(c) * a.tier_stride;
  for (int q0 = t0; q0 < t1; q0 += kChunk) {
    if (q0 > t0) __syncthreads();
    const int t = q0 + static_cast<int>(threadIdx.x);
    const bool kept = t < t1 && (tier == nullptr || t >= a.tier_len || tier[t] != kDROP);
    const uint32_t before = block_exclusive_scan_256(kept, list.scan);
    const int to = fork ? t : a.ws_kept[static_cast<int64_t>(c) * a.chunks + chunk] + static_cast<int>(before);
    // rows of shared pages keep their places; in a chunk they come first
    const bool moves = kept && to >= begin;
    const uint32_t skip = static_cast<uint32_t>(max(0, min(begin, t1) - q0));
    if (moves) {
      const int j = static_cast<int>(a.by_block.div(static_cast<uint32_t>(t))), k = static_cast<int>(a.by_block.div(static_cast<uint32_t>(to)));
      const uint32_t slot = before - skip;
      list.src[slot] = (static_cast<int64_t>(table[j]) * a.block_size + (t - j * a.block_size)) * a.row_bytes;
      list.dst[slot] = (static_cast<int64_t>(pages[k - shared]) * a.block_size + (to - k * a.block_size)) * a.row_bytes;
    }
    if (threadIdx.x == 255) list.count = static_cast<int>(before + kept) - static_cast<int>(skip);
    __syncthreads();
    copy_rows(a, list, list.count, plane0, plane1);
  }
}

// Releases tables: every page's count goes down by one for each entry that holds
// it.  An entry out of range, or one more than the count has, is passed over.
// alone: the launch is this workgroup, which clears the status itself.  Four
// entries of a thread are in flight together.
__global__ __launch_bounds__(kPlanThreads) void pages_free(const PageArgs a, int alone) {
  if (alone) {
    if (threadIdx.x == 0) *a.status = SKV_OK;
    __syncthreads();
  }
  const uint32_t width = static_cast<uint32_t>(max(1, a.width));  // (with none the lengths are still looked at)
  const uint32_t all = static_cast<uint32_t>(a.rows) * width, step = gridDim.x * kPlanThreads;
  bool bad = false;
  for (uint64_t e0 = blockIdx.x * kPlanThreads + threadIdx.x; e0 < all; e0 += 4 * static_cast<uint64_t>(step)) {
    int n[4], page[4];
    uint32_t j[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint64_t e = e0 + static_cast<uint64_t>(i) * step;
      n[i] = 0;
      if (e >= all) continue;
      const uint32_t b = a.by_width.div(static_cast<uint32_t>(e));
      j[i] = static_cast<uint32_t>(e) - b * width;
      n[i] = a.lens[b];
      page[i] = a.width > 0 ? a.tables[e] : -1;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (!length_ok(a, n[i])) {
        bad = true;
      } else if (n[i] > 0 && j[i] < static_cast<uint32_t>(pages_of(n[i], a.by_block, a.block_size))) {
        if (static_cast<uint32_t>(page[i]) >= static_cast<uint32_t>(a.num_blocks)) {
          bad = true;
        } else if (atomicSub(a.refs + page[i], 1) <= 0) {
          atomicAdd(a.refs + page[i], 1);
          bad = true;
        }
      }
    }
  }
  if (bad) *a.status = SKV_ERR_FORMAT;
}

__global__ void pages_clear_status(uint32_t* status) { *status = SKV_OK; }

// One workgroup: whether every pair of a copy lies in its pool.
__global__ __launch_bounds__(kPlanThreads) void pages_copy_check(const PageCopyArgs a) {
  bool bad = false;
  for (int i = threadIdx.x; i < a.count; i += kPlanThreads)
    bad |= static_cast<uint32_t>(a.src_pages[i]) >= static_cast<uint32_t>(a.src_blocks) ||
           static_cast<uint32_t>(a.dst_pages[i]) >= static_cast<uint32_t>(a.dst_blocks);
  const int any = __syncthreads_or(bad);
  if (threadIdx.x == 0) *a.status = any ? SKV_ERR_FORMAT : SKV_OK;
}

// Units of work: (pair, plane, 32 KB piece of a page); a workgroup copies four, one
// after the other, eight 16-byte loads per thread in flight.
constexpr int kPiece = 32768, kUnits = 4;
__global__ __launch_bounds__(256) void pages_copy(const PageCopyArgs a, uint32_t first) {
  if (*a.status != SKV_OK) return;
  const uint64_t u0 = static_cast<uint64_t>(first + blockIdx.x) * kUnits;
  for (uint64_t unit = u0; unit < min(u0 + kUnits, a.units); ++unit) {
    const uint32_t at = static_cast<uint32_t>(unit / a.pieces), piece = static_cast<uint32_t>(unit % a.pieces);
    const uint32_t plane = at % a.planes, pair = at / a.planes;
    const int32_t src_page = a.src_pages[pair], dst_page = a.dst_pages[pair];
    // (checked: passed over here only where the status was written by another call meanwhile)
    if (static_cast<uint32_t>(src_page) >= static_cast<uint32_t>(a.src_blocks) ||
        static_cast<uint32_t>(dst_page) >= static_cast<uint32_t>(a.dst_blocks))
      continue;
    const int64_t from = static_cast<int64_t>(plane >> 1) * a.src_plane_bytes + src_page * a.page_bytes;
    const int64_t to = static_cast<int64_t>(plane >> 1) * a.dst_plane_bytes + dst_page * a.page_bytes;
    const uint8_t* src = (plane & 1 ? a.src_v : a.src_k) + from;
    uint8_t* dst = (plane & 1 ? a.dst_v : a.dst_k) + to;
    const int64_t end = min(a.page_bytes, static_cast<int64_t>(piece + 1) * kPiece);
    const int64_t b0 = static_cast<int64_t>(piece) * kPiece + 16 * static_cast<int>(threadIdx.x);
    u32x4 x[kPiece / 4096];
#pragma unroll
    for (int i = 0; i < kPiece / 4096; ++i)
      if (b0 + 4096 * i < end) x[i] = ld_nt16(src + b0 + 4096 * i);
#pragma unroll
    for (int i = 0; i < kPiece / 4096; ++i)
      if (b0 + 4096 * i < end) st_nt16(dst + b0 + 4096 * i, x[i]);
  }
}

}  // namespace

hipError_t launch_pages(const PageArgs& a, hipStream_t stream) {
  hipError_t e = hipSuccess;
  if (a.op == kPagesCompact && a.rows > 0) {
    pages_check<<<static_cast<uint32_t>(a.rows) * static_cast<uint32_t>((a.chunks + 3) / 4), 256, 0, stream>>>(a);
    e = hipGetLastError();
  } else if (a.op == kPagesFork && a.checked) {
    pages_check<<<static_cast<uint32_t>(a.rows), 256, 0, stream>>>(a);
    e = hipGetLastError();
  }
  if (e != hipSuccess) return e;
  pages_plan<<<1, kPlanThreads, 0, stream>>>(a);
  if ((e = hipGetLastError()) != hipSuccess || a.op == kPagesReserve) return e;
  const uint64_t entries = (static_cast<uint64_t>(a.rows) * a.out_width + 1023) / 1024;
  if (a.rows == 0) return hipSuccess;
  pages_apply<<<static_cast<uint32_t>(a.copy_groups + entries), 256, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_pages_free(const PageArgs& a, hipStream_t stream) {
  // one workgroup clears the status itself (2000 entries: 3 us); more need it cleared
  // before any of them starts
  const uint64_t all = static_cast<uint64_t>(a.rows) * std::max(1, a.width);
  const uint32_t groups = all <= 8 * kPlanThreads ? 1 : static_cast<uint32_t>(std::min<uint64_t>((all + 4095) / 4096, 256));
  if (groups > 1) {
    pages_clear_status<<<1, 1, 0, stream>>>(a.status);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  pages_free<<<groups, kPlanThreads, 0, stream>>>(a, groups == 1);
  return hipGetLastError();
}

hipError_t launch_pages_copy(PageCopyArgs a, hipStream_t stream) {
  a.pieces = static_cast<uint32_t>((a.page_bytes + kPiece - 1) / kPiece);
  a.units = static_cast<uint64_t>(a.count) * a.planes * a.pieces;
  pages_copy_check<<<1, kPlanThreads, 0, stream>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  return launch_pieces((a.units + kUnits - 1) / kUnits, 256,
                       [&](uint32_t first, uint32_t blocks) { pages_copy<<<blocks, 256, 0, stream>>>(a, first); });
}

}  // namespace skv
