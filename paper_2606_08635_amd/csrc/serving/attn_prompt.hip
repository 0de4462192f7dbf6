// Attention over whole prompts: packed sequences, grouped heads, causal or not.
//
// A workgroup owns up to 128 packed rows (attn_core.h) of one (request, KV head)
// and walks the keys that any of them sees in tiles of 64, staged through two
// shared-memory buffers by direct global-to-LDS loads: the next tile is in
// flight while the current one is multiplied, and one barrier per tile orders
// both.  Tiles past a wave's last visible key are skipped, and only tiles that a
// row's limit cuts compare indexes.
//
// Order of the workgroups: KV heads fastest, so that consecutive workgroups --
// which the hardware deals to the 8 XCDs in turn -- read different heads and an
// XCD's L2 holds few of them; then the row blocks from the last to the first,
// since the last ones see the most keys and the launch ends with short ones.
//
// What bounds it: 4 d floating-point operations per (head, query, visible key) on the
// matrix units.  8189 causal tokens of 32 x 128 on 8 KV heads, binary16: 520-560 us by
// device, 980-1060 TFLOP/s of the visible products (a large matrix product: 1140);
// the matrix units are busy 64 % of the cycles at the clock that power then allows,
// no bank conflicts.  8192 of 16 x 256, bfloat16: 550-595 us, 920-1000 TFLOP/s.
// Staging moves 32 KB (64 KB at D = 256) per 64 keys and workgroup, out of L2: 8
// heads on 8 XCDs fetch 0.16 GB of K, V and Q from memory.  Two workgroups of four
// waves share a compute unit (237 registers, 65 KB): while one waits for a tile or
// exponentiates the other multiplies.  Short sequences pay 5-6 us per workgroup for
// its first loads and its end (24 of up to 2300 tokens: 460-475 us, 820-840 TFLOP/s).
#include "attn_core.h"
#include "serving_internal.h"

namespace skv {
namespace {

template <class E, int D, Form F>
__global__ __launch_bounds__(Stage<D>::kThreads, Stage<D>::kWavesPerSimd) void attn_prompt(const PromptArgs a) {
  typedef Stage<D> S;
  typedef WaveAttention<E, D, F> Wave;
  __shared__ __align__(1024) uint8_t stage[2 * S::kBytes];
  __shared__ typename Wave::AreaType area;
  const uint32_t block = blockIdx.x;
  // The last request that begins at or before this workgroup, by two loads of scalars
  // in turn; a search by halves waits for up to six (24 prompts of up to 2300 tokens:
  // 467 us against 465).
  int ri = 0;
  if (a.count > 1) {
#pragma unroll
    for (int i = 8; i < kMaxPromptBatch; i += 8) ri += a.begin[i] <= block ? 8 : 0;
    const uint32_t* eight = a.begin + ri;
#pragma unroll
    for (int i = 1; i < 8; ++i) ri += eight[i] <= block;
  }
  const PromptDesc& r = a.r[ri];
  const int rows = r.nq * a.G, per = a.row_tiles * 32;
  uint32_t at = block - a.begin[ri];
  const uint32_t of_head = a.by_H.div(at);
  const int h = static_cast<int>(at - of_head * static_cast<uint32_t>(a.H));
  at = of_head;
  int split = 0;
  if (r.splits > 1) {
    split = static_cast<int>(at % static_cast<uint32_t>(r.splits));
    at /= static_cast<uint32_t>(r.splits);
  }
  const int blk = r.row_blocks - 1 - static_cast<int>(at);

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  Wave w;
  w.init(stage, a.row_tiles, a.key_streams);
  const int row0 = blk * per + w.rt * 32;  // the wave's first row
  const bool active = row0 < rows;
  const int row = min(row0 + (lane & 31), rows - 1);
  const int token = static_cast<int>(a.by_G.div(static_cast<uint32_t>(row))), head = h * a.G + row - token * a.G;
  const int more = r.nk - r.nq;
  const int limit = a.causal ? token + more : r.nk - 1;  // the row's last visible key
  const int wave_min = __builtin_amdgcn_readfirstlane(limit);
  auto last_seen = [&](int to) {  // by rows up to `to`
    return a.causal ? static_cast<int>(a.by_G.div(static_cast<uint32_t>(min(to, rows - 1)))) + more : r.nk - 1;
  };
  const int wave_max = last_seen(row0 + 31), block_max = last_seen(blk * per + per - 1);
  const int all = block_max < 0 ? 0 : block_max / S::kKeys + 1;  // tiles that some row sees
  int t0 = 0, t1 = all;
  if (r.splits > 1) {
    t0 = static_cast<int>(static_cast<int64_t>(all) * split / r.splits);
    t1 = static_cast<int>(static_cast<int64_t>(all) * (split + 1) / r.splits);
  }

  w.load_q(r.q + token * a.q_token + head * a.q_head);

  // this thread's pieces of a stage: row tid / kCpr + u * kRowStep, place tid % kCpr
  const int prow = static_cast<int>(threadIdx.x) / S::kCpr, place = static_cast<int>(threadIdx.x) % S::kCpr;
  const uint16_t* kbase = r.k + h * r.kv_head;
  const uint16_t* vbase = r.v + h * r.kv_head;
  const uint32_t token_bytes = static_cast<uint32_t>(r.kv_token * 2);
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane(lds_address(stage) + static_cast<uint32_t>(wave * 1024));
  auto issue = [&](int t, int buffer) {
    const int64_t first = static_cast<int64_t>(t) * S::kKeys * r.kv_token;
    const int last = r.nk - 1 - t * S::kKeys;  // rows past it repeat the last key: hidden from every row
#pragma unroll
    for (int u = 0; u < S::kPieces; ++u) {
      const int rr = prow + u * S::kRowStep;
      const uint32_t off = static_cast<uint32_t>(min(rr, last)) * token_bytes +
                           16u * static_cast<uint32_t>(place ^ S::swz(rr));
      const uint32_t to = lds0 + static_cast<uint32_t>(buffer * S::kBytes + u * S::kThreads * 16);
      direct_load(kbase + first, off, to);
      direct_load(vbase + first, off, to + S::kHalf);
    }
  };
  auto tile = [&](int t, auto offset, auto second) {
    const int key0 = t * S::kKeys;
    w.template tile<decltype(offset)::value, decltype(second)::value>(
        area, a.alpha, key0, active && key0 <= wave_max, false, [&](int key, int keys) { return key + keys - 1 > wave_min; },
        [&](int key) { return key <= limit; });
  };
  walk_tiles(w, area, [&](auto second) { walk_once<D, decltype(second)::value>(w, t0, t1, issue, tile); });
  const bool writes = w.finish(stage, area, active);
  if (!writes || row0 + (lane & 31) >= rows) return;  // (both lane-halves of a row stay: write_out pairs them)
  const bool saw = t0 < t1 && t0 * S::kKeys <= limit;
  if (r.splits > 1) {
    const int64_t prow_at = r.rows_at + (static_cast<int64_t>(split) * a.H + h) * rows + row;
    w.write_partial(a.part_o + prow_at * D);
    if (w.writes_sum()) *reinterpret_cast<floatx2*>(a.part_ml + 2 * prow_at) = floatx2{w.m, part_sum(w.l, saw)};
    return;
  }
  w.write_out(r.out + token * a.out_token + head * a.out_head, inverse_sum(w.l, saw));
  if (r.lse != nullptr && w.writes_sum()) r.lse[static_cast<int64_t>(token) * a.H * a.G + head] = log_sum(w.m, w.l);
}

// Joins the parts of a request with splits > 1: WAVES waves per row.
template <class E, int D, int WAVES>
__global__ __launch_bounds__(256) void attn_prompt_join(const PromptArgs a, int ri) {
  __shared__ typename JoinedRow<D, WAVES>::Shared shared;
  const PromptDesc& r = a.r[ri];
  const int rows = r.nq * a.G;
  const int64_t at = (static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6)) / WAVES;  // h * rows + row
  if (at >= static_cast<int64_t>(rows) * a.H) return;
  const int h = static_cast<int>(at / rows), row = static_cast<int>(at % rows);
  JoinedRow<D, WAVES> j;
  j.add(a.part_o, a.part_ml, r.rows_at + at, static_cast<int64_t>(rows) * a.H, r.splits);
  if (!j.together(shared)) return;
  const int token = row / a.G, head = h * a.G + row % a.G;
  j.template write<E>(reinterpret_cast<typename E::elem*>(r.out + token * a.out_token + head * a.out_head));
  if (r.lse != nullptr && (threadIdx.x & 63) == 0)
    r.lse[static_cast<int64_t>(token) * a.H * a.G + head] = log_sum(j.m, j.l);
}

template <class E, int D>
hipError_t launch(const PromptArgs& a, hipStream_t stream) {
  if constexpr (D >= 256) attn_prompt<E, D, kPair><<<a.blocks, Stage<D>::kThreads, 0, stream>>>(a);
  else if (a.key_streams == 1) attn_prompt<E, D, kBoth><<<a.blocks, Stage<D>::kThreads, 0, stream>>>(a);
  else attn_prompt<E, D, kOne><<<a.blocks, Stage<D>::kThreads, 0, stream>>>(a);
  hipError_t e = hipGetLastError();
  for (int i = 0; i < a.count && e == hipSuccess; ++i) {
    if (a.r[i].splits <= 1) continue;
    const uint64_t rows = static_cast<uint64_t>(a.r[i].nq) * a.G * a.H;
    if (rows <= kFewRows) attn_prompt_join<E, D, 4><<<static_cast<uint32_t>(rows), 256, 0, stream>>>(a, i);
    else attn_prompt_join<E, D, 1><<<static_cast<uint32_t>((rows + 3) / 4), 256, 0, stream>>>(a, i);
    e = hipGetLastError();
  }
  return e;
}

template <class E>
hipError_t launch_d(const PromptArgs& a, int32_t d, hipStream_t stream) {
  switch (d) {
    case 32: return launch<E, 32>(a, stream);
    case 64: return launch<E, 64>(a, stream);
    case 128: return launch<E, 128>(a, stream);
    default: return launch<E, 256>(a, stream);
  }
}

}  // namespace

hipError_t launch_attn_prompt(const PromptArgs& a, int32_t dtype, int32_t d, hipStream_t stream) {
  return dtype == SKV_DTYPE_F16 ? launch_d<TypeF16>(a, d, stream) : launch_d<TypeBF16>(a, d, stream);
}

}  // namespace skv
