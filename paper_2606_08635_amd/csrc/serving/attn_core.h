// What the attention kernels share: one wave's online softmax(Q K^T) V over
// key tiles that its workgroup stages through shared memory.
//
// For a query q with visible keys t the kernels compute
//   z_t = alpha q.k_t (alpha = scale log2 e),  m = max z_t,
//   l = sum 2^(z_t - m),  o = (1/l) sum 2^(z_t - m) v_t,  lse = (m + log2 l) ln 2
// in one pass over the keys.  Both products run on v_mfma_f32_32x32x16 with
// binary32 accumulation.  The logits are formed transposed (keys as MFMA rows,
// queries as columns), so a lane holds 16 keys of one query per 32-key tile,
// keeps that query's m and l in registers, and its exponentials are already
// the second product's B operand (o^T = V^T P^T): no value crosses lanes
// between the two products.  V is read from its row-major stage by gfx950's
// transposing LDS reads (ds_read_b64_tr_b16).
//
// Rows are packed: the G = Hq / H query heads that share a KV head are rows of
// one product (row r is token r / G, head h G + r % G), so K and V of a head are
// staged once for all of them, and one token per request still gives G rows.
//
// Roundings: products exact, sums, m, l and o in binary32; the probabilities are
// rounded (nearest even) to the inputs' 16-bit type for the second product -- the
// MFMA takes both operands in one type -- while l sums them unrounded; the result
// is rounded once to the output type.  A row that sees few keys would show that
// rounding (over many it averages out), so where it costs little -- tiles that a
// row's limit cuts, among them every row's last and so all of a short one's, and the
// steps of small and of bandwidth-bound calls -- what the rounding left over is
// rounded too and multiplied as a second term.
#pragma once

#include <type_traits>

#include "../device_util.h"

namespace skv {

typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef short shortx4 __attribute__((ext_vector_type(4)));

constexpr float kRoom = 16.0f;  // log2 of the parts of a row whose sums are added without overflow

struct TypeF16 {
  typedef _Float16 elem;
  typedef _Float16 vec8 __attribute__((ext_vector_type(8)));
  typedef _Float16 vec2 __attribute__((ext_vector_type(2)));
  static constexpr uint16_t kInf = 0x7C00, kOne = 0x3C00;
  static constexpr float kTop = 8.0f;  // log2 of a row's largest probability when its reference is set
  static constexpr bool kWide = false;  // whether sums of V times unnormalized probabilities can pass binary32
  __device__ static __forceinline__ floatx16 mfma(vec8 a, vec8 b, floatx16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
  }
};
struct TypeBF16 {
  typedef __bf16 elem;
  typedef __bf16 vec8 __attribute__((ext_vector_type(8)));
  typedef __bf16 vec2 __attribute__((ext_vector_type(2)));
  static constexpr uint16_t kInf = 0x7F80, kOne = 0x3F80;
  static constexpr float kTop = 0.0f;
  static constexpr bool kWide = true;
  __device__ static __forceinline__ floatx16 mfma(vec8 a, vec8 b, floatx16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
};

// Two binary32 values rounded (nearest even) to E and packed low | high.
template <class E>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  const floatx2 f = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, typename E::vec2));
}

// Row of accumulator register r in lane-half hf of a 32x32 MFMA result (the
// column is lane % 32).
__device__ __forceinline__ int mfma_row(int r, int hf) { return 8 * (r >> 2) + 4 * hf + (r & 3); }

__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const uint8_t*)p));
}

// Direct global-to-LDS load: lane i's 16 bytes at src land at LDS byte address
// lds_base + 16 i.  From inline assembly, so that the compiler does not count it
// among its own loads; the tile loop waits for it itself (wait_direct_loads).  A
// load that reads m0 needs one wait state behind the write of it: the s_nop.  (m0 on
// the clobber list tells the compiler that its own value is gone; it warns that it
// would not save one, and it keeps none there across statements.)
__device__ __forceinline__ void direct_load(const void* src, uint32_t lds_base) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(src), "s"(lds_base) : "memory", "m0");
}
__device__ __forceinline__ void direct_load(const void* uniform_base, uint32_t offset, uint32_t lds_base) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(offset), "s"(uniform_base), "s"(lds_base)
               : "memory", "m0");
}
__device__ __forceinline__ void wait_direct_loads() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// Workgroup barrier that waits for this wave's shared-memory accesses but not
// for its global loads in flight.
__device__ __forceinline__ void stage_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// Shared-memory stage of kKeys keys: K rows, then V rows, each row D 16-bit
// values as kCpr chunks of 16 bytes, chunk c of row r at place c ^ swz(r).  The
// swizzle makes two access patterns free of bank conflicts at once: the first
// product reads one chunk of 16 consecutive rows (swz takes each value once over
// the rows that share 256 bytes of banks), the second reads 64 consecutive bytes
// of 4 consecutive rows (swz differs in the bits that select the 64-byte group).
template <int D>
struct Stage {
  static constexpr int kWaves = D >= 256 ? 8 : 4;
  static constexpr int kThreads = kWaves * 64;
  static constexpr int kKeys = 64;
  static constexpr int kCpr = D / 8;
  static constexpr int kPitch = D * 2;
  static constexpr int kHalf = kKeys * kPitch;  // bytes of K, and of V
  static constexpr int kBytes = 2 * kHalf;
  static constexpr int kPieces = kKeys * kCpr / kThreads;  // 16-byte loads of K per thread, and of V
  static constexpr int kRowStep = kThreads / kCpr;         // rows between a thread's pieces
  static constexpr int kWavesPerSimd = 2;                  // 256 registers each
  static_assert(kKeys * kCpr % kThreads == 0, "whole pieces per thread");
  __device__ static constexpr int swz(int r) {
    return D >= 128 ? ((r & 3) << 2) | ((r >> 2) & 3) : D == 64 ? (((r >> 1) & 1) << 2) | ((r >> 2) & 3) : (r >> 2) & 3;
  }
};

// How a workgroup's waves share a stage of two 32-key tiles.
enum Form {
  kBoth,  // a wave has 32 rows to itself and takes both tiles in one step
  kOne,   // a tile per step: both in turn, or with two key streams one each of two
          // waves with the same rows, whose results are added at the end
  kPair   // D = 256, where o and Q of 32 rows would not fit a wave's registers: two
          // waves share 32 rows, each forms the logits of one tile, they exchange
          // their probabilities through shared memory, and each sums half of V's
          // channels over both tiles
};

// Shared memory besides the stage.
struct Area {
  int32_t not_finite;  // whether a wave's result asks for the second walk (walk_tiles)
};
// kPair: probabilities [row tile][key tile][step][lane] (second terms two row tiles
// on: with more than two row tiles there are none), rows' maxima and sums, whether
// a wave's sum asks for a higher reference.
struct PairArea : Area {
  u32x4 p[4][2][2][64];
  float top[4][2][32];
  float l[4][2][32];
  alignas(16) uint32_t raise[8];
};
template <Form F>
struct AreaOf {
  typedef skv::Area type;
};
template <>
struct AreaOf<kPair> {
  typedef PairArea type;
};

// One wave's 32 query rows: state and arithmetic.
template <class E, int D, Form F>
struct WaveAttention {
  typedef typename E::vec8 vec8;
  typedef typename AreaOf<F>::type AreaType;
  typedef Stage<D> S;
  static constexpr int kChannels = F == kPair ? D / 2 : D;  // of o, in this wave
  static constexpr int kSteps = D / 16;                     // MFMA steps of a logit
  static constexpr int kTiles = kChannels / 32;             // 32-channel tiles of o
  static constexpr int NS = F == kBoth ? 2 : 1;             // 32-key tiles of a step's logits
  static constexpr int kReads = kSteps < 8 ? kSteps : 8;    // distinct LDS addresses of a K row's chunks
  // A step is exponentiated against the current reference m first, without its
  // maximum; only where that gives a sum past kHigh (or a NaN: m still -inf) is
  // the maximum taken, m raised and o rescaled.  2^15 keeps every probability
  // inside binary16.  m is some earlier step's maximum less E::kTop, so the largest
  // probability of the sum so far is at least 2^kTop.  What rounds to 0 for the second
  // product is added to l all the same, so many such keys would be missing from o
  // alone: binary16 ends at 2^-25, and with kTop = 8 that is 2^-33 of the largest
  // (2^20 keys just below it are 2^-13 of the result, under half a step of its type),
  // with room for 32 keys at the maximum and for references 2^2 to 2^7 too low.
  // bfloat16 ends far below either way and leaves the room to V.
  static constexpr float kHigh = 32768.0f;
  static constexpr uint16_t kInf = E::kInf, kOne1 = E::kOne;
  static constexpr int kAhead = 4;  // operands read ahead of their products

  vec8 q[kSteps];
  floatx16 o[kTiles];
  float m, l;
  uint32_t kaddr[kReads];  // LDS addresses in the first stage buffer
  uint32_t vaddr[kTiles][2];
  int tiles;               // row tiles of the workgroup
  int rt, ks, streams;     // row tile, place among the waves that share its rows, how many do

  // row_tiles: 32-row tiles of the workgroup; key_streams: of kOne
  __device__ __forceinline__ void init(const void* stage, int row_tiles, int key_streams) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = threadIdx.x & 63, hf = lane >> 5, j = lane & 31, i = lane & 15, g = (lane >> 4) & 1;
    tiles = row_tiles;
    rt = wave % tiles;
    ks = wave / tiles;
    streams = F == kPair ? 2 : F == kOne ? key_streams : 1;
    const uint32_t base = lds_address(stage);
    const uint32_t own = F == kPair ? base + static_cast<uint32_t>((ks & 1) * 32 * S::kPitch) : base;
#pragma unroll
    for (int s = 0; s < kReads; ++s) {
      kaddr[s] = own + static_cast<uint32_t>(j * S::kPitch + 16 * ((2 * s + hf) ^ S::swz(j)));
      asm volatile("" : "+v"(kaddr[s]));  // one register each: tile offsets become immediates
    }
    const int half = F == kPair ? (ks & 1) * 16 : 0;  // first chunk of this wave's channels
#pragma unroll
    for (int dt = 0; dt < kTiles; ++dt)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int row = 8 * u + 4 * hf + (i >> 2);
        const int chunk = half + 4 * dt + 2 * g + ((i & 3) >> 1);
        vaddr[dt][u] =
            base + static_cast<uint32_t>(S::kHalf + row * S::kPitch + 16 * (chunk ^ S::swz(row)) + 8 * (i & 1));
        asm volatile("" : "+v"(vaddr[dt][u]));
      }
    reset();
  }

  // Moves on to the other stage buffer where steps do not name it (D = 256: its
  // offset is past the 16 bits of an LDS instruction).
  __device__ __forceinline__ void move(int bytes) {
#pragma unroll
    for (int s = 0; s < kReads; ++s) kaddr[s] += bytes;
#pragma unroll
    for (int dt = 0; dt < kTiles; ++dt)
#pragma unroll
      for (int u = 0; u < 2; ++u) vaddr[dt][u] += bytes;
  }

  // Whether this wave multiplies (the others load tiles only).
  __device__ __forceinline__ bool multiplies() const { return ks < streams; }
  __device__ __forceinline__ void load_q(const void* row) {
    const uint8_t* p = static_cast<const uint8_t*>(row) + 16 * ((threadIdx.x >> 5) & 1);
#pragma unroll
    for (int s = 0; s < kSteps; ++s) q[s] = __builtin_bit_cast(vec8, *reinterpret_cast<const u32x4*>(p + 32 * s));
  }
  // Waits for Q (and every other load) before the tile loop.  The compiler's own wait
  // would sit in the loop, where it would also wait for the direct loads that it does
  // not know of.
  __device__ __forceinline__ void wait_q() {
    __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0)
#pragma unroll
    for (int s = 0; s < kSteps; ++s) asm volatile("" : "+v"(q[s]));
  }

  __device__ static __forceinline__ u32x4 lds16(uint32_t addr) {
    typedef __attribute__((address_space(3))) const u32x4* ptr;
    return *reinterpret_cast<ptr>(static_cast<uintptr_t>(addr));
  }
  // channels 32 dt + lane % 32 (of this wave's) of the 8 keys 16 s + {4 hf .. + 3, 8 + 4 hf .. + 3}
  template <int OFF>
  __device__ __forceinline__ u32x4 v_operand(int dt, int s) const {
    typedef __attribute__((address_space(3))) shortx4* ptr;
    u32x4 a;
    const uint32_t off = static_cast<uint32_t>(OFF + 16 * s * S::kPitch);
    const u32x2 lo = __builtin_bit_cast(
        u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<ptr>(static_cast<uintptr_t>(vaddr[dt][0] + off))));
    const u32x2 hi = __builtin_bit_cast(
        u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<ptr>(static_cast<uintptr_t>(vaddr[dt][1] + off))));
    a.x = lo.x;
    a.y = lo.y;
    a.z = hi.x;
    a.w = hi.y;
    return a;
  }

  __device__ __forceinline__ void rescale(float f) {
    l *= f;
#pragma unroll
    for (int dt = 0; dt < kTiles; ++dt)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[dt][r] *= f;
  }

  // x = K Q^T of N 32-key tiles at byte offset OFF of the stage.
  template <int OFF, int N>
  __device__ __forceinline__ void logits(floatx16 (&x)[N]) const {
#pragma unroll
    for (int n = 0; n < N; ++n) x[n] = floatx16{};
    constexpr int kAll = N * kSteps;
    u32x4 a[kAhead + 1];
#pragma unroll
    for (int i = 0; i < kAll + kAhead; ++i) {
      if (i < kAll) {
        const int s = i / N, n = i % N;
        a[i % (kAhead + 1)] = lds16(kaddr[s % kReads] + static_cast<uint32_t>(OFF + n * 32 * S::kPitch + s / kReads * 256));
      }
      if (i >= kAhead) {
        const int c = i - kAhead;
        x[c % N] = E::mfma(__builtin_bit_cast(vec8, a[c % (kAhead + 1)]), q[c / N], x[c % N]);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  }

  // e = 2^(alpha x - ref); returns the lane's sum.
  template <int N>
  __device__ __forceinline__ float exponentials(const floatx16 (&x)[N], float alpha, float ref, float (&e)[N][16]) const {
    float sum = 0.0f;
#pragma unroll
    for (int n = 0; n < N; ++n) {
#pragma unroll
      for (int r = 0; r < 16; ++r) e[n][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[n][r], alpha, -ref));
      float t[8];
#pragma unroll
      for (int r = 0; r < 8; ++r) t[r] = e[n][r] + e[n][r + 8];
      sum += ((t[0] + t[1]) + (t[2] + t[3])) + ((t[4] + t[5]) + (t[6] + t[7]));
    }
    return sum;
  }
  // The reference that puts the row's largest logit at 2^kTop (both lane-halves get it).
  template <int N>
  __device__ __forceinline__ float largest(const floatx16 (&x)[N], float alpha) const {
    float top = -INFINITY;
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int r = 0; r < 16; ++r) top = fmaxf(top, x[n][r]);
    const LanePair p = lane_pair32(__builtin_bit_cast(uint32_t, top * alpha));
    return fmaxf(__builtin_bit_cast(float, p.lo), __builtin_bit_cast(float, p.hi)) - E::kTop;
  }
  // Whether no row has a reference yet: the first step takes the maximum at once.
  __device__ __forceinline__ bool fresh() const { return __all(m == -INFINITY); }
  // Raises m to mn >= m; returns the value to exponentiate against (0 while nothing
  // has been seen, so that every probability is 0).
  __device__ __forceinline__ float raise(float mn) {
    const float ref = mn == -INFINITY ? 0.0f : mn;
    rescale(__builtin_amdgcn_exp2f(m - ref));
    m = mn;
    return ref;
  }
  // Probabilities as second-product operands, rounded to E.
  template <int N>
  __device__ static __forceinline__ void pack(const float (&e)[N][16], u32x4 (&p)[2 * N]) {
#pragma unroll
    for (int s = 0; s < 2 * N; ++s)
#pragma unroll
      for (int i = 0; i < 4; ++i) p[s][i] = pack2<E>(e[s >> 1][8 * (s & 1) + 2 * i], e[s >> 1][8 * (s & 1) + 2 * i + 1]);
  }
  // What that rounding left over, rounded to E.
  template <int N>
  __device__ static __forceinline__ void pack_rest(const float (&e)[N][16], const u32x4 (&p)[2 * N], u32x4 (&rest)[2 * N]) {
#pragma unroll
    for (int s = 0; s < 2 * N; ++s)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t both = p[s][i];  // (a bit cast of a vector's element itself would take the first)
        const floatx2 f = __builtin_convertvector(__builtin_bit_cast(typename E::vec2, both), floatx2);
        rest[s][i] = pack2<E>(e[s >> 1][8 * (s & 1) + 2 * i] - f.x, e[s >> 1][8 * (s & 1) + 2 * i + 1] - f.y);
      }
  }

  __device__ __forceinline__ void reset() {
#pragma unroll
    for (int dt = 0; dt < kTiles; ++dt) o[dt] = floatx16{};
    m = -INFINITY;
    l = 0.0f;
  }
  // Before a second walk.  Where V's type reaches as far as binary32, a sum of
  // unnormalized probabilities times V can overflow although the average is finite;
  // the first walk's m and l are the row's log-sum, and against 2^kRoom times that the
  // probabilities add up to 2^-kRoom: no sum of theirs, and none of up to 2^kRoom
  // parts', passes V's largest.
  __device__ __forceinline__ void again(AreaType& area) {
    float ref = -INFINITY;
    if constexpr (E::kWide) {
      const LanePair p = lane_pair32(__builtin_bit_cast(uint32_t, l));
      float sum = __builtin_bit_cast(float, p.lo) + __builtin_bit_cast(float, p.hi);
      if constexpr (F == kPair) {
        const int lane = threadIdx.x & 31;
        if (ks < 2) area.l[rt][ks][lane] = sum;
        stage_barrier();
        if (ks < 2) sum = area.l[rt][0][lane] + area.l[rt][1][lane];
      }
      ref = m + __builtin_amdgcn_logf(sum) + kRoom;
    }
    reset();
    if (__builtin_fabsf(ref) < INFINITY) m = ref;
  }
  // Whether the sums hold an infinity or NaN.
  __device__ __forceinline__ bool not_finite() const {
    float t = 0.0f;
#pragma unroll
    for (int dt = 0; dt < kTiles; ++dt)
#pragma unroll
      for (int r = 0; r < 16; ++r) t = __builtin_fmaf(o[dt][r], 0.0f, t);
    return __any(!(t == 0.0f));
  }

  // o += V^T P^T for keys with p != 0 alone: V's infinities and NaN are taken out
  // of the product and counted in products of their own, so that one that is
  // hidden from a row (p = 0) does not reach it.  (p >= 0, so its bits are 0
  // exactly where it is.)
  template <int OFF, int P>
  __device__ __forceinline__ void accumulate_safe(const u32x4 (&p)[P], const u32x4 (&rest)[P]) {
#pragma unroll
    for (int dt = 0; dt < kTiles; ++dt) {
      floatx16 pos{}, neg{};
#pragma unroll
      for (int s = 0; s < P; ++s) {
        asm volatile("" ::: "memory");  // one operand at a time: registers
        const u32x4 a = v_operand<OFF>(dt, s);
        u32x4 fin, up, down, seen;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t ai = a[i], pi = p[s][i];
          const u16x2 w = __builtin_bit_cast(u16x2, ai), mag = w & static_cast<uint16_t>(0x7FFF);
          const u16x2 zero = {0, 0}, one = {1, 1};
          const u16x2 odd = zero - __builtin_elementwise_min(__builtin_elementwise_sub_sat(mag, u16x2(kInf - 1)), one);
          const u16x2 nan = zero - __builtin_elementwise_min(__builtin_elementwise_sub_sat(mag, u16x2(kInf)), one);
          const u16x2 minus = zero - (w >> static_cast<uint16_t>(15));
          const u16x2 in = zero - __builtin_elementwise_min(__builtin_bit_cast(u16x2, pi), one);
          fin[i] = __builtin_bit_cast(uint32_t, w & ~odd);
          up[i] = __builtin_bit_cast(uint32_t, odd & (nan | ~minus) & u16x2(kOne1));
          down[i] = __builtin_bit_cast(uint32_t, odd & (nan | minus) & u16x2(kOne1));
          seen[i] = __builtin_bit_cast(uint32_t, in & u16x2(kOne1));
        }
        o[dt] = E::mfma(__builtin_bit_cast(vec8, fin), __builtin_bit_cast(vec8, p[s]), o[dt]);
        o[dt] = E::mfma(__builtin_bit_cast(vec8, fin), __builtin_bit_cast(vec8, rest[s]), o[dt]);
        pos = E::mfma(__builtin_bit_cast(vec8, up), __builtin_bit_cast(vec8, seen), pos);
        neg = E::mfma(__builtin_bit_cast(vec8, down), __builtin_bit_cast(vec8, seen), neg);
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        // a count of one or more becomes infinity, none 0 (compares would be 64 live masks)
        o[dt][r] += pos[r] * 0x1p127f * 4.0f;
        o[dt][r] -= neg[r] * 0x1p127f * 4.0f;
      }
    }
  }

  // o += V^T P^T of P 16-key steps at byte offset OFF.
  template <int OFF, int P>
  __device__ __forceinline__ void accumulate(const u32x4 (&p)[P]) {
    constexpr int kAll = P * kTiles;
    u32x4 a[kAhead + 1];
#pragma unroll
    for (int i = 0; i < kAll + kAhead; ++i) {
      if (i < kAll) a[i % (kAhead + 1)] = v_operand<OFF>(i % kTiles, i / kTiles);
      if (i >= kAhead) {
        const int c = i - kAhead;
        o[c % kTiles] = E::mfma(__builtin_bit_cast(vec8, a[c % (kAhead + 1)]), __builtin_bit_cast(vec8, p[c / kTiles]), o[c % kTiles]);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  }

  // The NS key tiles at byte offset OFF of the stage.  mask: whether some key is
  // hidden from some row; visible(n, r): whether the lane's query sees key
  // mfma_row(r, hf) of the n-th; fine: two-term probabilities.
  template <int OFF, bool SECOND, class Visible>
  __device__ __forceinline__ void step(float alpha, bool mask, bool fine, Visible visible) {
    floatx16 x[NS];
    logits<OFF>(x);
    if (__builtin_expect(mask, 0)) {
#pragma unroll
      for (int n = 0; n < NS; ++n)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (!visible(n, r)) x[n][r] = -INFINITY;
    }
    float e[NS][16];
    float sum = INFINITY;
    if (__builtin_expect(!fresh(), 1)) sum = exponentials(x, alpha, m, e);
    if (__builtin_expect(__any(!(sum <= kHigh)), 0)) sum = exponentials(x, alpha, raise(fmaxf(m, largest(x, alpha))), e);
    l += sum;
    u32x4 p[2 * NS], rest[2 * NS];
    pack(e, p);
    if constexpr (SECOND) {
      pack_rest(e, p, rest);
      accumulate_safe<OFF>(p, rest);
    } else {
      accumulate<OFF>(p);
      if (__builtin_expect(fine || mask, F == kOne)) {
        pack_rest(e, p, rest);
        accumulate<OFF>(rest);
      }
    }
  }

  // kPair: both tiles of the stage; every wave of the workgroup calls it.  on:
  // whether this wave's rows see any of it; fine: two-term probabilities.
  template <bool SECOND, class Visible>
  __device__ __forceinline__ void step_pair(AreaType& area, float alpha, bool on, bool mask, bool fine, Visible visible) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int tile = ks & 1;  // (a wave past the pairs has no rows: on is false)
    fine = (fine || mask) && tiles <= 2;
    floatx16 x[1];
    float e[1][16], sum = 0.0f;
    auto give = [&] {
      u32x4 p[2];
      pack(e, p);
      area.p[rt][tile][0][lane] = p[0];
      area.p[rt][tile][1][lane] = p[1];
      if (fine) {
        u32x4 rest[2];
        pack_rest(e, p, rest);
        area.p[rt + 2][tile][0][lane] = rest[0];
        area.p[rt + 2][tile][1][lane] = rest[1];
      }
    };
    bool high = false;
    if (__builtin_expect(on, 1)) {
      logits<0>(x);
      if (__builtin_expect(mask, 0)) {
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (!visible(tile, r)) x[0][r] = -INFINITY;
      }
      sum = exponentials(x, alpha, m, e);
      high = __any(!(sum <= kHigh));
      give();
    }
    if (lane == 0) area.raise[wave] = high;
    stage_barrier();
    const u32x4 f0 = *reinterpret_cast<const u32x4*>(area.raise), f1 = *reinterpret_cast<const u32x4*>(area.raise + 4);
    if (__builtin_expect(__any((f0.x | f0.y | f0.z | f0.w | f1.x | f1.y | f1.z | f1.w) != 0), 0)) {
      // both waves of a pair go on against one reference
      const float top = on ? largest(x, alpha) : -INFINITY;
      if (on && lane < 32) area.top[rt][tile][lane] = top;
      stage_barrier();
      if (on) {
        sum = exponentials(x, alpha, raise(fmaxf(m, fmaxf(area.top[rt][0][lane & 31], area.top[rt][1][lane & 31]))), e);
        give();
      }
      stage_barrier();
    }
    if (__builtin_expect(!on, 0)) return;
    l += sum;
    u32x4 p[4];
#pragma unroll
    for (int s = 0; s < 4; ++s) p[s] = area.p[rt][s >> 1][s & 1][lane];
    u32x4 rest[4];
    if constexpr (SECOND) {
#pragma unroll
      for (int s = 0; s < 4; ++s) rest[s] = fine ? area.p[rt + 2][s >> 1][s & 1][lane] : u32x4{};
      accumulate_safe<0>(p, rest);
    } else {
      accumulate<0>(p);
      if (__builtin_expect(fine, 0)) {
#pragma unroll
        for (int s = 0; s < 4; ++s) rest[s] = area.p[rt + 2][s >> 1][s & 1][lane];
        accumulate<0>(rest);
      }
    }
  }

  // The stage at byte offset OFF.  first_key: of the stage; masked(key, keys):
  // whether some of these keys is hidden from some row; shown(key): whether the
  // lane's query sees it.
  template <int OFF, bool SECOND, class Masked, class Shown>
  __device__ __forceinline__ void tile(AreaType& area, float alpha, int first_key, bool on, bool fine, Masked masked,
                                       Shown shown) {
    const int hf = (threadIdx.x >> 5) & 1;
    auto visible = [&](int n, int r) { return shown(first_key + 32 * n + mfma_row(r, hf)); };
    if constexpr (F == kPair) {
      step_pair<SECOND>(area, alpha, on && ks < 2, on && masked(first_key, 64), fine, visible);
    } else if constexpr (F == kBoth) {
      if (on && ks == 0) step<OFF, SECOND>(alpha, masked(first_key, 64), fine, visible);
    } else if (on && ks < streams) {
      if (streams == 1 || ks == 0) step<OFF, SECOND>(alpha, masked(first_key, 32), fine, visible);
      if (streams == 1 || ks == 1)
        step<OFF + 32 * S::kPitch, SECOND>(alpha, masked(first_key + 32, 32), fine, [&](int, int r) { return visible(1, r); });
    }
  }

  // Adds up what the waves that share rows have; every wave calls it, after the
  // last tile.  Returns whether this wave writes (kPair: its channels), with l the
  // row's sum.
  static constexpr int kStateBytes = (kChannels / 2 + 2) * 256;  // per wave
  __device__ __forceinline__ bool finish(uint8_t* stage, AreaType& area, bool on) {
    const int lane = threadIdx.x & 63;
    if constexpr (F == kOne) {
      if (streams == 2) {
        stage_barrier();
        uint8_t* at = stage + rt * kStateBytes;
        if (on && ks == 1) write_state(at);
        stage_barrier();
        if (on && ks == 0) merge_state(at);
      }
    }
    {
      const LanePair p = lane_pair32(__builtin_bit_cast(uint32_t, l));
      l = __builtin_bit_cast(float, p.lo) + __builtin_bit_cast(float, p.hi);
    }
    if constexpr (F == kPair) {
      if (on && ks < 2) area.l[rt][ks][lane & 31] = l;
      stage_barrier();
      if (on && ks < 2) l = area.l[rt][0][lane & 31] + area.l[rt][1][lane & 31];
    }
    return on && ks < (F == kPair ? 2 : 1);
  }
  __device__ __forceinline__ void write_state(uint8_t* to) const {
    floatx4* f = reinterpret_cast<floatx4*>(to) + (threadIdx.x & 63);
#pragma unroll
    for (int dt = 0; dt < kTiles; ++dt)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        f[64 * (4 * dt + r)] = floatx4{o[dt][4 * r], o[dt][4 * r + 1], o[dt][4 * r + 2], o[dt][4 * r + 3]};
    reinterpret_cast<floatx2*>(f - (threadIdx.x & 63) + 64 * 4 * kTiles)[threadIdx.x & 63] = floatx2{m, l};
  }
  __device__ __forceinline__ void merge_state(const uint8_t* from) {
    const floatx4* f = reinterpret_cast<const floatx4*>(from) + (threadIdx.x & 63);
    const floatx2 ml = reinterpret_cast<const floatx2*>(f - (threadIdx.x & 63) + 64 * 4 * kTiles)[threadIdx.x & 63];
    // (against twice the larger reference: two finite sums then add up to one)
    const float mn = fmaxf(m, ml.x) + 1.0f, ref = mn == -INFINITY ? 0.0f : mn;
    const float a = __builtin_amdgcn_exp2f(m - ref), b = __builtin_amdgcn_exp2f(ml.x - ref);
    m = mn;
    l = l * a + ml.y * b;
#pragma unroll
    for (int dt = 0; dt < kTiles; ++dt)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const floatx4 x = f[64 * (4 * dt + r)];
#pragma unroll
        for (int i = 0; i < 4; ++i) o[dt][4 * r + i] = o[dt][4 * r + i] * a + x[i] * b;
      }
  }
  // Whether this lane writes the row's reference and sum, or its lse.
  __device__ __forceinline__ bool writes_sum() const { return (threadIdx.x & 32) == 0 && ks == 0; }
  // The row's result, rounded to E: a lane-half writes 16 contiguous bytes.
  __device__ __forceinline__ void write_out(void* row, float inv) const {
    uint8_t* p = static_cast<uint8_t*>(row) + 16 * ((threadIdx.x >> 5) & 1) + (F == kPair ? ks * D : 0);
#pragma unroll
    for (int dt = 0; dt < kTiles; ++dt)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
          w[i] = pack2<E>(o[dt][8 * h + 2 * i] * inv, o[dt][8 * h + 2 * i + 1] * inv);
        // the halves hold channels 4 hf .. + 3 of two groups of 8: each half takes one group
        const auto s0 = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false);
        const auto s1 = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
        *reinterpret_cast<u32x4*>(p + 64 * dt + 32 * h) = u32x4{s0[0], s1[0], s0[1], s1[1]};
      }
  }
  // The row's unnormalized sum in binary32.
  __device__ __forceinline__ void write_partial(float* row) const {
    float* p = row + 4 * ((threadIdx.x >> 5) & 1) + (F == kPair ? ks * kChannels : 0);
#pragma unroll
    for (int dt = 0; dt < kTiles; ++dt)
#pragma unroll
      for (int h = 0; h < 4; ++h)
        *reinterpret_cast<floatx4*>(p + 32 * dt + 8 * h) =
            floatx4{o[dt][4 * h], o[dt][4 * h + 1], o[dt][4 * h + 2], o[dt][4 * h + 3]};
  }
};

// Walks tiles [t0, t1) of a workgroup: issue(t, b) starts the direct loads of tile
// t into buffer b, tile(t, off, second) multiplies the tile at stage offset `off`
// (integral constants).  The next tile is in flight while one is multiplied, and
// one barrier per tile orders both: when it is passed every wave has the tile and
// is done with the buffer that the next loads fill.
template <int D, bool SECOND, class Wave, class Issue, class Tile>
__device__ __forceinline__ void walk_once(Wave& w, int t0, int t1, Issue issue, Tile tile) {
  constexpr int kBytes = Stage<D>::kBytes;
  const std::integral_constant<bool, SECOND> second;
  if (t0 < t1) issue(t0, 0);
  w.wait_q();
  if constexpr (2 * kBytes <= 65536) {  // both buffers within an instruction's offset
    for (int t = t0; t < t1; t += 2) {
      wait_direct_loads();
      stage_barrier();
      if (t + 1 < t1) issue(t + 1, 1);
      tile(t, std::integral_constant<int, 0>{}, second);
      if (t + 1 >= t1) break;
      wait_direct_loads();
      stage_barrier();
      if (t + 2 < t1) issue(t + 2, 0);
      tile(t + 1, std::integral_constant<int, kBytes>{}, second);
    }
  } else {
    int by = kBytes;
    for (int t = t0; t < t1; ++t) {
      wait_direct_loads();
      stage_barrier();
      if (t + 1 < t1) issue(t + 1, (t + 1 - t0) & 1);
      tile(t, std::integral_constant<int, 0>{}, second);
      w.move(by);
      by = -by;
    }
    if (by < 0) w.move(by);  // back to the first buffer
  }
}
// walk(second) goes through all of a workgroup's tiles (walk_once).  The products of
// the first time let an infinity or NaN of V reach rows from which it is hidden (0
// times it is NaN), and second terms make NaN of one that is seen; so where a result
// is not finite, everything is done again by accumulate_safe, whose arithmetic would
// cost the first loop its registers, and against a reference that lets no sum overflow
// (again).  Ends with a barrier: the stage is free.
template <class Wave, class AreaType, class Walk>
__device__ __forceinline__ void walk_tiles(Wave& w, AreaType& area, Walk walk) {
  if (threadIdx.x == 0) area.not_finite = 0;
  walk(std::integral_constant<bool, false>{});
  stage_barrier();
  if (w.not_finite()) area.not_finite = 1;
  stage_barrier();
  if (__builtin_expect(*const_cast<volatile int32_t*>(&area.not_finite) != 0, 0)) {
    w.again(area);
    walk(std::integral_constant<bool, true>{});
    stage_barrier();
  }
}

// A row's sum l is 0 where it sees no key (its result is 0), and where the logits of
// all the keys it sees are -infinity: softmax over those is NaN (exp(-inf - -inf)).
// `saw`: whether it sees a key.
__device__ __forceinline__ float inverse_sum(float l, bool saw) {
  return l == 0.0f ? (saw ? NAN : 0.0f) : 1.0f / l;
}
// l of a part as it is written beside m: 1 with m = -infinity where the part's logits
// are all -infinity, which weighs nothing beside another part.
__device__ __forceinline__ float part_sum(float l, bool saw) { return l == 0.0f && saw ? 1.0f : l; }
__device__ __forceinline__ float log_sum(float m, float l) {
  return l == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

// op over the wave's 64 lanes (all active), in every lane; op is commutative.
template <class Op>
__device__ __forceinline__ float over_wave(float v, Op op) {
  auto moved = [](uint32_t x) { return __builtin_bit_cast(float, x); };
  auto bits = [](float x) { return __builtin_bit_cast(uint32_t, x); };
  const LanePair a = lane_pair16(bits(v));
  v = op(moved(a.lo), moved(a.hi));
  v = op(v, moved(dpp_mov<0x140>(bits(v))));  // lanes i and 15 - i
  v = op(v, moved(dpp_mov<0x141>(bits(v))));  // i and 7 - i
  v = op(v, moved(dpp_mov<0xB1>(bits(v))));   // i and i ^ 1
  v = op(v, moved(dpp_mov<0x4E>(bits(v))));   // i and i ^ 2
  const LanePair b = lane_pair32(bits(v));
  return op(moved(b.lo), moved(b.hi));
}

// Joins the parts of a row.  WAVES waves of a workgroup share it, every WAVES-th
// part to each; a lane has D / 64 channels (at D = 32 the upper half of a wave
// repeats the lower).  Finite parts are added against a reference 2^kRoom times their
// largest, so that their sum is finite too.  A wave reads the references and sums of 64
// parts at once, and eight parts' sums are in flight together.
template <int D, int WAVES>
struct JoinedRow {
  static constexpr int kPer = D >= 64 ? D / 64 : 1;
  typedef float vec __attribute__((ext_vector_type(kPer)));
  struct Shared {
    float m[4], l[4], o[4][64 * kPer];
    int32_t saw[4];
  };
  float m = -INFINITY, l = 0.0f, o[kPer] = {};
  bool saw = false;  // a part's keys, with logits of -infinity all of them (part_sum)

  // Part s is row first + s * stride of the partial results.
  __device__ __forceinline__ void add(const float* part_o, const float* part_ml, int64_t first, int64_t stride, int parts) {
    const int lane = threadIdx.x & 63, wave = WAVES > 1 ? static_cast<int>(threadIdx.x >> 6) % WAVES : 0;
    const float* po = part_o + kPer * (D >= 64 ? lane : lane & 31);
    const int mine = (parts - wave + WAVES - 1) / WAVES;
    for (int s0 = 0; s0 < mine; s0 += 64) {
      const int n = min(64, mine - s0);
      const int64_t from = first + (wave + static_cast<int64_t>(WAVES) * s0) * stride;
      floatx2 ml = {-INFINITY, 0.0f};
      if (lane < n) ml = *reinterpret_cast<const floatx2*>(part_ml + 2 * (from + WAVES * lane * stride));
      vec x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = *reinterpret_cast<const vec*>(po + (from + min(i, n - 1) * WAVES * stride) * D);
      const float top = over_wave(ml.x, [](float a, float b) { return fmaxf(a, b); });
      const float mn = fmaxf(m, top + kRoom), ref = mn == -INFINITY ? 0.0f : mn;
      const float keep = __builtin_amdgcn_exp2f(m - ref), f = __builtin_amdgcn_exp2f(ml.x - ref);
      const float sum = over_wave(ml.y * f, [](float a, float b) { return a + b; });  // 0 of a part that saw nothing
      l = l * keep + sum;
      m = mn;
#pragma unroll
      for (int i = 0; i < kPer; ++i) o[i] *= keep;
      const uint64_t seen = __ballot(ml.x != -INFINITY || ml.y != 0.0f);  // the others may have written no sums
      saw |= __any(ml.x == -INFINITY && ml.y > 0.0f);
      for (int s = 0; s < n; s += 8) {
        vec next[8];
        if (s + 8 < n) {
#pragma unroll
          for (int i = 0; i < 8; ++i)
            next[i] = *reinterpret_cast<const vec*>(po + (from + min(s + 8 + i, n - 1) * WAVES * stride) * D);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (s + i >= n) break;
          const float fs = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, f), s + i));
          const bool use = seen >> (s + i) & 1;
#pragma unroll
          for (int c = 0; c < kPer; ++c) o[c] += (use ? x[i][c] : 0.0f) * fs;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = next[i];
      }
    }
  }
  // The waves' shares together, in wave 0 of the row (true there).
  __device__ __forceinline__ bool together(Shared& sh) {
    if constexpr (WAVES > 1) {
      const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
      if (lane == 0) {
        sh.m[wave] = m;
        sh.l[wave] = l;
        sh.saw[wave] = saw;
      }
#pragma unroll
      for (int i = 0; i < kPer; ++i) sh.o[wave][kPer * lane + i] = o[i];
      __syncthreads();
      if (wave != 0) return false;
#pragma unroll
      for (int w = 1; w < WAVES; ++w) {
        const float mn = fmaxf(m, sh.m[w]), ref = mn == -INFINITY ? 0.0f : mn;
        const float a = __builtin_amdgcn_exp2f(m - ref), b = __builtin_amdgcn_exp2f(sh.m[w] - ref);
        m = mn;
        saw |= sh.saw[w] != 0;
        l = l * a + sh.l[w] * b;
#pragma unroll
        for (int i = 0; i < kPer; ++i) o[i] = o[i] * a + sh.o[w][kPer * lane + i] * b;
      }
    }
    return true;
  }
  template <class E>
  __device__ __forceinline__ void write(typename E::elem* out) const {
    const int lane = threadIdx.x & 63;
    const float inv = inverse_sum(l, saw);
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if (D >= 64 || lane < D) out[kPer * lane + i] = static_cast<typename E::elem>(o[i] * inv);
  }
};
// Rows for which a wave each would leave most of the GPU idle get four (2048 rows of 17
// parts, with the launch before: 39 us by four waves, 37 by one; 1024 rows of 33: 25.0
// and 26.2).
constexpr uint64_t kFewRows = 1024;

}  // namespace skv
