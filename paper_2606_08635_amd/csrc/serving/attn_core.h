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
// rounded (nearest even) to the inputs' 16-bit type for the second product --
// the MFMA takes both operands in one type -- while l sums them unrounded; the
// result is rounded once to the output type.
#pragma once

#include "../device_util.h"

namespace skv {

typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef short shortx4 __attribute__((ext_vector_type(4)));

struct TypeF16 {
  typedef _Float16 elem;
  typedef _Float16 vec8 __attribute__((ext_vector_type(8)));
  typedef _Float16 vec2 __attribute__((ext_vector_type(2)));
  static constexpr uint16_t kInf = 0x7C00, kOne = 0x3C00;
  __device__ static __forceinline__ floatx16 mfma(vec8 a, vec8 b, floatx16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
  }
};
struct TypeBF16 {
  typedef __bf16 elem;
  typedef __bf16 vec8 __attribute__((ext_vector_type(8)));
  typedef __bf16 vec2 __attribute__((ext_vector_type(2)));
  static constexpr uint16_t kInf = 0x7F80, kOne = 0x3F80;
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
// among its own loads; the tile loop waits for it itself (wait_direct_loads).
__device__ __forceinline__ void direct_load(const void* src, uint32_t lds_base) {
  asm volatile("s_mov_b32 m0, %1\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(src), "s"(lds_base) : "memory", "m0");
}
__device__ __forceinline__ void direct_load(const void* uniform_base, uint32_t offset, uint32_t lds_base) {
  asm volatile("s_mov_b32 m0, %2\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(offset), "s"(uniform_base), "s"(lds_base)
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
  static constexpr int kWaves = 4;
  static constexpr int kThreads = kWaves * 64;
  static constexpr int kKeys = 64;
  static constexpr int kCpr = D / 8;
  static constexpr int kPitch = D * 2;
  static constexpr int kHalf = kKeys * kPitch;  // bytes of K, and of V
  static constexpr int kBytes = 2 * kHalf;
  static constexpr int kPieces = kKeys * kCpr / kThreads;  // 16-byte loads of K per thread, and of V
  static constexpr int kRowStep = kThreads / kCpr;         // rows between a thread's pieces
  // waves per SIMD that the registers allow: o and Q alone are 3 D / 4 registers
  static constexpr int kWavesPerSimd = D >= 256 ? 1 : 2;
  static_assert(kKeys * kCpr % kThreads == 0, "whole pieces per thread");
  __device__ static constexpr int swz(int r) {
    return D >= 128 ? ((r & 3) << 2) | ((r >> 2) & 3) : D == 64 ? (((r >> 1) & 1) << 2) | ((r >> 2) & 3) : (r >> 2) & 3;
  }
};

// One wave's 32 query rows: state and arithmetic.  NS: 32-key tiles that it
// takes per step.
template <class E, int D, int NS>
struct WaveAttention {
  typedef typename E::vec8 vec8;
  typedef Stage<D> S;
  static constexpr int kSteps = D / 16;  // MFMA steps of a logit
  static constexpr int kTiles = D / 32;  // 32-channel tiles of o
  // A step is exponentiated against the current reference m first, without its
  // maximum; only where that gives a sum past kHigh (or a NaN: m still -inf) is
  // the maximum taken, m raised and o rescaled.  2^15 keeps every probability
  // inside binary16.  m is some earlier step's maximum, so what underflows
  // against it is negligible beside what is in the sum already.
  static constexpr float kHigh = 32768.0f;
  static constexpr uint16_t kInf = E::kInf, kOne = E::kOne;

  vec8 q[kSteps];
  floatx16 o[kTiles];
  float m, l;
  uint32_t kaddr[kSteps];               // LDS addresses in the first stage buffer
  uint32_t vaddr[kTiles < 4 ? kTiles : 4][2];
  uint32_t vrows;                       // this lane's 16 bytes of the wave's V rows

  // first: the wave's first key of a stage
  __device__ __forceinline__ void init(const void* stage, int first) {
    const int lane = threadIdx.x & 63, hf = lane >> 5, j = lane & 31, i = lane & 15, g = (lane >> 4) & 1;
    const uint32_t base = lds_address(stage) + static_cast<uint32_t>(first * S::kPitch);
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      kaddr[s] = base + static_cast<uint32_t>(j * S::kPitch + 16 * ((2 * s + hf) ^ S::swz(j)));
      asm volatile("" : "+v"(kaddr[s]));  // one register each: tile offsets become immediates
    }
#pragma unroll
    for (int dt = 0; dt < (kTiles < 4 ? kTiles : 4); ++dt)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int row = 8 * u + 4 * hf + (i >> 2);
        const int chunk = 4 * dt + 2 * g + ((i & 3) >> 1);
        vaddr[dt][u] =
            base + static_cast<uint32_t>(S::kHalf + row * S::kPitch + 16 * (chunk ^ S::swz(row)) + 8 * (i & 1));
        asm volatile("" : "+v"(vaddr[dt][u]));
      }
    vrows = base + static_cast<uint32_t>(S::kHalf + 16 * lane);
#pragma unroll
    for (int dt = 0; dt < kTiles; ++dt) o[dt] = floatx16{};
    m = -INFINITY;
    l = 0.0f;
  }

  // Moves on to the other stage buffer where steps do not name it (D = 256: its
  // offset is past the 16 bits of an LDS instruction).
  __device__ __forceinline__ void move(int bytes) {
#pragma unroll
    for (int s = 0; s < kSteps; ++s) kaddr[s] += bytes;
#pragma unroll
    for (int dt = 0; dt < (kTiles < 4 ? kTiles : 4); ++dt)
#pragma unroll
      for (int u = 0; u < 2; ++u) vaddr[dt][u] += bytes;
    vrows += bytes;
  }

  __device__ __forceinline__ void load_q(const void* row) {
    const uint8_t* p = static_cast<const uint8_t*>(row) + 16 * ((threadIdx.x >> 5) & 1);
#pragma unroll
    for (int s = 0; s < kSteps; ++s) q[s] = __builtin_bit_cast(vec8, *reinterpret_cast<const u32x4*>(p + 32 * s));
    // waited for here: the compiler's own wait would sit in the tile loop, where it
    // would also wait for the direct loads that it does not know of
    __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0)
#pragma unroll
    for (int s = 0; s < kSteps; ++s) asm volatile("" : "+v"(q[s]));
  }

  __device__ static __forceinline__ u32x4 lds16(uint32_t addr) {
    typedef __attribute__((address_space(3))) const u32x4* ptr;
    return *reinterpret_cast<ptr>(static_cast<uintptr_t>(addr));
  }
  // channels 32 dt + lane % 32 of the 8 keys 16 s + {4 hf .. + 3, 8 + 4 hf .. + 3}
  template <int OFF>
  __device__ __forceinline__ u32x4 v_operand(int dt, int s) const {
    typedef __attribute__((address_space(3))) shortx4* ptr;
    u32x4 a;
    const uint32_t off = static_cast<uint32_t>(OFF + 16 * s * S::kPitch + (dt >> 2) * 256);
    const u32x2 lo = __builtin_bit_cast(
        u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<ptr>(static_cast<uintptr_t>(vaddr[dt & 3][0] + off))));
    const u32x2 hi = __builtin_bit_cast(
        u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<ptr>(static_cast<uintptr_t>(vaddr[dt & 3][1] + off))));
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

  // Whether V holds an infinity or NaN in the wave's keys of this stage.
  template <int OFF>
  __device__ __forceinline__ bool v_not_finite() const {
    uint32_t top = 0;
#pragma unroll
    for (int u = 0; u < NS * 32 * S::kPitch / 1024; ++u)
      top = max(top, absmax_bits8(lds16(vrows + static_cast<uint32_t>(OFF + 1024 * u))));
    return __any(top >= E::kInf);
  }

  // o += V^T P^T for keys with p != 0 alone: V's infinities and NaN are taken out
  // of the product and counted in products of their own, so that one that is
  // hidden from a row (p = 0) does not reach it.
  // (p >= 0, so its bits are 0 exactly where it is.)
  template <int OFF>
  __device__ __forceinline__ void accumulate_safe(const u32x4 (&p)[2 * NS]) {
#pragma unroll
    for (int dt = 0; dt < kTiles; ++dt) {
      floatx16 pos{}, neg{};
#pragma unroll
      for (int s = 0; s < 2 * NS; ++s) {
        asm volatile("" ::: "memory");  // one operand at a time: this path is rare, its registers are not to cost the other
        const u32x4 a = v_operand<OFF>(dt, s);
        u32x4 fin, up, down, seen;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const u16x2 w = __builtin_bit_cast(u16x2, a[i]), mag = w & static_cast<uint16_t>(0x7FFF);
          const u16x2 zero = {0, 0}, one = {1, 1};
          const u16x2 odd = zero - __builtin_elementwise_min(__builtin_elementwise_sub_sat(mag, u16x2(kInf - 1)), one);
          const u16x2 nan = zero - __builtin_elementwise_min(__builtin_elementwise_sub_sat(mag, u16x2(kInf)), one);
          const u16x2 neg1 = zero - (w >> static_cast<uint16_t>(15));
          const u16x2 in = zero - __builtin_elementwise_min(__builtin_bit_cast(u16x2, p[s][i]), one);
          fin[i] = __builtin_bit_cast(uint32_t, w & ~odd);
          up[i] = __builtin_bit_cast(uint32_t, odd & (nan | ~neg1) & u16x2(kOne));
          down[i] = __builtin_bit_cast(uint32_t, odd & (nan | neg1) & u16x2(kOne));
          seen[i] = __builtin_bit_cast(uint32_t, in & u16x2(kOne));
        }
        o[dt] = E::mfma(__builtin_bit_cast(vec8, fin), __builtin_bit_cast(vec8, p[s]), o[dt]);
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

  // One step: the wave's NS * 32 keys of the stage at byte offset OFF of the
  // stage area.  mask: whether some key is hidden from some row; visible(n, r): is
  // key mfma_row(r, hf) of tile n seen by the lane's query.
  template <int OFF, class Visible>
  __device__ __forceinline__ void step(float alpha, bool mask, Visible visible) {
    floatx16 x[NS];
#pragma unroll
    for (int n = 0; n < NS; ++n) x[n] = floatx16{};
    // operands kAhead products early, so that their LDS reads are behind the matrix units' work
    constexpr int kAhead = 4;
    {
      constexpr int kAll = NS * kSteps;
      u32x4 a[kAhead + 1];
#pragma unroll
      for (int i = 0; i < kAll + kAhead; ++i) {
        if (i < kAll) a[i % (kAhead + 1)] = lds16(kaddr[i / NS] + static_cast<uint32_t>(OFF + i % NS * 32 * S::kPitch));
        if (i >= kAhead) {
          const int c = i - kAhead;
          x[c % NS] = E::mfma(__builtin_bit_cast(vec8, a[c % (kAhead + 1)]), q[c / NS], x[c % NS]);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    if (__builtin_expect(mask, 0)) {
#pragma unroll
      for (int n = 0; n < NS; ++n)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (!visible(n, r)) x[n][r] = -INFINITY;
    }
    float e[NS][16];
    float sum = 0.0f;
#pragma unroll
    for (int n = 0; n < NS; ++n) {
#pragma unroll
      for (int r = 0; r < 16; ++r) e[n][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[n][r], alpha, -m));
      float t[8];
#pragma unroll
      for (int r = 0; r < 8; ++r) t[r] = e[n][r] + e[n][r + 8];
      sum += ((t[0] + t[1]) + (t[2] + t[3])) + ((t[4] + t[5]) + (t[6] + t[7]));
    }
    if (__builtin_expect(__any(!(sum <= kHigh)), 0)) {
      float top = -INFINITY;
#pragma unroll
      for (int n = 0; n < NS; ++n)
#pragma unroll
        for (int r = 0; r < 16; ++r) top = fmaxf(top, x[n][r]);
      const LanePair p = lane_pair32(__builtin_bit_cast(uint32_t, top * alpha));
      const float mn = fmaxf(m, fmaxf(__builtin_bit_cast(float, p.lo), __builtin_bit_cast(float, p.hi)));
      const float ref = mn == -INFINITY ? 0.0f : mn;  // nothing seen yet: every probability 0
      rescale(__builtin_amdgcn_exp2f(m - ref));
      m = mn;
      sum = 0.0f;
#pragma unroll
      for (int n = 0; n < NS; ++n)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          e[n][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[n][r], alpha, -ref));
          sum += e[n][r];
        }
    }
    l += sum;
    u32x4 p[2 * NS];
#pragma unroll
    for (int s = 0; s < 2 * NS; ++s) {
      const float* f = &e[s >> 1][8 * (s & 1)];
      p[s].x = pack2<E>(f[0], f[1]);
      p[s].y = pack2<E>(f[2], f[3]);
      p[s].z = pack2<E>(f[4], f[5]);
      p[s].w = pack2<E>(f[6], f[7]);
    }
    if (__builtin_expect(mask && v_not_finite<OFF>(), 0)) {
      accumulate_safe<OFF>(p);
      return;
    }
    constexpr int kAll = 2 * NS * kTiles;
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

  // Adds the state that another wave left at `from` (write_state) to this one's.
  static constexpr int kStateBytes = (D / 2 + 2) * 256;  // per wave
  __device__ __forceinline__ void write_state(uint8_t* to) const {
    float* f = reinterpret_cast<float*>(to) + (threadIdx.x & 63);
    f[0] = m;
    f[64] = l;
#pragma unroll
    for (int dt = 0; dt < kTiles; ++dt)
#pragma unroll
      for (int r = 0; r < 16; ++r) f[64 * (2 + 16 * dt + r)] = o[dt][r];
  }
  __device__ __forceinline__ void merge_state(const uint8_t* from) {
    const float* f = reinterpret_cast<const float*>(from) + (threadIdx.x & 63);
    const float m2 = f[0], mn = fmaxf(m, m2), ref = mn == -INFINITY ? 0.0f : mn;
    const float a = __builtin_amdgcn_exp2f(m - ref), b = __builtin_amdgcn_exp2f(m2 - ref);
    m = mn;
    l = l * a + f[64] * b;
#pragma unroll
    for (int dt = 0; dt < kTiles; ++dt)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[dt][r] = o[dt][r] * a + f[64 * (2 + 16 * dt + r)] * b;
  }
  // l over both lane-halves.
  __device__ __forceinline__ float total() const {
    const LanePair p = lane_pair32(__builtin_bit_cast(uint32_t, l));
    return __builtin_bit_cast(float, p.lo) + __builtin_bit_cast(float, p.hi);
  }
  // The row's result, rounded to E: a lane-half writes 16 contiguous bytes.
  __device__ __forceinline__ void write_out(void* row, float inv) const {
    uint8_t* p = static_cast<uint8_t*>(row) + 16 * ((threadIdx.x >> 5) & 1);
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
    float* p = row + 4 * ((threadIdx.x >> 5) & 1);
#pragma unroll
    for (int dt = 0; dt < kTiles; ++dt)
#pragma unroll
      for (int h = 0; h < 4; ++h)
        *reinterpret_cast<floatx4*>(p + 32 * dt + 8 * h) =
            floatx4{o[dt][4 * h], o[dt][4 * h + 1], o[dt][4 * h + 2], o[dt][4 * h + 3]};
  }
};

// Walks tiles [t0, t1) of a workgroup: issue(t, b) starts the direct loads of tile
// t into buffer b, tile(t, off) multiplies the tile at stage offset `off` (an
// integral constant).  The next tile is in flight while one is multiplied, and one
// barrier per tile orders both: when it is passed every wave has the tile and is
// done with the buffer that the next loads fill.
template <int D, class Wave, class Issue, class Tile>
__device__ __forceinline__ void walk_tiles(Wave& w, int t0, int t1, Issue issue, Tile tile) {
  constexpr int kBytes = Stage<D>::kBytes;
  if (t0 < t1) issue(t0, 0);
  if constexpr (2 * kBytes <= 65536) {  // both buffers within an instruction's offset
    for (int t = t0; t < t1; t += 2) {
      wait_direct_loads();
      stage_barrier();
      if (t + 1 < t1) issue(t + 1, 1);
      tile(t, std::integral_constant<int, 0>{});
      if (t + 1 >= t1) break;
      wait_direct_loads();
      stage_barrier();
      if (t + 2 < t1) issue(t + 2, 0);
      tile(t + 1, std::integral_constant<int, kBytes>{});
    }
  } else {
    int by = kBytes;
    for (int t = t0; t < t1; ++t) {
      wait_direct_loads();
      stage_barrier();
      if (t + 1 < t1) issue(t + 1, (t + 1 - t0) & 1);
      tile(t, std::integral_constant<int, 0>{});
      w.move(by);
      by = -by;
    }
    if (by < 0) w.move(by);  // back to the first buffer
  }
}

__device__ __forceinline__ float inverse_or_zero(float l) { return l == 0.0f ? 0.0f : 1.0f / l; }
__device__ __forceinline__ float log_sum(float m, float l) {
  return l == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

// Joins the parts of one row: part s is row first + s * stride of the partial
// results.  A wave takes a row, its lanes D / 64 channels each (at D = 32 the
// lower half, and lanes past D are given nothing to write).
template <int D>
struct JoinedRow {
  static constexpr int kPer = D >= 64 ? D / 64 : 1;
  typedef float vec __attribute__((ext_vector_type(kPer)));
  float m = -INFINITY, l = 0.0f, o[kPer] = {};

  __device__ __forceinline__ JoinedRow(const float* part_o, const float* part_ml, int64_t first, int64_t stride,
                                       int parts) {
    const int lane = threadIdx.x & 63;
    const float* po = part_o + kPer * (D >= 64 ? lane : lane & 31);
    for (int s0 = 0; s0 < parts; s0 += 64) {  // references and sums of up to 64 parts at once
      floatx2 ml = {-INFINITY, 0.0f};
      if (s0 + lane < parts) ml = *reinterpret_cast<const floatx2*>(part_ml + 2 * (first + (s0 + lane) * stride));
      float top = ml.x;
#pragma unroll
      for (int x = 32; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor(top, x));
      const float mn = fmaxf(m, top), ref = mn == -INFINITY ? 0.0f : mn;
      const float keep = __builtin_amdgcn_exp2f(m - ref), f = __builtin_amdgcn_exp2f(ml.x - ref);
      float sum = ml.y * f;  // 0 of a part that saw nothing
#pragma unroll
      for (int x = 32; x > 0; x >>= 1) sum += __shfl_xor(sum, x);
      l = l * keep + sum;
      m = mn;
#pragma unroll
      for (int i = 0; i < kPer; ++i) o[i] *= keep;
      const uint64_t seen = __ballot(ml.x != -INFINITY || ml.y != 0.0f);  // the others wrote no sums
      const int n = min(64, parts - s0);
#pragma unroll 4
      for (int s = 0; s < n; ++s) {
        const float fs = __shfl(f, s);
        if (!(seen >> s & 1)) continue;
        const vec x = *reinterpret_cast<const vec*>(po + (first + (s0 + s) * stride) * D);
#pragma unroll
        for (int i = 0; i < kPer; ++i) o[i] += x[i] * fs;
      }
    }
  }
  template <class E>
  __device__ __forceinline__ void write(typename E::elem* out) const {
    const int lane = threadIdx.x & 63;
    const float inv = inverse_or_zero(l);
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if (D >= 64 || lane < D) out[kPer * lane + i] = static_cast<typename E::elem>(o[i] * inv);
  }
};

}  // namespace skv
