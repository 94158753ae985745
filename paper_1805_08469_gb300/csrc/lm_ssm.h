// Selective state space scan: what the forward and the backward kernels share (internal).
//
// Work is cut into blocks of one sequence, a split of its time, and up to CH channels of a group.  A block
// goes over its split in tiles of 16 steps: its threads stage a tile (step and step x of every channel, b and c) in
// shared memory as fp32, all once; then each thread takes four states of K channels through the tile in
// registers.  The LS lanes of a channel add up what the states give together.
//
//   lane = (state quad g, channel lane c), c fastest: the lanes of a quarter warp read the same b and c
//
// Splits: time is one split where the channels fill the GPU.  Else a first pass takes each split from a state of 0
// and leaves its last state and the sum of its steps; a block of the second pass composes the splits before its own,
//   h = exp(A sum step) h + last,
// and goes on from there.  A sum of +inf marks a split in which the state was dropped.
#pragma once

#include <type_traits>

#include "lm_internal.h"

namespace gem {
namespace lm {
namespace ssm {

constexpr int kTile = GEM_SSM_CHUNK;
static_assert(kTile == 16, "a reduction's lanes hold whole steps");
constexpr int kWarps = 4, kSsmThreads = 32 * kWarps;
constexpr int kQuad = 4;                        // states of a thread and channel
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct SsmArgs {
  gem_ssm_t in;
  gem_seq_t y, dy, dx, ddt, db, dc, dz;
  const float* h0;         // backward: dh_last
  float* h_last;           // backward: dh0
  float* saved;
  float *dA, *dskip, *ddt_bias;
  float *states, *sums;    // [B][splits][D][N], [B][splits][D]
  float* bc_part;          // [B][T][G][blocks][2][4 LS]
  float* param_part;       // [B][splits][N + 2][D]
  bool params;             // whether any of dA, dskip and ddt_bias is asked for
  int splits, blocks;      // of a sequence's time, of a group's channels
  int64_t steps;           // of a split
  bool wide;               // pieces of all tensors are whole and lie at multiples of their size (16 bytes at most)
};

__device__ __forceinline__ float ex2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float reciprocal(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
template <int V>
__device__ __forceinline__ Vec<V> ex2(Vec<V> x) {
#pragma unroll
  for (int k = 0; k < V; ++k) x.v[k] = ex2(x.v[k]);
  return x;
}
template <int V>
__device__ __forceinline__ Vec<V> reciprocal(Vec<V> x) {
#pragma unroll
  for (int k = 0; k < V; ++k) x.v[k] = reciprocal(x.v[k]);
  return x;
}
template <int V>
__device__ __forceinline__ Vec<V> sigmoid(const Vec<V>& v) { return reciprocal<V>(ex2<V>(v * splat<V>(-kLog2e)) + splat<V>(1.0f)); }

// max(v, 0) + log(1 + w), w = exp(-|v|): log(1 + w) = 2 artanh(s) with s = w / (2 + w) <= 1/3, by its
// series in s^2, whose first term left out is 2e-8 of the sum.
template <int V>
__device__ __forceinline__ Vec<V> softplus(const Vec<V>& v) {
  Vec<V> w, most;
#pragma unroll
  for (int k = 0; k < V; ++k) {
    w.v[k] = ex2(fabsf(v.v[k]) * -kLog2e);
    most.v[k] = fmaxf(v.v[k], 0.0f);
  }
  const Vec<V> s = w * reciprocal<V>(w + splat<V>(2.0f)), q = s * s;
  Vec<V> r = fma<V>(q, splat<V>(1.0f / 13), splat<V>(1.0f / 11));
  r = fma<V>(q, r, splat<V>(1.0f / 9));
  r = fma<V>(q, r, splat<V>(1.0f / 7));
  r = fma<V>(q, r, splat<V>(1.0f / 5));
  r = fma<V>(q, r, splat<V>(1.0f / 3));
  r = fma<V>(q, r, splat<V>(1.0f));
  return fma<V>(s + s, r, most);
}

// Four states.
struct Quad {
  Vec<2> a, b;
};
__device__ __forceinline__ Quad zeros() { return {splat<2>(0.0f), splat<2>(0.0f)}; }
__device__ __forceinline__ Quad quad(const float4& v) { return {{v.x, v.y}, {v.z, v.w}}; }

// A decay is exp2 of step A log2(e) and a little more, the nudge.  The GPU's approximate exp2 gives too little on average, which
// a state of slow decay adds up over its memory of 1 / |step A| steps.  Measured on the GB300, in 2^-24 of the result: 0.11
// at exponents of size below 0.002, 0.28 to 0.004, 0.44 to 0.016, 0.3 falling to 0.14 at 0.5; so much more in the exponent
// leaves a mean of some 0.05.  The size is taken at the first step of a tile.  (One nudge of 0.125 for all left three times the
// error of an exact exponential in dA at exponents of 0.005.)  A step of 0 still decays by exactly 1: what is added there is below
// half a unit.
__device__ __forceinline__ float nudge(float x) {
  constexpr float kUnit = 5.9604645e-8f * kLog2e;
  const float size = fabsf(x);
  return size < 0.002f * kLog2e ? 0.11f * kUnit : size < 0.004f * kLog2e || size > 0.016f * kLog2e ? 0.28f * kUnit : 0.44f * kUnit;
}
__device__ __forceinline__ Quad nudges(float step, const Quad& A2) {
  return {{nudge(step * A2.a.v[0]), nudge(step * A2.a.v[1])}, {nudge(step * A2.b.v[0]), nudge(step * A2.b.v[1])}};
}
__device__ __forceinline__ Vec<2> decay(float step, const Vec<2>& A2, const Vec<2>& more) {
  const Vec<2> x = fma<2>(splat<2>(step), A2, more);
  return {ex2(x.v[0]), ex2(x.v[1])};
}
// A state, or its gradient, after a split with this sum of steps: exp(sum A) state + last.  In two factors, which leave fp32 only
// where the product does (growing states).  They are kept above 0, so that an infinite state does not become NaN; nor does
// a state of 0 by growing.
__device__ __forceinline__ Quad after_split(float sum, const Quad& A2, const Quad& state, const Quad& last) {
  auto one = [sum](float a, float h, float more) {
    const float f = fmaxf(ex2(0.5f * sum * a), 1.4e-45f);
    return h == 0.0f ? more : fmaf(f, f * h, more);
  };
  return {{one(A2.a.v[0], state.a.v[0], last.a.v[0]), one(A2.a.v[1], state.a.v[1], last.a.v[1])},
          {one(A2.b.v[0], state.b.v[0], last.b.v[0]), one(A2.b.v[1], state.b.v[1], last.b.v[1])}};
}

// V neighbouring elements as they are in memory: in words where WIDE (all of them exist or none), else one by one, of which
// `there` exist.  (Loads that pack single elements would wait for each.)
template <typename E, int V, bool WIDE>
struct Raw {
  static constexpr bool kInWords = WIDE && V * sizeof(E) >= 4;
  static constexpr int kWords = kInWords ? V * int(sizeof(E)) / 4 : 1, kSingles = kInWords ? 1 : V;
  uint32_t w[kWords];
  E x[kSingles];
  __device__ __forceinline__ void read(const E* p, int there) {
    if constexpr (kInWords) {
#pragma unroll
      for (int i = 0; i < kWords; ++i) w[i] = 0;
      if (there <= 0) return;
      if constexpr (kWords >= 4) {
#pragma unroll
        for (int i = 0; i < kWords; i += 4) {
          const uint4 q = *reinterpret_cast<const uint4*>(p + i * 4 / int(sizeof(E)));
          w[i] = q.x, w[i + 1] = q.y, w[i + 2] = q.z, w[i + 3] = q.w;
        }
      } else if constexpr (kWords == 2) {
        const uint2 q = *reinterpret_cast<const uint2*>(p);
        w[0] = q.x, w[1] = q.y;
      } else {
        w[0] = *reinterpret_cast<const uint32_t*>(p);
      }
    } else {
#pragma unroll
      for (int k = 0; k < V; ++k) {
        x[k] = from_f32<E>(0.0f);
        if (k < there) x[k] = p[k];
      }
    }
  }
  __device__ __forceinline__ float operator[](int k) const {
    if constexpr (!kInWords) {
      return to_f32(x[k]);
    } else if constexpr (sizeof(E) == 4) {
      return __uint_as_float(w[k]);
    } else if constexpr (std::is_same_v<E, __nv_bfloat16>) {
      return __uint_as_float(k % 2 ? w[k / 2] & 0xffff0000u : w[k / 2] << 16);
    } else {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[k / 2]));
      return k % 2 ? f.y : f.x;
    }
  }
  template <int U>
  __device__ __forceinline__ Vec<U> at(int k) const {
    Vec<U> r;
#pragma unroll
    for (int i = 0; i < U; ++i) r.v[i] = (*this)[k + i];
    return r;
  }
};
template <typename E, int V, bool WIDE>
__device__ __forceinline__ void store_piece(E* p, int there, const float (&v)[V]) {
  if constexpr (Raw<E, V, WIDE>::kInWords) {
    constexpr int kBytes = V * int(sizeof(E)) < 16 ? V * int(sizeof(E)) : 16, kEach = kBytes / int(sizeof(E));
    if (there <= 0) return;
#pragma unroll
    for (int i = 0; i < V; i += kEach) {
      alignas(16) E e[kEach];
#pragma unroll
      for (int k = 0; k < kEach; ++k) e[k] = from_f32<E>(v[i + k]);
      if constexpr (kBytes == 16)
        *reinterpret_cast<uint4*>(p + i) = *reinterpret_cast<const uint4*>(e);
      else if constexpr (kBytes == 8)
        *reinterpret_cast<uint2*>(p + i) = *reinterpret_cast<const uint2*>(e);
      else
        *reinterpret_cast<uint32_t*>(p + i) = *reinterpret_cast<const uint32_t*>(e);
    }
  } else {
#pragma unroll
    for (int k = 0; k < V; ++k)
      if (k < there) p[k] = from_f32<E>(v[k]);
  }
}

// Four states from p on, of which `there` exist (WIDE: all or none).
template <bool WIDE>
__device__ __forceinline__ Quad load_quad(const float* p, int there) {
  float4 v = make_float4(0, 0, 0, 0);
  if constexpr (WIDE) {
    if (there > 0) v = *reinterpret_cast<const float4*>(p);
  } else {
    if (there > 0) v.x = p[0];
    if (there > 1) v.y = p[1];
    if (there > 2) v.z = p[2];
    if (there > 3) v.w = p[3];
  }
  return quad(v);
}
template <bool WIDE>
__device__ __forceinline__ void store_quad(float* p, int there, const Quad& q) {
  if constexpr (WIDE) {
    if (there > 0) *reinterpret_cast<float4*>(p) = make_float4(q.a.v[0], q.a.v[1], q.b.v[0], q.b.v[1]);
  } else {
    if (there > 0) p[0] = q.a.v[0];
    if (there > 1) p[1] = q.a.v[1];
    if (there > 2) p[2] = q.b.v[0];
    if (there > 3) p[3] = q.b.v[1];
  }
}

// How a block is laid out.
template <int LS_, int K_>
struct Shape {
  static constexpr int LS = LS_, K = K_;
  static constexpr int lanes = 32 / LS;            // channel lanes of a warp
  static constexpr int CH = kWarps * lanes * K;    // channels
  static constexpr int V = CH / 8;                 // channels of a staging thread (8 of them to a step),
  static constexpr int U = V > 1 ? 2 : 1;          // taken two at a time
  static constexpr int row = CH + 8;               // of the tiles' rows: steps lie 8 banks (floats) apart
  static constexpr int NP = kQuad * LS;            // states, padded
};

// The block's place, and a thread's in it.
template <typename S>
struct Place {
  int64_t b, n;              // sequence, its steps
  int64_t first, end;        // steps of the split
  int split, group, part;    // part: block of the group's channels
  int d0, channels;          // first channel and how many
  int states;                // N
  // staging: step and first channel of the piece
  int s, o, c0, there;
  // computing
  int g, quads;              // state quad, how many of its states exist
  int pos;                   // column of channel 0 in the tiles; channel k is k lanes further

  __device__ Place(const SsmArgs& p) {
    int64_t i = blockIdx.x;
    part = int(i % p.blocks);
    i /= p.blocks;
    group = int(i % p.in.G);
    i /= p.in.G;
    split = int(i % p.splits);
    b = i / p.splits;
    n = p.in.lengths ? min(max(int64_t(p.in.lengths[b]), int64_t(0)), p.in.T) : p.in.T;
    first = split * p.steps;
    end = min(first + p.steps, p.in.T);
    const int per = int(p.in.D / p.in.G);
    d0 = group * per + part * S::CH;
    channels = min(S::CH, per - part * S::CH);
    states = p.in.N;
    s = threadIdx.x / 8;
    o = threadIdx.x % 8;
    c0 = o * S::V;
    there = min(max(channels - c0, 0), S::V);
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    g = lane / S::lanes;
    quads = min(max(states - g * kQuad, 0), kQuad);
    pos = warp * S::K * S::lanes + lane % S::lanes;
  }
  // Column i of the tiles holds channel (i % 8) V + i / 8, so that both ways of access are free of conflicts.
  __device__ int channel(int k) const {
    const int i = pos + k * S::lanes;
    return i % 8 * S::V + i / 8;
  }
  __device__ bool has(int k) const { return channel(k) < channels; }
  // Of a [..][D][N] array's row: where the thread's states of channel k begin.
  __device__ int64_t state(int64_t row, int64_t D, int k) const { return (row * D + d0 + channel(k)) * states + g * kQuad; }
};

template <typename E>
__device__ __forceinline__ E* at(const gem_seq_t& s, int64_t b, int64_t t, int d) {
  return static_cast<E*>(s.data) + b * s.stride_b + t * s.stride_t + d;
}

// b and c of a tile, loaded ahead: a thread has quads of states of some steps.
template <typename E, typename S, bool WIDE, bool HAS_B, bool HAS_C>
struct States {
  static constexpr int each = (HAS_B && HAS_C ? 2 : 1) * kTile * S::LS / kSsmThreads > 0 ? (HAS_B && HAS_C ? 2 : 1) * kTile * S::LS / kSsmThreads : 1;
  static constexpr int total = (HAS_B && HAS_C ? 2 : 1) * kTile * S::LS;
  Raw<E, kQuad, WIDE> e[each];
  __device__ __forceinline__ void load(const SsmArgs& p, const Place<S>& a, int64_t t0) {
#pragma unroll
    for (int i = 0; i < each; ++i) {
      const int at_ = i * kSsmThreads + threadIdx.x, q = at_ % S::LS, s = at_ / S::LS % kTile;
      const bool is_c = !HAS_B || (HAS_C && at_ >= kTile * S::LS);
      const int there = at_ < total && t0 + s < a.n ? min(max(a.states - q * kQuad, 0), kQuad) : 0;
      const gem_seq_t& from = is_c ? p.in.c : p.in.b;
      e[i].read(at<E>(from, a.b, t0 + s, a.group * a.states + q * kQuad), there);
    }
  }
  // Into [HAS_B + HAS_C][kTile][LS] quads.
  __device__ __forceinline__ void stage(float4* to) const {
#pragma unroll
    for (int i = 0; i < each; ++i) {
      const int at_ = i * kSsmThreads + threadIdx.x;
      if (at_ < total) to[at_] = make_float4(e[i][0], e[i][1], e[i][2], e[i][3]);
    }
  }
};

// Bits of the tile's steps at which the state is dropped; steps past the end have none.
__device__ __forceinline__ unsigned resets_of(const SsmArgs& p, int64_t b, int64_t t0, int64_t end) {
  if (!p.in.reset) return 0u;
  const int64_t t = t0 + threadIdx.x % 32;
  return __ballot_sync(~0u, threadIdx.x % 32 < kTile && t < end && p.in.reset[b * p.in.T + t] != 0);
}

// Sums of v over the lanes that differ in the bits from LOW to HIGH (lane masks): the first N / lanes values of v
// are then those of the N sums from index N / lanes * (the lane's number among them) on; with more lanes than values,
// lanes with neighbouring numbers have the same one.
template <int N, int HIGH, int LOW>
__device__ __forceinline__ void scatter_sums(float (&v)[N]) {
  int count = N;
#pragma unroll
  for (int bit = HIGH; bit >= LOW; bit /= 2) {
    if (count == 1) {
      v[0] += __shfl_xor_sync(~0u, v[0], bit);
      continue;
    }
    const bool upper = threadIdx.x & bit;
    count /= 2;
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      if (i >= count) break;
      const float keep = upper ? v[count + i] : v[i], give = upper ? v[i] : v[count + i];
      v[i] = keep + __shfl_xor_sync(~0u, give, bit);
    }
  }
}

// How time and channels are cut (for kernels of CH channels a block, of which an SM holds `resident`).
struct SsmCut {
  int64_t blocks, splits, steps;
};
SsmCut ssm_cut(int64_t B, int64_t T, int64_t D, int G, int CH, bool backward, int resident);

template <typename E>
cudaError_t launch_forward(SsmArgs p, cudaStream_t stream);
template <typename E>
cudaError_t launch_backward(SsmArgs p, cudaStream_t stream);

// Shapes by N: LS lanes for 4 LS states.
inline int state_lanes(int N) { return N <= 16 ? 4 : N <= 32 ? 8 : 16; }
// Channels of a thread.  Two in the backward pass of more than 16 states: fewer instructions a state, but no more than two
// blocks an SM (both calls, 3 x 1777 x 1000 x 64: 711 us instead of 770 with one; with 16 states one is as fast or up to
// 10% faster).  One in the forward pass, bf16 in us with one and with two: 8 x 2048 x 2048 x 16 261, 430; x 32 400, 441; x 64 826, 853; 3
// x 1777 x 1000 x 64 173, 205.
constexpr int kForwardK = 1;
template <int LS>
constexpr int kBackwardK = LS == 4 ? 1 : 2;
template <int LS>
constexpr int kBackwardResident = LS == 4 ? 4 : 2;   // blocks of an SM
inline int backward_k(int LS) { return LS == 4 ? kBackwardK<4> : kBackwardK<16>; }
inline int backward_resident(int LS) { return LS == 4 ? kBackwardResident<4> : kBackwardResident<16>; }
inline int block_channels(int N, int K) { return kWarps * 32 / state_lanes(N) * K; }

}  // namespace ssm
}  // namespace lm
}  // namespace gem
