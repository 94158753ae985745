// Short causal convolution of each channel over time (include/gem_lm.h).
//
// A thread has K neighbouring channels and walks over a segment of time with the last W inputs in
// registers, so x is read once but for the W - 1 steps before a segment.  The backward pass walks forward
// as well: step t's dp_t goes to the gradients of the W inputs it used, the oldest of which is then complete; it
// goes W - 1 steps past the segment for that.  Sums for the weights are taken in registers over the
// segment, in shared memory over the block's warps, which may have several short sequences, and by a second kernel over the blocks, in that
// order.
//
// 8 x 4096 x 2048 bf16, W = 4, SiLU: forward 46 us (5.8 TB/s of input and output), backward 101 us (4.0 TB/s; 0.63 of the issue
// slots with 17 warps an SM, which wait for their own chains of products and for the copies), the parameters' sums 5.
#include <type_traits>

#include "lm_internal.h"

namespace gem {
namespace lm {
namespace {

constexpr int kConvWarps = 4;       // most segments of a block, a warp each
constexpr int kSegment = 64;        // steps of a segment
constexpr int kGroup = 4;           // steps that are taken together
constexpr float kLog2e = 1.4426950408889634f;

struct ConvArgs {
  gem_seq_t x, y;          // backward: y is dx
  gem_seq_t dy;
  const float *weight, *bias, *state;
  float* state_last;
  const float* dstate_last;
  float* dstate;
  float* partial;          // [rows of blocks][W + 1][D]
  const int32_t* lengths;
  const uint8_t* reset;
  int64_t T;
  int D, columns;          // blocks along the channels
  unsigned segments, total;   // of a sequence, of all
};

template <int V>
__device__ __forceinline__ Vec<V> sigmoid(const Vec<V>& v) {
  Vec<V> e = v * splat<V>(-kLog2e);
#pragma unroll
  for (int k = 0; k < V; ++k) asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e.v[k]) : "f"(e.v[k]));
  e = e + splat<V>(1.0f);
#pragma unroll
  for (int k = 0; k < V; ++k) asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(e.v[k]) : "f"(e.v[k]));
  return e;
}

// A thread's K channels: four or two as pairs, or one.
template <int K>
constexpr int kVec = K > 1 ? 2 : 1;
template <int K>
struct Channels {
  static constexpr int V = kVec<K>, P = K / V;
  Vec<V> c[P];
};
template <int K>
__device__ __forceinline__ Channels<K> none() {
  Channels<K> r;
#pragma unroll
  for (int i = 0; i < Channels<K>::P; ++i) r.c[i] = splat<Channels<K>::V>(0.0f);
  return r;
}

// K neighbouring elements as they are in memory, aligned to all K.
template <typename E, int K>
struct Raw;
template <typename E>
struct Raw<E, 1> {
  E x;
  __device__ __forceinline__ void read(const E* p) { x = *p; }
  __device__ __forceinline__ void clear() { x = from_f32<E>(0.0f); }
  __device__ __forceinline__ Channels<1> floats() const { return {{{to_f32(x)}}}; }
};
template <>
struct Raw<float, 4> {
  float4 x;
  __device__ __forceinline__ void read(const float* p) { x = *reinterpret_cast<const float4*>(p); }
  __device__ __forceinline__ Channels<4> floats() const { return {{{x.x, x.y}, {x.z, x.w}}}; }
};
template <typename E>
__device__ __forceinline__ Vec<2> two(uint32_t w) {
  if constexpr (std::is_same_v<E, __nv_bfloat16>) {
    return {__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)};
  } else {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
    return {f.x, f.y};
  }
}
template <typename E>
struct Raw<E, 4> {
  uint2 x;
  __device__ __forceinline__ void read(const E* p) { x = *reinterpret_cast<const uint2*>(p); }
  __device__ __forceinline__ Channels<4> floats() const { return {{two<E>(x.x), two<E>(x.y)}}; }
};
template <>
struct Raw<float, 2> {
  float2 x;
  __device__ __forceinline__ void read(const float* p) { x = *reinterpret_cast<const float2*>(p); }
  __device__ __forceinline__ Channels<2> floats() const { return {{{x.x, x.y}}}; }
};
template <typename E>
struct Raw<E, 2> {
  uint32_t x;
  __device__ __forceinline__ void read(const E* p) { x = *reinterpret_cast<const uint32_t*>(p); }
  __device__ __forceinline__ Channels<2> floats() const { return {{two<E>(x)}}; }
};
template <typename E, int K>
__device__ __forceinline__ void write_step(E* at, const Channels<K>& v) {
  if constexpr (K == 1) {
    *at = from_f32<E>(v.c[0].v[0]);
  } else if constexpr (K == 2 && sizeof(E) == 4) {
    *reinterpret_cast<float2*>(at) = make_float2(v.c[0].v[0], v.c[0].v[1]);
  } else if constexpr (K == 2) {
    alignas(4) E e[2] = {from_f32<E>(v.c[0].v[0]), from_f32<E>(v.c[0].v[1])};
    *reinterpret_cast<uint32_t*>(at) = *reinterpret_cast<const uint32_t*>(e);
  } else if constexpr (sizeof(E) == 4) {
    *reinterpret_cast<float4*>(at) = make_float4(v.c[0].v[0], v.c[0].v[1], v.c[1].v[0], v.c[1].v[1]);
  } else {
    alignas(8) E e[4] = {from_f32<E>(v.c[0].v[0]), from_f32<E>(v.c[0].v[1]), from_f32<E>(v.c[1].v[0]), from_f32<E>(v.c[1].v[1])};
    *reinterpret_cast<uint2*>(at) = *reinterpret_cast<const uint2*>(e);
  }
}

// What a warp works on.
struct ConvPlace {
  int64_t b, first, end, n;   // its steps [first, end) of the sequence's n
  int64_t row;                // the block's number along the segments of all sequences
  int d;                      // the thread's first channel
  bool on;
};
template <int K>
__device__ __forceinline__ ConvPlace conv_place(const ConvArgs& p) {
  ConvPlace a;
  a.row = blockIdx.x / p.columns;
  a.d = ((blockIdx.x % p.columns) * 32 + threadIdx.x % 32) * K;
  const unsigned segment = unsigned(a.row) * (blockDim.x / 32) + threadIdx.x / 32;
  const bool live = segment < p.total;   // (a block's other warps have no channels, and no steps)
  a.b = segment / p.segments;
  a.first = int64_t(segment % p.segments) * kSegment;
  a.end = min(a.first + kSegment, p.T);
  a.n = !live ? 0 : p.lengths ? min(max(int64_t(p.lengths[a.b]), int64_t(0)), p.T) : p.T;
  a.on = live && a.d < p.D;
  return a;
}

// The steps of a segment, and those around it that it looks at, at which the state is dropped.  One warp calls.
struct Resets {
  static constexpr int kBefore = 4;
  uint32_t bits[3];   // of steps first - kBefore + 32 i and on
  __device__ __forceinline__ Resets(const ConvArgs& p, const ConvPlace& a) {
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      const int64_t t = a.first - kBefore + 32 * i + threadIdx.x % 32;
      bits[i] = p.reset ? __ballot_sync(~0u, t >= 0 && t < a.n && p.reset[a.b * p.T + t] != 0) : 0u;
    }
  }
  // Of the segment's steps i to i + kGroup - 1, the lowest bit that of i.
  __device__ __forceinline__ unsigned group(int i) const {
    i += kBefore;
    const uint32_t low = i < 32 ? bits[0] : i < 64 ? bits[1] : bits[2], high = i < 32 ? bits[1] : i < 64 ? bits[2] : 0u;
    return __funnelshift_r(low, high, i % 32) & ((1u << kGroup) - 1);
  }
};

template <int W, int K>
struct Taps {
  Channels<K> w[W], bias;
  __device__ __forceinline__ void read(const ConvArgs& p, const ConvPlace& a) {
    bias = none<K>();
#pragma unroll
    for (int j = 0; j < W; ++j) w[j] = none<K>();
    if (!a.on) return;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (p.bias) bias.c[k / kVec<K>].v[k % kVec<K>] = p.bias[a.d + k];
#pragma unroll
      for (int j = 0; j < W; ++j) w[j].c[k / kVec<K>].v[k % kVec<K>] = p.weight[int64_t(a.d + k) * W + j];
    }
  }
};

// The last W inputs, oldest first; tap j reaches W - 1 - j steps back, at most `age` of which lie in the
// step's own document.
template <typename E, int W, int K>
struct Window {
  Channels<K> x[W];
  int age;

  // The inputs before the segment's first step (which lie in the sequence, or in its state).
  __device__ __forceinline__ void start(const ConvArgs& p, const ConvPlace& a, const Resets& resets, const E* row) {
    age = W;
#pragma unroll
    for (int j = 0; j < W; ++j) x[j] = none<K>();
#pragma unroll
    for (int j = 1; j < W; ++j) {
      const int64_t t = a.first - W + j;
      if (resets.group(j - W) & 1) drop();   // (none before step 0 or past the end)
      age = min(age + 1, W);
      if (!a.on) continue;
      if (t >= 0) {
        Raw<E, K> raw;
        raw.read(row + t * p.x.stride_t);
        x[j] = raw.floats();
      } else if (p.state) {
#pragma unroll
        for (int k = 0; k < K; ++k) x[j].c[k / kVec<K>].v[k % kVec<K>] = p.state[(a.b * (W - 1) + t + W - 1) * p.D + a.d + k];
      }
    }
  }
  // Every input so far counts as 0 from now on.
  __device__ __forceinline__ void drop() {
    age = -1;
#pragma unroll
    for (int j = 0; j < W; ++j) x[j] = none<K>();
  }
  __device__ __forceinline__ void push(const Raw<E, K>& raw) {
#pragma unroll
    for (int j = 0; j + 1 < W; ++j) x[j] = x[j + 1];
    x[W - 1] = raw.floats();
  }
};

// Feeds a thread the elements of N sequences, a group of steps at a time, loaded ahead.  Four or two channels: by
// asynchronous copies into places of the thread's own in shared memory (its registers are taken by sums and taps); one:
// into registers.  What lies past the last step, or a thread without channels gets, is not defined.
template <typename E>
constexpr int kStages = sizeof(E) == 2 ? 4 : 2;
template <typename E, int K, int N>
struct Feed {
  using Shared = Raw<E, K>[kStages<E>][N][kGroup][kConvWarps * 32];
  Shared& ring;
  const E* at[N];      // the next step to load
  int64_t stride[N];
  int left;            // steps not loaded yet (0 or less: none; of a thread without channels always)
  int stage = 0;
  __device__ __forceinline__ void issue(int to) {
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int u = 0; u < kGroup; ++u) {
        const uint32_t slot = static_cast<uint32_t>(__cvta_generic_to_shared(&ring[to][i][u][threadIdx.x]));
        if (u < left)
          asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(slot), "l"(at[i]), "n"(int(sizeof(Raw<E, K>))) : "memory");
        at[i] += stride[i];
      }
    asm volatile("cp.async.commit_group;" ::: "memory");
    left -= kGroup;
  }
  __device__ __forceinline__ void start() {
#pragma unroll
    for (int i = 0; i + 1 < kStages<E>; ++i) issue(i);
  }
  __device__ __forceinline__ void take(Raw<E, K> (&to)[N][kGroup]) {
    asm volatile("cp.async.wait_group %0;" ::"n"(kStages<E> - 2) : "memory");
    issue(stage == 0 ? kStages<E> - 1 : stage - 1);
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int u = 0; u < kGroup; ++u) to[i][u] = ring[stage][i][u][threadIdx.x];
    stage = stage + 1 == kStages<E> ? 0 : stage + 1;
  }
};
template <typename E, int N>
struct Feed<E, 1, N> {
  using Shared = int;
  Shared& ring;
  const E* at[N];
  int64_t stride[N];
  int left;
  int stage = 0;
  Raw<E, 1> ahead[N][kGroup];
  __device__ __forceinline__ void start() {
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int u = 0; u < kGroup; ++u) {
        ahead[i][u].clear();
        if (u < left) ahead[i][u].read(at[i]);
        at[i] += stride[i];
      }
    left -= kGroup;
  }
  __device__ __forceinline__ void take(Raw<E, 1> (&to)[N][kGroup]) {
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int u = 0; u < kGroup; ++u) to[i][u] = ahead[i][u];
    start();
  }
};
template <typename E, int K>
__device__ __forceinline__ void write_zeros(E* row, int64_t stride, const ConvPlace& a) {
  if (!a.on) return;
  for (int64_t t = max(a.first, a.n); t < a.end; ++t) write_step<E, K>(row + t * stride, none<K>());
}

template <int W, int K>
__device__ __forceinline__ Vec<kVec<K>> pre_activation(const Taps<W, K>& taps, const Channels<K> (&x)[W], int i) {
  Vec<kVec<K>> v = taps.bias.c[i];
#pragma unroll
  for (int j = 0; j < W; ++j) v = fma<kVec<K>>(taps.w[j].c[i], x[j].c[i], v);
  return v;
}

// A sequence's last inputs, by the warp whose segment it ends in (state_last may be state: only where one warp has
// the whole sequence, else conv_state_kernel writes them).
template <typename E, int W, int K, bool SILU>
__global__ void __launch_bounds__(kConvWarps * 32) conv_forward_kernel(const ConvArgs p) {
  __shared__ typename Feed<E, K, 1>::Shared ring;
  pdl_entry();
  const ConvPlace a = conv_place<K>(p);
  const int64_t end = min(a.end, a.n);
  const E* const row = static_cast<const E*>(p.x.data) + a.b * p.x.stride_b + a.d;
  E* const out = static_cast<E*>(p.y.data) + a.b * p.y.stride_b + a.d;
  const Resets resets(p, a);
  if (a.first < end || a.first == 0) {
    constexpr int V = kVec<K>, P = Channels<K>::P;
    Taps<W, K> taps;
    taps.read(p, a);
    Window<E, W, K> win;
    win.start(p, a, resets, row);
    const int own = int(end - a.first);
    Feed<E, K, 1> feed{ring, {row + a.first * p.x.stride_t}, {p.x.stride_t}, a.on ? own : 0};
    feed.start();
    E* to = out + a.first * p.y.stride_t;
    auto step = [&](const Raw<E, K>& raw) {
      win.push(raw);
      Channels<K> y;
#pragma unroll
      for (int i = 0; i < P; ++i) {
        y.c[i] = pre_activation<W, K>(taps, win.x, i);
        if (SILU) y.c[i] = y.c[i] * sigmoid<V>(y.c[i]);
      }
      if (a.on) write_step<E, K>(to, y);
      to += p.y.stride_t;
    };
    for (int i = 0; i < own; i += kGroup) {
      Raw<E, K> raw[1][kGroup];
      feed.take(raw);
      const unsigned drops = resets.group(i);
      if (i + kGroup <= own && drops == 0) {
#pragma unroll
        for (int u = 0; u < kGroup; ++u) step(raw[0][u]);
      } else {
#pragma unroll
        for (int u = 0; u < kGroup; ++u) {
          if (i + u >= own) break;
          if (drops >> u & 1) win.drop();
          step(raw[0][u]);
        }
      }
    }
    if (p.state_last && a.on) {
#pragma unroll
      for (int j = 1; j < W; ++j)
#pragma unroll
        for (int k = 0; k < K; ++k) p.state_last[(a.b * (W - 1) + j - 1) * p.D + a.d + k] = win.x[j].c[k / kVec<K>].v[k % kVec<K>];
    }
  }
  write_zeros<E, K>(out, p.y.stride_t, a);
}

template <typename E, int W>
__global__ void __launch_bounds__(128) conv_state_kernel(const ConvArgs p, int64_t count) {
  pdl_entry();
  const int64_t i = int64_t(blockIdx.x) * 128 + threadIdx.x;
  if (i >= count) return;
  const int64_t b = i / p.D, d = i % p.D;
  const int64_t n = p.lengths ? min(max(int64_t(p.lengths[b]), int64_t(0)), p.T) : p.T;
  float v[W - 1];
#pragma unroll
  for (int j = 0; j + 1 < W; ++j) {
    const int64_t t = n - (W - 1) + j;
    v[j] = t >= 0  ? to_f32(static_cast<const E*>(p.x.data)[b * p.x.stride_b + t * p.x.stride_t + d])
           : p.state ? p.state[(b * (W - 1) + t + W - 1) * p.D + d]
                     : 0.0f;
    for (int64_t s = max(t + 1, int64_t(0)); p.reset && s < n; ++s)
      if (p.reset[b * p.T + s]) v[j] = 0.0f;
  }
#pragma unroll
  for (int j = 0; j + 1 < W; ++j) p.state_last[(b * (W - 1) + j) * p.D + d] = v[j];
}

template <typename E, int W, int K, bool SILU>
__global__ void __launch_bounds__(kConvWarps * 32) conv_backward_kernel(const ConvArgs p) {
  pdl_entry();
  __shared__ typename Feed<E, K, 2>::Shared ring;
  __shared__ float sums[kConvWarps][W + 1][K][32];
  const ConvPlace a = conv_place<K>(p);
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int64_t end = min(a.end, a.n), reach = min(a.end + W - 1, a.n);
  const E* const row = static_cast<const E*>(p.x.data) + a.b * p.x.stride_b + a.d;
  const E* const dy = static_cast<const E*>(p.dy.data) + a.b * p.dy.stride_b + a.d;
  E* const out = static_cast<E*>(p.y.data) + a.b * p.y.stride_b + a.d;
  const Resets resets(p, a);
  constexpr int V = kVec<K>, P = Channels<K>::P;
  Channels<K> dw[W + 1];
#pragma unroll
  for (int j = 0; j <= W; ++j) dw[j] = none<K>();
  if (a.first < end || a.first == 0) {
    Taps<W, K> taps;
    taps.read(p, a);
    Window<E, W, K> win;
    win.start(p, a, resets, row);
    const int own = int(end - a.first), all = int(reach - a.first);
    Feed<E, K, 2> feed{ring, {row + a.first * p.x.stride_t, dy + a.first * p.dy.stride_t}, {p.x.stride_t, p.dy.stride_t}, a.on ? all : 0};
    feed.start();
    Channels<K> dx[W];   // gradients of the window's inputs
#pragma unroll
    for (int j = 0; j < W; ++j) dx[j] = none<K>();
    // the complete gradient of input t, which is the segment's, or the state's for the first one
    auto put = [&](int64_t t, const Channels<K>& v) {
      if (!a.on || t >= a.end) return;
      if (t >= a.first) {
        write_step<E, K>(out + t * p.y.stride_t, v);
      } else if (t < 0 && a.first == 0 && p.dstate) {
#pragma unroll
        for (int k = 0; k < K; ++k) p.dstate[(a.b * (W - 1) + t + W - 1) * p.D + a.d + k] = v.c[k / V].v[k % V];
      }
    };
    // one step: `whole`, all of its taps lie in its document; `mine`, it is the segment's own
    auto step = [&](const Raw<E, K>& raw_x, const Raw<E, K>& raw_g, bool whole, bool mine) {
      win.push(raw_x);
      const Channels<K> dy = raw_g.floats();
#pragma unroll
      for (int i = 0; i < P; ++i) {
        Vec<V> g = dy.c[i];
        if (SILU) {
          const Vec<V> v = pre_activation<W, K>(taps, win.x, i), s = sigmoid<V>(v), one = splat<V>(1.0f);
          g = g * (s * fma<V>(v, one - s, one));
        }
#pragma unroll
        for (int j = 0; j < W; ++j) {
          dx[j].c[i] = j + 1 < W ? dx[j + 1].c[i] : splat<V>(0.0f);
          if (whole || W - 1 - j <= win.age) dx[j].c[i] = fma<V>(g, taps.w[j].c[i], dx[j].c[i]);
          if (mine) dw[j].c[i] = fma<V>(g, win.x[j].c[i], dw[j].c[i]);
        }
        if (mine) dw[W].c[i] = dw[W].c[i] + g;
      }
    };
    E* to = out + (a.first - W + 1) * p.y.stride_t;   // where the input goes that a step completes
    for (int i = 0; i < all; i += kGroup) {
      Raw<E, K> raw[2][kGroup];
      feed.take(raw);
      const unsigned drops = resets.group(i);
      if (i + kGroup <= own && drops == 0 && win.age >= W - 2 && i >= W - 1) {
#pragma unroll
        for (int u = 0; u < kGroup; ++u) {
          step(raw[0][u], raw[1][u], true, true);
          if (a.on) write_step<E, K>(to, dx[0]);
          to += p.y.stride_t;
        }
        win.age = W;
      } else {
#pragma unroll
        for (int u = 0; u < kGroup; ++u) {
          if (i + u >= all) break;
          if (drops >> u & 1) win.drop();
          win.age = min(win.age + 1, W);
          step(raw[0][u], raw[1][u], false, i + u < own);   // (steps past the segment only complete its inputs' gradients)
          put(a.first + i + u - W + 1, dx[0]);
          to += p.y.stride_t;
        }
      }
    }
    if (reach == a.n) {   // the sequence ends here: no later step completes its last inputs
#pragma unroll
      for (int j = 1; j < W; ++j) {
        if (p.dstate_last && a.on && (a.n == 0 || W - 1 - j <= win.age)) {
#pragma unroll
          for (int k = 0; k < K; ++k) dx[j].c[k / V].v[k % V] += p.dstate_last[(a.b * (W - 1) + j - 1) * p.D + a.d + k];
        }
        put(a.n - W + j, dx[j]);
      }
    }
  }
  write_zeros<E, K>(out, p.y.stride_t, a);
  if (!p.partial) return;
#pragma unroll
  for (int j = 0; j <= W; ++j)
#pragma unroll
    for (int k = 0; k < K; ++k) sums[warp][j][k][lane] = dw[j].c[k / V].v[k % V];
  __syncthreads();
  if (warp != 0 || !a.on) return;
#pragma unroll
  for (int j = 0; j <= W; ++j)
#pragma unroll
    for (int k = 0; k < K; ++k) {
      float v = dw[j].c[k / V].v[k % V];
      for (int q = 1; q < int(blockDim.x) / 32; ++q) v += sums[q][j][k][lane];
      p.partial[(a.row * (W + 1) + j) * p.D + a.d + k] = v;
    }
}

// Sums of the blocks' partial sums: 32 channels of a tap by a block, of whose WARPS each takes every WARPS-th row.  Many rows
// want many warps: 1024 of them (1 x 262,144 x 256 bf16) 106 us for the whole backward call with 32 and 123 with 8; 128 (8 x 4096 x 2048) 5
// us with 8 and 9.5 with 32 for this kernel.
constexpr int64_t kManyRows = 256;
template <int WARPS>
__global__ void __launch_bounds__(WARPS * 32) conv_join_kernel(const float* partial, int64_t rows, int D, int W, float* dweight, float* dbias) {
  __shared__ float sums[WARPS][32];
  pdl_entry();
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, d = blockIdx.x * 32 + lane, j = blockIdx.y;
  float v = 0.0f;
  if (d < D)
#pragma unroll 8
    for (int64_t i = warp; i < rows; i += WARPS) v += partial[(i * (W + 1) + j) * D + d];
  sums[warp][lane] = v;
  __syncthreads();
  if (warp != 0 || d >= D) return;
#pragma unroll
  for (int w = 1; w < WARPS; ++w) v += sums[w][lane];
  if (j < W) {
    if (dweight) dweight[int64_t(d) * W + j] = v;
  } else if (dbias) {
    dbias[d] = v;
  }
}

// How sequences are cut: segments of one, of all, warps of a block, rows of blocks.  A block has the segments of one or several sequences,
// but one alone where blocks of four would not give every SM one (in a graph, bf16, us with one and with four: 16 x 1 x 2048 2.0, 2.3, backward 4.1,
// 4.8; 1 x 1000 x 2048 5.9, 6.1, backward 9.8, 10.5).  Blocks of one sequence each left short ones a row of sums for every sequence: 4096 x 64
// x 256, backward 192 instead of 100.
struct ConvCut {
  int64_t segments, total, warps, rows;
};
ConvCut conv_cut(int64_t B, int64_t T, int64_t D) {
  ConvCut c;
  c.segments = T < 1 ? 1 : (T + kSegment - 1) / kSegment;
  c.total = B * c.segments;
  c.warps = c.total * ((D + 63) / 64) < 152 * kConvWarps ? 1 : kConvWarps;
  c.rows = (c.total + c.warps - 1) / c.warps;
  return c;
}

bool conv_sizes_ok(int64_t B, int64_t T, int64_t D, int W) {
  if (W < 2 || W > 4 || !extent_ok(B) || !extent_ok(T) || !channels_ok(D)) return false;
  if (B == 0 || D == 0) return true;
  const int64_t columns = (D + 31) / 32, segments = T < 1 ? 1 : (T + kSegment - 1) / kSegment;
  return segments < kMaxExtent / B && columns <= (kMaxExtent - 1) / conv_cut(B, T, D).rows;   // a block at least for 32 channels and its warps
}

// Whether pieces of K channels of every step lie at multiples of their size.
bool in_pieces(const gem_seq_t& s, int dtype, int64_t B, int64_t T, int64_t D, int K) {
  return D % K == 0 && aligned_to(s.data, size_t(K * dtype_size(dtype))) && (B <= 1 || s.stride_b % K == 0) && (T <= 1 || s.stride_t % K == 0);
}

template <typename E, int W, int K>
cudaError_t launch_forward_as(ConvArgs p, int form, int64_t B, cudaStream_t stream) {
  const ConvCut cut = conv_cut(B, p.T, p.D);
  const bool whole = p.T <= kSegment;   // a warp has the whole sequence
  float* const state_last = p.state_last;
  if (!whole) p.state_last = nullptr;
  p.columns = (p.D + 32 * K - 1) / (32 * K);
  p.segments = unsigned(cut.segments);
  p.total = unsigned(cut.total);
  const dim3 grid(unsigned(cut.rows * p.columns)), block(unsigned(cut.warps * 32));
  const cudaError_t e = form == GEM_CONV_SILU ? launch_pdl(conv_forward_kernel<E, W, K, true>, grid, block, 0, stream, p)
                                              : launch_pdl(conv_forward_kernel<E, W, K, false>, grid, block, 0, stream, p);
  if (e != cudaSuccess || whole || !state_last) return e;
  p.state_last = state_last;
  return launch_pdl(conv_state_kernel<E, W>, dim3(unsigned((B * p.D + 127) / 128)), dim3(128), 0, stream, p, B * p.D);
}
template <typename E, int W, int K>
cudaError_t launch_backward_as(ConvArgs p, int form, int64_t B, cudaStream_t stream) {
  const ConvCut cut = conv_cut(B, p.T, p.D);
  p.columns = (p.D + 32 * K - 1) / (32 * K);
  p.segments = unsigned(cut.segments);
  p.total = unsigned(cut.total);
  const dim3 grid(unsigned(cut.rows * p.columns)), block(unsigned(cut.warps * 32));
  return form == GEM_CONV_SILU ? launch_pdl(conv_backward_kernel<E, W, K, true>, grid, block, 0, stream, p)
                               : launch_pdl(conv_backward_kernel<E, W, K, false>, grid, block, 0, stream, p);
}

// Channels of a thread: the most that the tensors' rows allow, 4, 2 or 1 (pieces).  The backward pass takes no more than two: its sums,
// taps and windows of four fill the registers (110 us instead of 98).
template <typename E, int W>
cudaError_t launch_conv_of(const ConvArgs& p, int form, int64_t B, int pieces, bool backward, cudaStream_t stream) {
  if (backward)
    return pieces > 1 ? launch_backward_as<E, W, 2>(p, form, B, stream) : launch_backward_as<E, W, 1>(p, form, B, stream);
  return pieces == 4   ? launch_forward_as<E, W, 4>(p, form, B, stream)
         : pieces == 2 ? launch_forward_as<E, W, 2>(p, form, B, stream)
                       : launch_forward_as<E, W, 1>(p, form, B, stream);
}
template <typename E>
cudaError_t launch_conv(const ConvArgs& p, int form, int64_t B, int W, int pieces, bool backward, cudaStream_t stream) {
  return W == 2   ? launch_conv_of<E, 2>(p, form, B, pieces, backward, stream)
         : W == 3 ? launch_conv_of<E, 3>(p, form, B, pieces, backward, stream)
                  : launch_conv_of<E, 4>(p, form, B, pieces, backward, stream);
}

}  // namespace
}  // namespace lm
}  // namespace gem

using namespace gem;
using namespace gem::lm;

extern "C" {

int gem_conv_forward(int dtype, int form, int64_t B, int64_t T, int64_t D, int W, const gem_seq_t* x,
                     const float* weight, const float* bias, const float* state,
                     const int32_t* lengths, const uint8_t* reset, const gem_seq_t* y,
                     float* state_last, void* stream) {
  if (!dtype_ok(dtype) || (form != GEM_CONV_LINEAR && form != GEM_CONV_SILU) || !conv_sizes_ok(B, T, D, W)) return GEM_EINVAL;
  if (!input_ok(x, dtype, B, T, D) || !output_ok(y, dtype, B, T, D)) return GEM_EINVAL;
  if (!optional_ok(bias) || !optional_ok(state) || !optional_ok(lengths) || !optional_ok(state_last)) return GEM_EINVAL;
  if (B == 0 || D == 0 || (T == 0 && !state_last)) return GEM_OK;
  if (!array_ok(weight)) return GEM_EINVAL;
  ConvArgs p = {};
  p.x = *x;
  p.y = *y;
  p.weight = weight;
  p.bias = bias;
  p.state = state;
  p.state_last = state_last;
  p.lengths = lengths;
  p.reset = reset;
  p.T = T;
  p.D = int(D);
  int pieces = 4;
  while (pieces > 1 && !(in_pieces(p.x, dtype, B, T, D, pieces) && in_pieces(p.y, dtype, B, T, D, pieces))) pieces /= 2;
  return launch_status(BY_TYPE(launch_conv, p, form, B, W, pieces, false, static_cast<cudaStream_t>(stream)));
}

int64_t gem_conv_workspace(int64_t B, int64_t T, int64_t D, int W) {
  if (!conv_sizes_ok(B, T, D, W)) return -1;
  return conv_cut(B, T, D).rows * (W + 1) * D;
}

int gem_conv_backward(int dtype, int form, int64_t B, int64_t T, int64_t D, int W,
                      const gem_seq_t* x, const float* weight, const float* bias,
                      const float* state, const int32_t* lengths, const uint8_t* reset,
                      const gem_seq_t* dy, const float* dstate_last, const gem_seq_t* dx,
                      float* dweight, float* dbias, float* dstate, float* workspace, void* stream) {
  if (!dtype_ok(dtype) || (form != GEM_CONV_LINEAR && form != GEM_CONV_SILU) || !conv_sizes_ok(B, T, D, W)) return GEM_EINVAL;
  if (!input_ok(x, dtype, B, T, D) || !input_ok(dy, dtype, B, T, D) || !output_ok(dx, dtype, B, T, D)) return GEM_EINVAL;
  if (!optional_ok(bias) || !optional_ok(state) || !optional_ok(lengths) || !optional_ok(dstate_last)) return GEM_EINVAL;
  if (!optional_ok(dweight) || !optional_ok(dbias) || !optional_ok(dstate) || !optional_ok(workspace)) return GEM_EINVAL;
  if (dstate && dstate == dstate_last) return GEM_EINVAL;   // (other warps read the one while this one writes the other)
  if (D == 0) return GEM_OK;
  if (B > 0 && !array_ok(weight)) return GEM_EINVAL;
  const bool sums = dweight || dbias;
  if (B > 0 && sums && !workspace) return GEM_EINVAL;
  ConvArgs p = {};
  p.x = *x;
  p.y = *dx;
  p.dy = *dy;
  p.weight = weight;
  p.bias = bias;
  p.state = state;
  p.dstate_last = dstate_last;
  p.dstate = dstate;
  p.partial = sums ? workspace : nullptr;
  p.lengths = lengths;
  p.reset = reset;
  p.T = T;
  p.D = int(D);
  const cudaStream_t on = static_cast<cudaStream_t>(stream);
  cudaError_t e = cudaSuccess;
  if (B > 0) {
    const bool pairs = in_pieces(p.x, dtype, B, T, D, 2) && in_pieces(p.dy, dtype, B, T, D, 2) && in_pieces(p.y, dtype, B, T, D, 2);
    e = BY_TYPE(launch_conv, p, form, B, W, pairs ? 2 : 1, true, on);
  }
  if (e == cudaSuccess && sums) {
    const int64_t rows = conv_cut(B, T, D).rows;
    const dim3 joins(unsigned((D + 31) / 32), unsigned(W + 1));
    const float* const partial = workspace;
    e = rows > kManyRows ? launch_pdl(conv_join_kernel<32>, joins, dim3(32 * 32), 0, on, partial, rows, int(D), W, dweight, dbias)
                         : launch_pdl(conv_join_kernel<8>, joins, dim3(8 * 32), 0, on, partial, rows, int(D), W, dweight, dbias);
  }
  return launch_status(e);
}

}  // extern "C"
