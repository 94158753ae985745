// Gated linear recurrence (include/gem_lm.h): h_t = a_t h_{t-1} + u_t with a = sigmoid(f) and
// u = (1 - a) x or x, and its backward pass.
#include <cooperative_groups.h>

#include "lm_internal.h"

namespace cg = cooperative_groups;

namespace gem {
namespace lm {
namespace {

constexpr int kChunk = GEM_GLR_CHUNK;

struct GlrArgs {
  gem_seq_t x, f, h, dh, dx, df;
  const float* h0;
  const int32_t* lengths;
  const uint8_t* reset;
  const float* saved_in;
  float* saved_out;
  float* h_last;
  const float* dh_last;
  float* dh0;
  int64_t B, T, D;
};

template <typename E>
__device__ __forceinline__ E* at(const gem_seq_t& s, int64_t b, int64_t t, int64_t d) {
  return static_cast<E*>(s.data) + b * s.stride_b + t * s.stride_t + d;
}

__device__ __forceinline__ int64_t steps_of(const GlrArgs& p, int64_t b) {
  if (!p.lengths) return p.T;
  const int64_t n = p.lengths[b];
  return n < 0 ? 0 : n > p.T ? p.T : n;
}

// a = sigmoid(f) and b = 1 - a = sigmoid(-f), each to its own relative precision: with e = exp(-f),
// a = 1 / (1 + e) and b = e a.  f below -80 counts as -80 (a = 2e-35): e stays finite.  NaN stays.
template <typename E>
__device__ __forceinline__ void gate(float f, float& a, float& b) {
  asm("max.NaN.f32 %0, %0, 0fC2A00000;" : "+f"(f));
  // 16-bit inputs carry 2^-9 themselves; the fast exponential's 2 + |f| units are far below that
  const float e = sizeof(E) == 4 ? expf(-f) : __expf(-f);
  a = __fdividef(1.0f, 1.0f + e);
  b = e * a;
}

// ---- a few steps: one thread per channel, one step after the other ----

template <typename E, bool LERP>
__global__ void glr_step_kernel(const GlrArgs p) {
  pdl_entry();
  const int64_t i = int64_t(blockIdx.x) * blockDim.x + threadIdx.x;
  if (i >= p.B * p.D) return;
  const int64_t b = i / p.D, d = i % p.D;
  const int64_t n = steps_of(p, b);
  float h = p.h0 ? p.h0[i] : 0.0f;
  if (p.saved_out && p.T > 0) p.saved_out[i] = h;
  for (int64_t t = 0; t < p.T; ++t) {
    float shown = 0.0f;
    if (t < n) {
      float a, c;
      gate<E>(to_f32(*at<const E>(p.f, b, t, d)), a, c);
      const float x = to_f32(*at<const E>(p.x, b, t, d));
      const float u = LERP ? c * x : x;
      h = p.reset && p.reset[b * p.T + t] ? u : fmaf(a, h, u);
      shown = h;
    }
    *at<E>(p.h, b, t, d) = from_f32<E>(shown);
  }
  if (p.h_last) p.h_last[i] = h;
}
constexpr int64_t kStepT = 2;   // longest call of the kernel above (one chunk: saved is h0)

// ---- tiles: a scan over time in registers, warps, blocks and rounds ----
//
// A step is the map h -> a h + u; maps compose, (A2, H2) after (A1, H1) being (A2 A1, A2 H1 + H2).
// A thread takes kChunk steps of one 4-byte word of channels (two 16-bit ones or one), composes
// their map, and applies the steps once it knows the state before them.  A warp is 32 words side by
// side, 128 bytes of a row; the block's warps are consecutive chunks of time, the blocks of a
// cluster consecutive groups of those, and the cluster goes over the sequence in rounds with the
// state carried from one to the next.  Per round: one barrier of the block, after which every
// thread composes the earlier warps' maps from shared memory, and in a cluster one exchange of the
// blocks' maps over distributed shared memory.  Every element is read and written once.
//
// The copies of a thread's next rounds are in flight while it works (cp.async into slots of its
// own, which need no barrier), so memory does not wait for the scan.
//
// A map whose steps contain a reset has A = -1: it forgets the state whatever that holds (0 times
// an infinity would not).

constexpr int kMaxWarps = 8;

template <int V>
struct Map {
  float A[V], H[V];
};

template <int V>
__device__ __forceinline__ void apply(float (&h)[V], const Map<V>& m) {
#pragma unroll
  for (int v = 0; v < V; ++v) h[v] = m.A[v] < 0.0f ? m.H[v] : fmaf(m.A[v], h[v], m.H[v]);
}

// m after the maps composed so far.
template <int V>
__device__ __forceinline__ void compose(Map<V>& sofar, const Map<V>& m) {
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const bool forgets = m.A[v] < 0.0f;
    sofar.H[v] = forgets ? m.H[v] : fmaf(m.A[v], sofar.H[v], m.H[v]);
    sofar.A[v] = forgets || sofar.A[v] < 0.0f ? -1.0f : sofar.A[v] * m.A[v];
  }
}

// From every thread's map of a round: the state before the thread's chunk, and `state` moved on to
// the state after the round.  maps: [2][kMaxWarps][32], blocks: [2][C][32] (C > 1) in shared memory.
template <int V>
__device__ __forceinline__ void scan_round(const Map<V>& own, int round, int warps, int rank, int C, Map<V>* maps,
                                           Map<V>* blocks, float (&state)[V], float (&before)[V]) {
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  Map<V>* buf = maps + (round & 1) * kMaxWarps * 32;
  buf[warp * 32 + lane] = own;
  __syncthreads();
  if (C == 1) {
    for (int w = 0; w < warps; ++w) {
      if (w == warp) {
#pragma unroll
        for (int v = 0; v < V; ++v) before[v] = state[v];
      }
      apply<V>(state, buf[w * 32 + lane]);
    }
    return;
  }
  Map<V> all, mine;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    all.A[v] = 1.0f;
    all.H[v] = 0.0f;
  }
  mine = all;
  for (int w = 0; w < warps; ++w) {
    if (w == warp) mine = all;
    compose<V>(all, buf[w * 32 + lane]);
  }
  cg::cluster_group cluster = cg::this_cluster();
  Map<V>* out = blocks + (round & 1) * C * 32;
  for (int c = warp; c < C; c += warps) cluster.map_shared_rank(out, c)[rank * 32 + lane] = all;
  cluster.sync();
  for (int c = 0; c < C; ++c) {
    if (c == rank) {
#pragma unroll
      for (int v = 0; v < V; ++v) before[v] = state[v];
    }
    apply<V>(state, out[c * 32 + lane]);
  }
  apply<V>(before, mine);
}

// V elements of one word.
template <typename E, int V>
__device__ __forceinline__ void unpack(uint32_t w, float (&v)[V]) {
  if constexpr (sizeof(E) == 4) {
    v[0] = __uint_as_float(w);
  } else {
    const E* e = reinterpret_cast<const E*>(&w);
#pragma unroll
    for (int k = 0; k < V; ++k) v[k] = to_f32(e[k]);
  }
}

template <typename E, int V>
__device__ __forceinline__ void store(E* at, const float (&v)[V]) {
  if constexpr (V == 2) {
    E e[2] = {from_f32<E>(v[0]), from_f32<E>(v[1])};
    *reinterpret_cast<uint32_t*>(at) = *reinterpret_cast<uint32_t*>(e);
  } else {
    *at = from_f32<E>(v[0]);
  }
}

// Copies one word of channels to a slot of the calling thread: asynchronously where it is 4 bytes
// at a 4-byte boundary, else (one 16-bit channel) through a register.
template <typename E, int V>
__device__ __forceinline__ void fetch(uint32_t* slot, const E* from) {
  if constexpr (sizeof(E) * V == 4) {
    const uint32_t s = static_cast<uint32_t>(__cvta_generic_to_shared(slot));
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(s), "l"(from) : "memory");
  } else {
    *reinterpret_cast<E*>(slot) = *from;
  }
}
__device__ __forceinline__ void fetch_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void fetch_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// Bit k: a reset at step t0 + k (k < m).  All lanes of the warp call.
__device__ __forceinline__ uint32_t reset_bits(const GlrArgs& p, int64_t b, int64_t t0, int m) {
  if (!p.reset) return 0;
  const int lane = threadIdx.x % 32;
  const bool r = lane < m && p.reset[b * p.T + t0 + lane] != 0;
  return __ballot_sync(~0u, r);
}

// Where a thread works: sequence b, channels d.., the rank of its block in the cluster.
struct Place {
  int64_t b, d;
  int rank, warp, warps;
  bool on;
};

template <int V>
__device__ __forceinline__ Place place_of(const GlrArgs& p, int C) {
  Place w;
  const int64_t words = (p.D + 32 * V - 1) / (32 * V);
  const int64_t id = blockIdx.x / C;
  w.rank = blockIdx.x % C;
  w.b = id / words;
  w.d = (id % words * 32 + threadIdx.x % 32) * V;
  w.on = w.d < p.D;
  w.warp = threadIdx.x / 32;
  w.warps = blockDim.x / 32;
  return w;
}

constexpr int kForwardStages = 3;

template <typename E, int V, bool LERP>
__global__ void __launch_bounds__(kMaxWarps * 32, 2) glr_forward_kernel(const GlrArgs p, int C) {
  extern __shared__ __align__(16) uint32_t slots[];   // [stage][x, f][kChunk][threads], then the blocks' maps
  __shared__ Map<V> maps[2 * kMaxWarps * 32];
  Map<V>* blocks = reinterpret_cast<Map<V>*>(slots + kForwardStages * 2 * kChunk * blockDim.x);
  pdl_entry();
  const Place w = place_of<V>(p, C);
  const int64_t n = steps_of(p, w.b);
  const int threads = blockDim.x;
  const int64_t chunks = (n + kChunk - 1) / kChunk, all_chunks = (p.T + kChunk - 1) / kChunk;
  const int64_t per_round = int64_t(w.warps) * C;
  const int rounds = int((chunks + per_round - 1) / per_round);
  const int64_t first = int64_t(w.rank) * w.warps + w.warp;   // chunk of round 0
  const E* x = at<const E>(p.x, w.b, 0, w.d);
  const E* f = at<const E>(p.f, w.b, 0, w.d);
  E* h_out = at<E>(p.h, w.b, 0, w.d);
  const int64_t state_at = w.b * p.D + w.d;
  float state[V];
#pragma unroll
  for (int v = 0; v < V; ++v) state[v] = p.h0 && w.on ? p.h0[state_at + v] : 0.0f;

  auto slot = [&](int stage, int what, int k) { return slots + ((stage * 2 + what) * kChunk + k) * threads + threadIdx.x; };
  auto issue = [&](int round) {
    const int64_t c = first + round * per_round;
    if (round < rounds && c < chunks && w.on) {
      const int64_t t0 = c * kChunk;
      const int m = int(n - t0 < kChunk ? n - t0 : kChunk);
      const int stage = round % kForwardStages;
      const E* xs = x + t0 * p.x.stride_t;
      const E* fs = f + t0 * p.f.stride_t;
#pragma unroll
      for (int k = 0; k < kChunk; ++k) {
        if (k < m) {
          fetch<E, V>(slot(stage, 0, k), xs);
          fetch<E, V>(slot(stage, 1, k), fs);
        }
        xs += p.x.stride_t;
        fs += p.f.stride_t;
      }
    }
    fetch_commit();
  };
#pragma unroll
  for (int r = 0; r < kForwardStages - 1; ++r) issue(r);

  for (int round = 0; round < rounds; ++round) {
    issue(round + kForwardStages - 1);
    const int64_t c = first + round * per_round, t0 = c * kChunk;
    const bool busy = c < chunks;
    const int m = busy ? int(n - t0 < kChunk ? n - t0 : kChunk) : 0;
    const uint32_t fresh = reset_bits(p, w.b, t0, m);
    const bool plain = m == kChunk && fresh == 0;
    fetch_wait<kForwardStages - 1>();
    const int stage = round % kForwardStages;
    float a[kChunk][V], u[kChunk][V];
    Map<V> own;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      own.A[v] = 1.0f;
      own.H[v] = 0.0f;
    }
#pragma unroll
    for (int k = 0; k < kChunk; ++k) {
      float xv[V], fv[V];
      unpack<E, V>(*slot(stage, 0, k), xv);
      unpack<E, V>(*slot(stage, 1, k), fv);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        float g;
        gate<E>(fv[v], a[k][v], g);
        u[k][v] = LERP ? g * xv[v] : xv[v];
        if (!plain && k >= m) {
          a[k][v] = 1.0f;
          u[k][v] = 0.0f;
        }
        own.H[v] = !plain && (fresh >> k & 1) ? u[k][v] : fmaf(a[k][v], own.H[v], u[k][v]);
        own.A[v] *= a[k][v];
      }
    }
    if (fresh) {
#pragma unroll
      for (int v = 0; v < V; ++v) own.A[v] = -1.0f;
    }
    float h[V];
    scan_round<V>(own, round, w.warps, w.rank, C, maps, blocks, state, h);
    if (!busy || !w.on) continue;
    if (p.saved_out) {
      float* s = p.saved_out + (w.b * all_chunks + c) * p.D + w.d;
#pragma unroll
      for (int v = 0; v < V; ++v) s[v] = h[v];
    }
    E* out = h_out + t0 * p.h.stride_t;
#pragma unroll
    for (int k = 0; k < kChunk; ++k) {
#pragma unroll
      for (int v = 0; v < V; ++v) h[v] = !plain && (fresh >> k & 1) ? u[k][v] : fmaf(a[k][v], h[v], u[k][v]);
      if (plain || k < m) store<E, V>(out, h);
      out += p.h.stride_t;
    }
  }
  // all have read h0 before it is replaced (rounds have barriers of their own)
  if (rounds == 0) C == 1 ? __syncthreads() : cg::this_cluster().sync();
  if (!w.on) return;
  // past the sequence's end: zeros, and the state as it stays
  float zero[V] = {};
  for (int64_t t = n + first; t < p.T; t += per_round) store<E, V>(h_out + t * p.h.stride_t, zero);
  if (p.saved_out)
    for (int64_t c = chunks + first; c < all_chunks; c += per_round)
#pragma unroll
      for (int v = 0; v < V; ++v) p.saved_out[(w.b * all_chunks + c) * p.D + w.d + v] = state[v];
  if (p.h_last && first == 0) {
#pragma unroll
    for (int v = 0; v < V; ++v) p.h_last[state_at + v] = state[v];
  }
}

// Backward: the same scan from the end.  A step's map is g -> a (dh + g), g being what the step
// after it hands back.  The states before the chunk's steps are computed again from the saved one.
constexpr int kBackwardStages = 2;

template <typename E, int V, bool LERP>
__global__ void __launch_bounds__(kMaxWarps * 32, 2) glr_backward_kernel(const GlrArgs p, int C) {
  constexpr int kWords = 3 * kChunk + V;
  extern __shared__ __align__(16) uint32_t slots[];   // [stage][x, f, dh: kChunk each, saved: V][threads], then the blocks' maps
  __shared__ Map<V> maps[2 * kMaxWarps * 32];
  Map<V>* blocks = reinterpret_cast<Map<V>*>(slots + kBackwardStages * kWords * blockDim.x);
  pdl_entry();
  const Place w = place_of<V>(p, C);
  const int64_t n = steps_of(p, w.b);
  const int threads = blockDim.x;
  const int64_t chunks = (n + kChunk - 1) / kChunk, all_chunks = (p.T + kChunk - 1) / kChunk;
  const int64_t per_round = int64_t(w.warps) * C;
  const int rounds = int((chunks + per_round - 1) / per_round);
  const int64_t first = int64_t(w.rank) * w.warps + w.warp;   // chunks are counted from the end
  const E* x = at<const E>(p.x, w.b, 0, w.d);
  const E* f = at<const E>(p.f, w.b, 0, w.d);
  const E* dh = at<const E>(p.dh, w.b, 0, w.d);
  E* dx_out = at<E>(p.dx, w.b, 0, w.d);
  E* df_out = at<E>(p.df, w.b, 0, w.d);
  const int64_t state_at = w.b * p.D + w.d;
  float state[V];
#pragma unroll
  for (int v = 0; v < V; ++v) state[v] = p.dh_last && w.on ? p.dh_last[state_at + v] : 0.0f;

  auto slot = [&](int stage, int word) { return slots + (stage * kWords + word) * threads + threadIdx.x; };
  auto issue = [&](int round) {
    const int64_t l = first + round * per_round;
    if (round < rounds && l < chunks && w.on) {
      const int64_t c = chunks - 1 - l, t0 = c * kChunk;
      const int m = int(n - t0 < kChunk ? n - t0 : kChunk);
      const int stage = round % kBackwardStages;
      const E* xs = x + t0 * p.x.stride_t;
      const E* fs = f + t0 * p.f.stride_t;
      const E* ds = dh + t0 * p.dh.stride_t;
#pragma unroll
      for (int k = 0; k < kChunk; ++k) {
        if (k < m) {
          fetch<E, V>(slot(stage, k), xs);
          fetch<E, V>(slot(stage, kChunk + k), fs);
          fetch<E, V>(slot(stage, 2 * kChunk + k), ds);
        }
        xs += p.x.stride_t;
        fs += p.f.stride_t;
        ds += p.dh.stride_t;
      }
#pragma unroll
      for (int v = 0; v < V; ++v)
        fetch<float, 1>(slot(stage, 3 * kChunk + v), p.saved_in + (w.b * all_chunks + c) * p.D + w.d + v);
    }
    fetch_commit();
  };
#pragma unroll
  for (int r = 0; r < kBackwardStages - 1; ++r) issue(r);

  for (int round = 0; round < rounds; ++round) {
    issue(round + kBackwardStages - 1);
    const int64_t l = first + round * per_round, c = chunks - 1 - l, t0 = c * kChunk;
    const bool busy = l < chunks;
    const int m = busy ? int(n - t0 < kChunk ? n - t0 : kChunk) : 0;
    const uint32_t fresh = reset_bits(p, w.b, t0, m);
    const bool plain = m == kChunk && fresh == 0;
    fetch_wait<kBackwardStages - 1>();
    const int stage = round % kBackwardStages;
    // a, b = 1 - a, and what the gate's gradient multiplies: h_{t-1} - x_t, or h_{t-1}
    float a[kChunk][V], b[kChunk][V], q[kChunk][V], h[V];
#pragma unroll
    for (int v = 0; v < V; ++v) h[v] = __uint_as_float(*slot(stage, 3 * kChunk + v));
#pragma unroll
    for (int k = 0; k < kChunk; ++k) {
      float xv[V], fv[V];
      unpack<E, V>(*slot(stage, k), xv);
      unpack<E, V>(*slot(stage, kChunk + k), fv);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        gate<E>(fv[v], a[k][v], b[k][v]);
        const float u = LERP ? b[k][v] * xv[v] : xv[v];
        const bool r = !plain && (fresh >> k & 1);
        q[k][v] = (r ? 0.0f : h[v]) - (LERP ? xv[v] : 0.0f);
        h[v] = r ? u : fmaf(a[k][v], h[v], u);
      }
    }
    Map<V> own;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      own.A[v] = 1.0f;
      own.H[v] = 0.0f;
    }
#pragma unroll
    for (int k = kChunk - 1; k >= 0; --k) {
      float dv[V];
      unpack<E, V>(*slot(stage, 2 * kChunk + k), dv);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        if (plain || k < m) {
          own.H[v] = !plain && (fresh >> k & 1) ? 0.0f : a[k][v] * (dv[v] + own.H[v]);
          own.A[v] *= a[k][v];
        }
      }
    }
    if (fresh) {
#pragma unroll
      for (int v = 0; v < V; ++v) own.A[v] = -1.0f;
    }
    float g[V];
    scan_round<V>(own, round, w.warps, w.rank, C, maps, blocks, state, g);
    if (!busy || !w.on) continue;
    E* dxs = dx_out + t0 * p.dx.stride_t;
    E* dfs = df_out + t0 * p.df.stride_t;
#pragma unroll
    for (int k = kChunk - 1; k >= 0; --k) {
      if (!plain && k >= m) continue;
      float dv[V], dx[V], df[V];
      unpack<E, V>(*slot(stage, 2 * kChunk + k), dv);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        g[v] += dv[v];
        dx[v] = LERP ? b[k][v] * g[v] : g[v];
        df[v] = g[v] * q[k][v] * (a[k][v] * b[k][v]);
        g[v] = !plain && (fresh >> k & 1) ? 0.0f : a[k][v] * g[v];
      }
      store<E, V>(dxs + k * p.dx.stride_t, dx);
      store<E, V>(dfs + k * p.df.stride_t, df);
    }
  }
  if (rounds == 0) C == 1 ? __syncthreads() : cg::this_cluster().sync();
  if (!w.on) return;
  float zero[V] = {};
  for (int64_t t = n + first; t < p.T; t += per_round) {
    store<E, V>(dx_out + t * p.dx.stride_t, zero);
    store<E, V>(df_out + t * p.df.stride_t, zero);
  }
  if (p.dh0 && first == 0) {
#pragma unroll
    for (int v = 0; v < V; ++v) p.dh0[state_at + v] = state[v];
  }
}

// How the work is cut: warps of a block and blocks of a cluster are taken only as far as there are
// chunks for them, and a cluster is as small as gives the GPU about 16 warps per SM (each with
// copies of 8 KB and more in flight).
struct Cut {
  int warps, cluster;
  int64_t blocks;
};

Cut cut(const GlrArgs& p, int V) {
  const int64_t chunks = (p.T + kChunk - 1) / kChunk;
  const int64_t words = (p.D + 32 * V - 1) / (32 * V);
  Cut c;
  c.warps = int(chunks < 1 ? 1 : chunks < kMaxWarps ? chunks : kMaxWarps);
  c.cluster = 1;
  while (c.cluster < 8 && words * p.B * c.cluster * c.warps < 152 * 16 && int64_t(c.cluster) * c.warps < chunks) c.cluster *= 2;
  c.blocks = words * p.B * c.cluster;
  return c;
}

template <typename E, int V, bool LERP>
cudaError_t launch_tiles(const GlrArgs& p, bool backward, cudaStream_t stream) {
  const Cut c = cut(p, V);
  auto* kernel = backward ? glr_backward_kernel<E, V, LERP> : glr_forward_kernel<E, V, LERP>;
  const size_t smem = size_t(c.warps) * 32 * 4 * (backward ? kBackwardStages * (3 * kChunk + V) : kForwardStages * 2 * kChunk) +
                      (c.cluster > 1 ? size_t(2) * c.cluster * 32 * sizeof(Map<V>) : 0);
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, int(smem));
  if (e != cudaSuccess) return e;
  return launch_cluster_pdl(kernel, unsigned(c.blocks), unsigned(c.warps * 32), unsigned(c.cluster), smem, stream, p, c.cluster);
}

template <typename E>
cudaError_t launch(const GlrArgs& p, int form, bool backward, cudaStream_t stream) {
  const bool lerp = form == GEM_GLR_LERP;
  if (!backward && p.T <= kStepT) {
    const int64_t blocks = (p.B * p.D + 127) / 128;
    return launch_pdl(lerp ? glr_step_kernel<E, true> : glr_step_kernel<E, false>, dim3(unsigned(blocks)), dim3(128), 0, stream, p);
  }
  if constexpr (sizeof(E) == 4) {
    return lerp ? launch_tiles<E, 1, true>(p, backward, stream) : launch_tiles<E, 1, false>(p, backward, stream);
  } else {
    // pairs of channels where every row of every tensor starts at a 4-byte boundary
    bool pairs = p.D % 2 == 0;
    for (const gem_seq_t* s : {&p.x, &p.f, backward ? &p.dh : &p.h, backward ? &p.dx : &p.h, backward ? &p.df : &p.h})
      pairs = pairs && aligned_to(s->data, 4) && (p.B == 1 || s->stride_b % 2 == 0) && (p.T == 1 || s->stride_t % 2 == 0);
    if (pairs) return lerp ? launch_tiles<E, 2, true>(p, backward, stream) : launch_tiles<E, 2, false>(p, backward, stream);
    return lerp ? launch_tiles<E, 1, true>(p, backward, stream) : launch_tiles<E, 1, false>(p, backward, stream);
  }
}

cudaError_t launch_glr(int dtype, const GlrArgs& p, int form, bool backward, cudaStream_t stream) {
  switch (dtype) {
    case GEM_F32: return launch<float>(p, form, backward, stream);
    case GEM_BF16: return launch<__nv_bfloat16>(p, form, backward, stream);
    default: return launch<__half>(p, form, backward, stream);
  }
}

bool sizes_ok(int dtype, int form, int64_t B, int64_t T, int64_t D) {
  if (!dtype_ok(dtype) || (form != GEM_GLR_LERP && form != GEM_GLR_ADD)) return false;
  if (!extent_ok(B) || !extent_ok(T) || !extent_ok(D)) return false;
  return B == 0 || (D + 31) / 32 <= (int64_t(1) << 27) / B;   // a grid of clusters of up to 8 blocks
}

// An input: any strides (0: one step or sequence for all).
bool input_ok(const gem_seq_t* s, int dtype, int64_t B, int64_t T, int64_t D) {
  if (!s) return false;
  if (B == 0 || T == 0 || D == 0) return true;
  if (!s->data || !aligned_to(s->data, size_t(dtype_size(dtype)))) return false;
  if (B > 1 && (s->stride_b < 0 || s->stride_b > kMaxStride / B)) return false;
  if (T > 1 && (s->stride_t < 0 || s->stride_t > kMaxStride / T)) return false;
  return true;
}

// An output: its elements also have places of their own.
bool output_ok(const gem_seq_t* s, int dtype, int64_t B, int64_t T, int64_t D) {
  if (!input_ok(s, dtype, B, T, D)) return false;
  if (B == 0 || T == 0 || D == 0) return true;
  const int64_t sb = s->stride_b, st = s->stride_t;
  if (T == 1) return B == 1 || sb >= D;
  if (B == 1) return st >= D;
  return (st >= D && sb >= (T - 1) * st + D) || (sb >= D && st >= (B - 1) * sb + D);
}

}  // namespace
}  // namespace lm
}  // namespace gem

using namespace gem::lm;

extern "C" {

int64_t gem_glr_saved_count(int64_t B, int64_t T, int64_t D) {
  if (!extent_ok(B) || !extent_ok(T) || !extent_ok(D)) return -1;
  const int64_t chunks = (T + kChunk - 1) / kChunk;
  if (B == 0 || chunks == 0 || D == 0) return 0;
  return D > INT64_MAX / 4 / B / chunks ? -1 : B * chunks * D;
}

int gem_glr_forward(int dtype, int form, int64_t B, int64_t T, int64_t D, const gem_seq_t* x,
                    const gem_seq_t* f, const float* h0, const int32_t* lengths,
                    const uint8_t* reset, const gem_seq_t* h, float* h_last, float* saved,
                    void* stream) {
  if (!sizes_ok(dtype, form, B, T, D)) return GEM_EINVAL;
  if (!input_ok(x, dtype, B, T, D) || !input_ok(f, dtype, B, T, D) || !output_ok(h, dtype, B, T, D))
    return GEM_EINVAL;
  if (!optional_ok(h0) || !optional_ok(lengths) || !optional_ok(h_last) || !optional_ok(saved))
    return GEM_EINVAL;
  if (B == 0 || D == 0 || (T == 0 && !h_last)) return GEM_OK;
  GlrArgs p = {};
  p.x = *x;
  p.f = *f;
  p.h = *h;
  p.h0 = h0;
  p.lengths = lengths;
  p.reset = reset;
  p.h_last = h_last;
  p.saved_out = saved;
  p.B = B;
  p.T = T;
  p.D = D;
  return launch_status(launch_glr(dtype, p, form, false, static_cast<cudaStream_t>(stream)));
}

int gem_glr_backward(int dtype, int form, int64_t B, int64_t T, int64_t D, const gem_seq_t* x,
                     const gem_seq_t* f, const int32_t* lengths, const uint8_t* reset,
                     const float* saved, const gem_seq_t* dh, const float* dh_last,
                     const gem_seq_t* dx, const gem_seq_t* df, float* dh0, void* stream) {
  if (!sizes_ok(dtype, form, B, T, D)) return GEM_EINVAL;
  if (!input_ok(x, dtype, B, T, D) || !input_ok(f, dtype, B, T, D) || !input_ok(dh, dtype, B, T, D))
    return GEM_EINVAL;
  if (!output_ok(dx, dtype, B, T, D) || !output_ok(df, dtype, B, T, D)) return GEM_EINVAL;
  if (!optional_ok(lengths) || !optional_ok(saved) || !optional_ok(dh_last) || !optional_ok(dh0))
    return GEM_EINVAL;
  if (B == 0 || D == 0 || (T == 0 && !dh0)) return GEM_OK;
  if (T > 0 && !saved) return GEM_EINVAL;
  GlrArgs p = {};
  p.x = *x;
  p.f = *f;
  p.dh = *dh;
  p.dx = *dx;
  p.df = *df;
  p.lengths = lengths;
  p.reset = reset;
  p.saved_in = saved;
  p.dh_last = dh_last;
  p.dh0 = dh0;
  p.B = B;
  p.T = T;
  p.D = D;
  return launch_status(launch_glr(dtype, p, form, true, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
