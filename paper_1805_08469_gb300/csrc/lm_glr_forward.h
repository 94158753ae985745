// Gated linear recurrence: forward kernels (internal; included once for each element type).
#pragma once

#include <array>

#include "lm_glr.h"

namespace gem {
namespace lm {
namespace glr {

// ---- a few steps: one thread per channel, one step after the other (1.5 us for 4 x 1 x 1024) ----

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
      Vec<1> a, c;
      gate<E, 1>({to_f32(*at<const E>(p.f, b, t, d))}, a, c);
      const float x = to_f32(*at<const E>(p.x, b, t, d));
      const float u = LERP ? c.v[0] * x : x;
      h = p.reset && p.reset[b * p.T + t] ? u : fmaf(a.v[0], h, u);
      shown = h;
    }
    *at<E>(p.h, b, t, d) = from_f32<E>(shown);
  }
  if (p.h_last) p.h_last[i] = h;
}
constexpr int64_t kStepT = 2;   // longest call of the kernel above (one chunk: saved is h0)

// The steps of a chunk: all kChunk of them without a reset (PLAIN), or the first m with resets
// where `fresh` has a bit.
template <typename E, int V, Mode MODE, bool LERP, bool PLAIN>
__device__ __forceinline__ Map<V> forward_map(const uint32_t* x, const uint32_t* f, uint32_t odd_x, uint32_t odd_f, int m,
                                              uint32_t fresh, Vec<V> (&a)[kChunk], Vec<V> (&u)[kChunk]) {
  Map<V> own = {splat<V>(1.0f), splat<V>(0.0f)};
#pragma unroll
  for (int k = 0; k < kChunk; ++k) {
    Vec<V> b;
    u[k] = unpack<E, V>(read_word<MODE>(x, k, odd_x));
    gate<E, V>(unpack<E, V>(read_word<MODE>(f, k, odd_f)), a[k], b);
    if constexpr (LERP) u[k] = b * u[k];
    if (!PLAIN && k >= m) {
      a[k] = splat<V>(1.0f);
      u[k] = splat<V>(0.0f);
    }
    const Vec<V> moved = fma<V>(a[k], own.H, u[k]);
    own.H = !PLAIN && (fresh >> k & 1) ? u[k] : moved;
    own.A = own.A * a[k];
  }
  at_least_some<V, false>(own.A);
  if (!PLAIN && fresh) own.A = splat<V>(-1.0f);
  return own;
}

template <typename E, int V, Mode MODE, bool PLAIN>
__device__ __forceinline__ void forward_apply(uint32_t* out, int m, uint32_t fresh, const Vec<V> (&a)[kChunk], const Vec<V> (&u)[kChunk],
                                              Vec<V> h) {
#pragma unroll
  for (int k = 0; k < kChunk; ++k) {
    const Vec<V> moved = fma<V>(a[k], h, u[k]);
    h = !PLAIN && (fresh >> k & 1) ? u[k] : moved;
    out[k * kPitch<MODE>] = PLAIN || k < m ? pack<E, V>(h) : 0u;   // (a row past the sequence's end)
  }
}

constexpr int kForwardStages = 3;

template <typename E, int V, Mode MODE, bool LERP, bool CLUSTER, bool RESETS>
__global__ void __launch_bounds__(kMaxWarps * 32, 2) glr_forward_kernel(const GlrArgs p, int blocks_of_cluster) {
  const int C = CLUSTER ? blocks_of_cluster : 1;
  extern __shared__ __align__(16) uint32_t tiles[];   // [warp][stage][x, f][kTile], then the blocks' maps
  __shared__ Map<V> maps[2 * kMaxWarps * 32];
  __shared__ Exchange exchange;
  pdl_entry();
  start_exchange<CLUSTER>(exchange);
  const Place w = place_of<E, V, MODE>(p, C);
  constexpr int kStage = 2 * kTile<MODE>;
  uint32_t* const ring = tiles + w.warp * kForwardStages * kStage;
  Map<V>* const blocks = reinterpret_cast<Map<V>*>(tiles + w.warps * kForwardStages * kStage);
  const int64_t n = steps_of(p, w.b);
  const int64_t chunks = (n + kChunk - 1) / kChunk, all_chunks = (p.T + kChunk - 1) / kChunk;
  const int64_t per_round = int64_t(w.warps) * C;
  const int rounds = int((chunks + per_round - 1) / per_round);
  const int64_t first = int64_t(w.rank) * w.warps + w.warp;   // chunk of round 0
  const E* x = at<const E>(p.x, w.b, 0, w.move_d);
  const E* f = at<const E>(p.f, w.b, 0, w.move_d);
  E* h_out = at<E>(p.h, w.b, 0, w.move_d);
  const int64_t state_at = w.b * p.D + w.d;
  Vec<V> state;
#pragma unroll
  for (int v = 0; v < V; ++v) state.v[v] = p.h0 && v < w.own ? p.h0[state_at + v] : 0.0f;

  auto issue = [&](int round, int stage) {
    const int64_t c = first + round * per_round;
    if (round < rounds && c < chunks && w.moves) {
      const int64_t t0 = c * kChunk;
      const int m = int(n - t0 < kChunk ? n - t0 : kChunk);
      fetch_tile<E, MODE>(ring + stage * kStage, x + t0 * p.x.stride_t, p.x.stride_t, m, w.lane, p.x.data, w.slab);
      fetch_tile<E, MODE>(ring + stage * kStage + kTile<MODE>, f + t0 * p.f.stride_t, p.f.stride_t, m, w.lane, p.f.data, w.slab);
    }
    fetch_commit();
  };
#pragma unroll
  for (int r = 0; r < kForwardStages - 1; ++r) issue(r, r);

  int stage = 0;
  uint8_t next_reset = load_reset<RESETS>(p, w.b, first * kChunk + w.lane);
  for (int round = 0; round < rounds; ++round) {
    issue(round + kForwardStages - 1, stage == 0 ? kForwardStages - 1 : stage - 1);
    const int64_t c = first + round * per_round, t0 = c * kChunk;
    const bool busy = c < chunks;
    const int m = busy ? int(n - t0 < kChunk ? n - t0 : kChunk) : 0;
    const uint32_t fresh = reset_bits<RESETS>(next_reset, m);
    next_reset = load_reset<RESETS>(p, w.b, t0 + per_round * kChunk + w.lane);
    const bool plain = m == kChunk && fresh == 0;
    fetch_wait<kForwardStages - 1>();
    __syncwarp();
    uint32_t* const tile = ring + stage * kStage;
    stage = stage == kForwardStages - 1 ? 0 : stage + 1;
    Vec<V> a[kChunk], u[kChunk];
    const uint32_t odd_x = odd_rows<E, MODE>(x + t0 * p.x.stride_t, p.x.stride_t);
    const uint32_t odd_f = odd_rows<E, MODE>(f + t0 * p.f.stride_t, p.f.stride_t);
    const uint32_t *const xs = tile + w.lane, *const fs = xs + kTile<MODE>;
    const Map<V> own = plain ? forward_map<E, V, MODE, LERP, true>(xs, fs, odd_x, odd_f, m, fresh, a, u)
                             : forward_map<E, V, MODE, LERP, false>(xs, fs, odd_x, odd_f, m, fresh, a, u);
    const Vec<V> h = scan_round<V, RESETS, CLUSTER>(own, round, w.warps, w.rank, C, maps, blocks, exchange, state);
    if (!busy) continue;
    if (p.saved_out && w.on) {
      float* s = p.saved_out + (w.b * all_chunks + c) * p.D + w.d;
#pragma unroll
      for (int v = 0; v < V; ++v)
        if (v < w.own) s[v] = h.v[v];
    }
    if (plain)
      forward_apply<E, V, MODE, true>(tile + w.lane, m, fresh, a, u, h);
    else
      forward_apply<E, V, MODE, false>(tile + w.lane, m, fresh, a, u, h);
    store_tile<E, MODE>(tile, h_out + t0 * p.h.stride_t, p.h.stride_t, int(p.T - t0 < kChunk ? p.T - t0 : kChunk), w.lane, w.moves, w.slab);
  }
  // all have read h0 before it is replaced, and no block leaves before what the others sent it
  CLUSTER ? cg::this_cluster().sync() : __syncthreads();
  // past the sequence's end: zeros, and the state as it stays
  if (chunks < all_chunks) {
    clear_tile<E, MODE>(ring);
    store_zeros<E, MODE>(ring, h_out, p.h.stride_t, chunks + first, per_round, all_chunks, p.T, w.lane, w.moves, w.slab);
  }
  if (!w.on) return;
  if (p.saved_out)
    for (int64_t c = chunks + first; c < all_chunks; c += per_round)
#pragma unroll
      for (int v = 0; v < V; ++v)
        if (v < w.own) p.saved_out[(w.b * all_chunks + c) * p.D + w.d + v] = state.v[v];
  if (p.h_last && first == 0) {
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (v < w.own) p.h_last[state_at + v] = state.v[v];
  }
}

struct Forward {
  static constexpr int kTensors = 2;
  static constexpr int kStages = kForwardStages;
  template <typename E, int V, Mode MODE, bool LERP, bool CLUSTER, bool RESETS>
  static constexpr auto kernel() { return &glr_forward_kernel<E, V, MODE, LERP, CLUSTER, RESETS>; }
  static std::array<const gem_seq_t*, 3> tensors(const GlrArgs& p) { return {&p.x, &p.f, &p.h}; }
};

template <typename E>
cudaError_t launch_step(const GlrArgs& p, int form, cudaStream_t stream) {
  auto* kernel = form == GEM_GLR_LERP ? glr_step_kernel<E, true> : glr_step_kernel<E, false>;
  return launch_pdl(kernel, dim3(unsigned((p.B * p.D + 127) / 128)), dim3(128), 0, stream, p);
}

template <typename E>
cudaError_t launch_forward(const GlrArgs& p, int form, cudaStream_t stream) {
  return p.T > kStepT ? launch_tiles<Forward, E>(p, form, stream) : launch_step<E>(p, form, stream);
}

}  // namespace glr
}  // namespace lm
}  // namespace gem
