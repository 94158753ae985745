// Gated linear recurrence: backward kernels (internal; included once for each element type).
#pragma once

#include <array>

#include "lm_glr.h"

namespace gem {
namespace lm {
namespace glr {

// Backward: the same scan from the end.  A step's map is g -> a (dh + g), g being what the step
// after it hands back.  A chunk's map is sum_k (a_0 .. a_k) dh_k + (a_0 .. a_15) g, so it is
// composed in the same pass over the steps that computes the states before them again, from the
// saved one; nothing counts from the first reset on.  q: what the gate's gradient multiplies,
// h_{t-1} - x_t or h_{t-1}.  The gates are kept in registers for one channel a thread; for two they would
// take 64 (and spilled: 173 us instead of 116 at 8 x 4096 x 2048 bf16), and are computed again.
struct Words {
  const uint32_t *x, *f, *dh;   // the lane's words of the tiles
  uint32_t odd_x, odd_f, odd_dh;
};

template <int V>
constexpr int kKeep = V == 1 ? kChunk : 1;

template <typename E, int V, Mode MODE, bool LERP, bool PLAIN>
__device__ __forceinline__ Map<V> backward_map(const Words& in, int m, uint32_t fresh,
                                               Vec<V> h, Vec<V> (&q)[kChunk], Vec<V> (&gates)[2][kKeep<V>]) {
  Map<V> own = {splat<V>(1.0f), splat<V>(0.0f)};
  bool counts = true;
#pragma unroll
  for (int k = 0; k < kChunk; ++k) {
    if (!PLAIN && k >= m) continue;
    Vec<V> a, b;
    const Vec<V> xv = unpack<E, V>(read_word<MODE>(in.x, k, in.odd_x));
    gate<E, V>(unpack<E, V>(read_word<MODE>(in.f, k, in.odd_f)), a, b);
    const Vec<V> u = LERP ? b * xv : xv;
    const bool r = !PLAIN && (fresh >> k & 1);
    if (r) h = splat<V>(0.0f);
    q[k] = LERP ? h - xv : h;
    h = r ? u : fma<V>(a, h, u);
    if constexpr (V == 1) {
      gates[0][k] = a;
      gates[1][k] = b;
    }
    if (r) counts = false;
    if (counts) {
      own.A = own.A * a;
      at_least_some<V, false>(own.A);   // (at every step: any dh may be infinite)
      own.H = fma<V>(own.A, unpack<E, V>(read_word<MODE>(in.dh, k, in.odd_dh)), own.H);
    }
  }
  if (!PLAIN && fresh) own.A = splat<V>(-1.0f);
  return own;
}

template <typename E, int V, Mode MODE, bool LERP, bool PLAIN>
__device__ __forceinline__ void backward_apply(const Words& in, uint32_t* dx, uint32_t* df, int m, uint32_t fresh,
                                               const Vec<V> (&q)[kChunk], const Vec<V> (&gates)[2][kKeep<V>], Vec<V> g) {
#pragma unroll
  for (int k = kChunk - 1; k >= 0; --k) {
    if (!PLAIN && k >= m) {   // a row past the sequence's end
      dx[k * kPitch<MODE>] = df[k * kPitch<MODE>] = 0u;
      continue;
    }
    g = g + unpack<E, V>(read_word<MODE>(in.dh, k, in.odd_dh));
    Vec<V> a, b;
    if constexpr (V == 1) {
      a = gates[0][k];
      b = gates[1][k];
    } else {
      gate<E, V>(unpack<E, V>(read_word<MODE>(in.f, k, in.odd_f)), a, b);   // again from f (its slot is df's)
    }
    if constexpr (MODE == kOdd) __syncwarp();   // (a neighbour reads the word of f that df replaces)
    dx[k * kPitch<MODE>] = pack<E, V>(LERP ? b * g : g);
    g = a * g;
    df[k * kPitch<MODE>] = pack<E, V>(g * (q[k] * b));
    if (!PLAIN && (fresh >> k & 1)) g = splat<V>(0.0f);
  }
}

constexpr int kBackwardStages = 2;

template <typename E, int V, Mode MODE, bool LERP, bool CLUSTER, bool RESETS>
__global__ void __launch_bounds__(kMaxWarps * 32, 2) glr_backward_kernel(const GlrArgs p, int blocks_of_cluster) {
  const int C = CLUSTER ? blocks_of_cluster : 1;
  extern __shared__ __align__(16) uint32_t tiles[];   // [warp][stage][x, f, dh][kTile], then the blocks' maps
  __shared__ Map<V> maps[2 * kMaxWarps * 32];
  __shared__ Exchange exchange;
  pdl_entry();
  start_exchange<CLUSTER>(exchange);
  const Place w = place_of<E, V, MODE>(p, C);
  constexpr int kStage = 3 * kTile<MODE>;
  uint32_t* const ring = tiles + w.warp * kBackwardStages * kStage;
  Map<V>* const blocks = reinterpret_cast<Map<V>*>(tiles + w.warps * kBackwardStages * kStage);
  const int64_t n = steps_of(p, w.b);
  const int64_t chunks = (n + kChunk - 1) / kChunk, all_chunks = (p.T + kChunk - 1) / kChunk;
  const int64_t per_round = int64_t(w.warps) * C;
  const int rounds = int((chunks + per_round - 1) / per_round);
  const int64_t first = int64_t(w.rank) * w.warps + w.warp;   // chunks are counted from the end
  const E* x = at<const E>(p.x, w.b, 0, w.move_d);
  const E* f = at<const E>(p.f, w.b, 0, w.move_d);
  const E* dh = at<const E>(p.dh, w.b, 0, w.move_d);
  E* dx_out = at<E>(p.dx, w.b, 0, w.move_d);
  E* df_out = at<E>(p.df, w.b, 0, w.move_d);
  const int64_t state_at = w.b * p.D + w.d;
  Vec<V> state, saved = splat<V>(0.0f);
#pragma unroll
  for (int v = 0; v < V; ++v) state.v[v] = p.dh_last && v < w.own ? p.dh_last[state_at + v] : 0.0f;

  auto issue = [&](int round, int stage) {
    const int64_t l = first + round * per_round;
    if (round < rounds && l < chunks && w.moves) {
      const int64_t t0 = (chunks - 1 - l) * kChunk;
      const int m = int(n - t0 < kChunk ? n - t0 : kChunk);
      uint32_t* tile = ring + stage * kStage;
      fetch_tile<E, MODE>(tile, x + t0 * p.x.stride_t, p.x.stride_t, m, w.lane, p.x.data, w.slab);
      fetch_tile<E, MODE>(tile + kTile<MODE>, f + t0 * p.f.stride_t, p.f.stride_t, m, w.lane, p.f.data, w.slab);
      fetch_tile<E, MODE>(tile + 2 * kTile<MODE>, dh + t0 * p.dh.stride_t, p.dh.stride_t, m, w.lane, p.dh.data, w.slab);
    }
    fetch_commit();
  };
  // the saved state of a round, read one round ahead
  auto load_saved = [&](int round) {
    const int64_t l = first + round * per_round;
    if (l < chunks && w.on) {
      const float* s = p.saved_in + (w.b * all_chunks + chunks - 1 - l) * p.D + w.d;
#pragma unroll
      for (int v = 0; v < V; ++v)
        if (v < w.own) saved.v[v] = s[v];
    }
  };
#pragma unroll
  for (int r = 0; r < kBackwardStages - 1; ++r) issue(r, r);
  load_saved(0);

  int stage = 0;
  uint8_t next_reset = first < chunks ? load_reset<RESETS>(p, w.b, (chunks - 1 - first) * kChunk + w.lane) : 0;
  for (int round = 0; round < rounds; ++round) {
    issue(round + kBackwardStages - 1, stage == 0 ? kBackwardStages - 1 : stage - 1);
    const int64_t l = first + round * per_round, t0 = (chunks - 1 - l) * kChunk;
    const bool busy = l < chunks;
    const int m = busy ? int(n - t0 < kChunk ? n - t0 : kChunk) : 0;
    const uint32_t fresh = reset_bits<RESETS>(next_reset, m);
    next_reset = l + per_round < chunks ? load_reset<RESETS>(p, w.b, t0 - per_round * kChunk + w.lane) : 0;
    const bool plain = m == kChunk && fresh == 0;
    fetch_wait<kBackwardStages - 1>();
    __syncwarp();
    uint32_t* const tile = ring + stage * kStage;
    const Words in = {tile + w.lane, tile + kTile<MODE> + w.lane, tile + 2 * kTile<MODE> + w.lane,
                      odd_rows<E, MODE>(x + t0 * p.x.stride_t, p.x.stride_t), odd_rows<E, MODE>(f + t0 * p.f.stride_t, p.f.stride_t),
                      odd_rows<E, MODE>(dh + t0 * p.dh.stride_t, p.dh.stride_t)};
    stage = stage == kBackwardStages - 1 ? 0 : stage + 1;
    Vec<V> q[kChunk], gates[2][kKeep<V>];
    const Vec<V> h = saved;
    load_saved(round + 1);
    const Map<V> own = plain ? backward_map<E, V, MODE, LERP, true>(in, m, fresh, h, q, gates)
                             : backward_map<E, V, MODE, LERP, false>(in, m, fresh, h, q, gates);
    const Vec<V> g = scan_round<V, RESETS, CLUSTER>(own, round, w.warps, w.rank, C, maps, blocks, exchange, state);
    if (!busy) continue;
    if (plain)
      backward_apply<E, V, MODE, LERP, true>(in, tile + w.lane, tile + kTile<MODE> + w.lane, m, fresh, q, gates, g);
    else
      backward_apply<E, V, MODE, LERP, false>(in, tile + w.lane, tile + kTile<MODE> + w.lane, m, fresh, q, gates, g);
    const int shown = int(p.T - t0 < kChunk ? p.T - t0 : kChunk);
    store_tile<E, MODE>(tile, dx_out + t0 * p.dx.stride_t, p.dx.stride_t, shown, w.lane, w.moves, w.slab);
    store_tile<E, MODE>(tile + kTile<MODE>, df_out + t0 * p.df.stride_t, p.df.stride_t, shown, w.lane, w.moves, w.slab);
  }
  CLUSTER ? cg::this_cluster().sync() : __syncthreads();
  if (chunks < all_chunks) {
    clear_tile<E, MODE>(ring);
    store_zeros<E, MODE>(ring, dx_out, p.dx.stride_t, chunks + first, per_round, all_chunks, p.T, w.lane, w.moves, w.slab);
    store_zeros<E, MODE>(ring, df_out, p.df.stride_t, chunks + first, per_round, all_chunks, p.T, w.lane, w.moves, w.slab);
  }
  if (!w.on) return;
  if (p.dh0 && first == 0) {
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (v < w.own) p.dh0[state_at + v] = state.v[v];
  }
}

struct Backward {
  static constexpr int kTensors = 3;
  static constexpr int kStages = kBackwardStages;
  template <typename E, int V, Mode MODE, bool LERP, bool CLUSTER, bool RESETS>
  static constexpr auto kernel() { return &glr_backward_kernel<E, V, MODE, LERP, CLUSTER, RESETS>; }
  static std::array<const gem_seq_t*, 5> tensors(const GlrArgs& p) { return {&p.x, &p.f, &p.dh, &p.dx, &p.df}; }
};

template <typename E>
cudaError_t launch_backward(const GlrArgs& p, int form, cudaStream_t stream) {
  return launch_tiles<Backward, E>(p, form, stream);
}

}  // namespace glr
}  // namespace lm
}  // namespace gem
