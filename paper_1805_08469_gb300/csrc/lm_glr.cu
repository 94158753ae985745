// Gated linear recurrence (include/gem_lm.h): h_t = a_t h_{t-1} + u_t with a = sigmoid(f) and
// u = (1 - a) x or x.  Forward kernels and the calls; lm_glr_backward.cu has the backward kernels.
#include <array>

#include "lm_glr.h"

namespace gem {
namespace lm {
namespace glr {
namespace {

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
template <typename E, int V, bool LERP, bool PLAIN>
__device__ __forceinline__ Map<V> forward_map(const uint32_t* x, const uint32_t* f, int m, uint32_t fresh, Vec<V> (&a)[kChunk],
                                              Vec<V> (&u)[kChunk]) {
  Map<V> own = {splat<V>(1.0f), splat<V>(0.0f)};
#pragma unroll
  for (int k = 0; k < kChunk; ++k) {
    Vec<V> b;
    u[k] = unpack<E, V>(x[k * 32]);
    gate<E, V>(unpack<E, V>(f[k * 32]), a[k], b);
    if constexpr (LERP) u[k] = b * u[k];
    if (!PLAIN && k >= m) {
      a[k] = splat<V>(1.0f);
      u[k] = splat<V>(0.0f);
    }
    const Vec<V> moved = fma<V>(a[k], own.H, u[k]);
    own.H = !PLAIN && (fresh >> k & 1) ? u[k] : moved;
    own.A = own.A * a[k];
  }
  if (!PLAIN && fresh) own.A = splat<V>(-1.0f);
  return own;
}

template <typename E, int V, bool PLAIN>
__device__ __forceinline__ void forward_apply(uint32_t* out, uint32_t fresh, const Vec<V> (&a)[kChunk], const Vec<V> (&u)[kChunk],
                                              Vec<V> h) {
#pragma unroll
  for (int k = 0; k < kChunk; ++k) {
    const Vec<V> moved = fma<V>(a[k], h, u[k]);
    h = !PLAIN && (fresh >> k & 1) ? u[k] : moved;
    out[k * 32] = pack<E, V>(h);
  }
}

// Stages of a thread's copies and blocks of an SM.  16-bit rows at odd addresses are copied through
// registers, so more threads hide their latency instead of more stages (4 x 3,001 x 777 bf16: 34 us
// against 52); fp32 rows gain nothing from it (276 against 270 at 100,003 x 1024).
template <Mode MODE>
constexpr int kForwardStages = MODE == kHalf ? 2 : 3;
template <Mode MODE>
constexpr int kForwardBlocks = MODE == kHalf ? 3 : 2;

template <typename E, int V, Mode MODE, bool LERP, bool CLUSTER, bool RESETS>
__global__ void __launch_bounds__(kMaxWarps * 32, kForwardBlocks<MODE>) glr_forward_kernel(const GlrArgs p, int blocks_of_cluster) {
  const int C = CLUSTER ? blocks_of_cluster : 1;
  extern __shared__ __align__(16) uint32_t tiles[];   // [warp][stage][x, f][kTile], then the blocks' maps
  __shared__ Map<V> maps[2 * kMaxWarps * 32];
  __shared__ uint64_t mbarriers[2];
  pdl_entry();
  Exchange exchange = start_exchange<CLUSTER>(mbarriers);
  const Place w = place_of<E, V, MODE>(p, C);
  constexpr int kStage = 2 * kTile;
  uint32_t* const ring = tiles + w.warp * kForwardStages<MODE> * kStage;
  Map<V>* const blocks = reinterpret_cast<Map<V>*>(tiles + w.warps * kForwardStages<MODE> * kStage);
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
  for (int v = 0; v < V; ++v) state.v[v] = p.h0 && w.on ? p.h0[state_at + v] : 0.0f;

  auto issue = [&](int round, int stage) {
    const int64_t c = first + round * per_round;
    if (round < rounds && c < chunks && w.moves) {
      const int64_t t0 = c * kChunk;
      const int m = int(n - t0 < kChunk ? n - t0 : kChunk);
      fetch_tile<E, MODE>(ring + stage * kStage, x + t0 * p.x.stride_t, p.x.stride_t, m, w.lane);
      fetch_tile<E, MODE>(ring + stage * kStage + kTile, f + t0 * p.f.stride_t, p.f.stride_t, m, w.lane);
    }
    fetch_commit();
  };
#pragma unroll
  for (int r = 0; r < kForwardStages<MODE> - 1; ++r) issue(r, r);

  int stage = 0;
  uint8_t next_reset = load_reset<RESETS>(p, w.b, first * kChunk + w.lane);
  for (int round = 0; round < rounds; ++round) {
    issue(round + kForwardStages<MODE> - 1, stage == 0 ? kForwardStages<MODE> - 1 : stage - 1);
    const int64_t c = first + round * per_round, t0 = c * kChunk;
    const bool busy = c < chunks;
    const int m = busy ? int(n - t0 < kChunk ? n - t0 : kChunk) : 0;
    const uint32_t fresh = reset_bits<RESETS>(next_reset, m);
    next_reset = load_reset<RESETS>(p, w.b, t0 + per_round * kChunk + w.lane);
    const bool plain = m == kChunk && fresh == 0;
    fetch_wait<kForwardStages<MODE> - 1>();
    __syncwarp();
    uint32_t* const tile = ring + stage * kStage;
    stage = stage == kForwardStages<MODE> - 1 ? 0 : stage + 1;
    Vec<V> a[kChunk], u[kChunk];
    const Map<V> own = plain ? forward_map<E, V, LERP, true>(tile + w.lane, tile + kTile + w.lane, m, fresh, a, u)
                             : forward_map<E, V, LERP, false>(tile + w.lane, tile + kTile + w.lane, m, fresh, a, u);
    const Vec<V> h = scan_round<V, RESETS, CLUSTER>(own, round, w.warps, w.rank, C, maps, blocks, exchange, state);
    if (!busy) continue;
    if (p.saved_out && w.on) {
      float* s = p.saved_out + (w.b * all_chunks + c) * p.D + w.d;
#pragma unroll
      for (int v = 0; v < V; ++v) s[v] = h.v[v];
    }
    if (plain)
      forward_apply<E, V, true>(tile + w.lane, fresh, a, u, h);
    else
      forward_apply<E, V, false>(tile + w.lane, fresh, a, u, h);
    store_tile<E, MODE>(tile, h_out + t0 * p.h.stride_t, p.h.stride_t, m, w.lane, w.moves);
  }
  // all have read h0 before it is replaced, and no block leaves before what the others sent it
  CLUSTER ? cg::this_cluster().sync() : __syncthreads();
  if (!w.on) return;
  // past the sequence's end: zeros, and the state as it stays
  store_zeros<E, V>(at<E>(p.h, w.b, 0, w.d), p.h.stride_t, n + first, per_round, p.T);
  if (p.saved_out)
    for (int64_t c = chunks + first; c < all_chunks; c += per_round)
#pragma unroll
      for (int v = 0; v < V; ++v) p.saved_out[(w.b * all_chunks + c) * p.D + w.d + v] = state.v[v];
  if (p.h_last && first == 0) {
#pragma unroll
    for (int v = 0; v < V; ++v) p.h_last[state_at + v] = state.v[v];
  }
}

struct Forward {
  static constexpr int kTensors = 2;
  template <Mode MODE>
  static constexpr int stages() { return kForwardStages<MODE>; }
  template <Mode MODE>
  static constexpr int blocks() { return kForwardBlocks<MODE>; }
  template <typename E, int V, Mode MODE, bool LERP, bool CLUSTER, bool RESETS>
  static constexpr auto kernel() { return &glr_forward_kernel<E, V, MODE, LERP, CLUSTER, RESETS>; }
  static std::array<const gem_seq_t*, 3> tensors(const GlrArgs& p) { return {&p.x, &p.f, &p.h}; }
};

template <typename E>
cudaError_t launch_step(const GlrArgs& p, int form, cudaStream_t stream) {
  auto* kernel = form == GEM_GLR_LERP ? glr_step_kernel<E, true> : glr_step_kernel<E, false>;
  return launch_pdl(kernel, dim3(unsigned((p.B * p.D + 127) / 128)), dim3(128), 0, stream, p);
}

cudaError_t launch_forward(int dtype, const GlrArgs& p, int form, cudaStream_t stream) {
  if (p.T > kStepT) return launch_tiles<Forward>(dtype, p, form, stream);
  switch (dtype) {
    case GEM_F32: return launch_step<float>(p, form, stream);
    case GEM_BF16: return launch_step<__nv_bfloat16>(p, form, stream);
    default: return launch_step<__half>(p, form, stream);
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
}  // namespace glr
}  // namespace lm
}  // namespace gem

using namespace gem::lm;
using namespace gem::lm::glr;

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
  return launch_status(launch_forward(dtype, p, form, static_cast<cudaStream_t>(stream)));
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
  return launch_status(launch_backward(dtype, p, form, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
