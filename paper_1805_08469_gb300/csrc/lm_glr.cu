// Gated linear recurrence (include/gem_lm.h): h_t = a_t h_{t-1} + u_t with a = sigmoid(f) and
// u = (1 - a) x or x, and its backward pass.
#include <cooperative_groups.h>

#include <type_traits>

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
template <typename E, int V>
__device__ __forceinline__ void gate(Vec<V> f, Vec<V>& a, Vec<V>& b) {
  Vec<V> e;
#pragma unroll
  for (int k = 0; k < V; ++k) asm("max.NaN.f32 %0, %0, 0fC2A00000;" : "+f"(f.v[k]));
  if constexpr (sizeof(E) == 4) {
    e.v[0] = expf(-f.v[0]);
  } else {
    // 16-bit inputs carry 2^-9 themselves; rounding f log2(e) costs |f| 2^-24 of e
    f = f * splat<V>(-1.44269504f);
#pragma unroll
    for (int k = 0; k < V; ++k) asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e.v[k]) : "f"(f.v[k]));
  }
  const Vec<V> s = e + splat<V>(1.0f);
#pragma unroll
  for (int k = 0; k < V; ++k) asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(a.v[k]) : "f"(s.v[k]));
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
constexpr int kMaxCluster = 16;   // (more than 8 blocks are for this GPU only)

template <int V>
struct Map {
  Vec<V> A, H;
};

// h after the map m, and m after the maps composed so far.  RESETS: a map may forget.
template <int V, bool RESETS>
__device__ __forceinline__ Vec<V> apply(const Vec<V>& h, const Map<V>& m) {
  Vec<V> r = fma<V>(m.A, h, m.H);
  if constexpr (RESETS) {
#pragma unroll
    for (int k = 0; k < V; ++k) r.v[k] = m.A.v[k] < 0.0f ? m.H.v[k] : r.v[k];
  }
  return r;
}

template <int V, bool RESETS>
__device__ __forceinline__ Map<V> compose(const Map<V>& sofar, const Map<V>& m) {
  Map<V> r = {sofar.A * m.A, apply<V, RESETS>(sofar.H, m)};
  if constexpr (RESETS) {
#pragma unroll
    for (int k = 0; k < V; ++k) r.A.v[k] = m.A.v[k] < 0.0f || sofar.A.v[k] < 0.0f ? -1.0f : r.A.v[k];
  }
  return r;
}

// The exchange of the blocks' maps in a cluster: each block sends its map to every block with stores
// that count their bytes on the receiver's mbarrier, so nothing else (a cluster barrier would wait for
// all of a block's stores to memory) holds the round up.
struct Exchange {
  uint32_t full;   // shared address of two mbarriers, one for each parity of the round
  bool gave_up;    // a wait passed its limit: the states are NaN from there on
};

__device__ __forceinline__ uint32_t shared_address(const void* p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }

__device__ __forceinline__ uint32_t in_block(uint32_t address, int rank) {
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(address), "r"(rank));
  return r;
}

template <int V>
__device__ __forceinline__ void send(uint32_t to, const Map<V>& m, uint32_t mbarrier) {
  if constexpr (V == 2)
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.b32 [%0], {%1, %2, %3, %4}, [%5];" ::"r"(to),
                 "r"(__float_as_uint(m.A.v[0])), "r"(__float_as_uint(m.A.v[1])), "r"(__float_as_uint(m.H.v[0])),
                 "r"(__float_as_uint(m.H.v[1])), "r"(mbarrier)
                 : "memory");
  else
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.b32 [%0], {%1, %2}, [%3];" ::"r"(to),
                 "r"(__float_as_uint(m.A.v[0])), "r"(__float_as_uint(m.H.v[0])), "r"(mbarrier)
                 : "memory");
}

// Waits until the phase of this parity is complete; false after two seconds (it never takes
// microseconds unless a block of the cluster is gone).
__device__ __forceinline__ bool wait_phase(uint32_t mbarrier, uint32_t parity) {
  uint64_t start = 0;
  for (unsigned i = 1;; ++i) {
    uint32_t done;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(done)
        : "r"(mbarrier), "r"(parity)
        : "memory");
    if (done) return true;
    if (i % 256 == 0) {
      uint64_t now;
      asm volatile("mov.u64 %0, %globaltimer;" : "=l"(now));
      if (start == 0)
        start = now;
      else if (now - start > 2000000000ull)
        return false;
    }
  }
}

// Sets the mbarriers up; all threads call.  No block sends before all have.
template <bool CLUSTER>
__device__ __forceinline__ Exchange start_exchange(uint64_t (&mbarriers)[2]) {
  Exchange x = {shared_address(mbarriers), false};
  if constexpr (CLUSTER) {
    if (threadIdx.x == 0) {
      for (int b = 0; b < 2; ++b) asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(x.full + 8 * b) : "memory");
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    cg::this_cluster().sync();
  }
  return x;
}

// From every thread's map of a round: the state before the thread's chunk, and `state` moved on to
// the state after the round.  maps: [2][kMaxWarps][32], blocks: [2][C][32] (C > 1) in shared memory.
template <int V, bool RESETS, bool CLUSTER>
__device__ __forceinline__ Vec<V> scan_round(const Map<V>& own, int round, int warps, int rank, int C, Map<V>* maps, Map<V>* blocks,
                                             Exchange& x, Vec<V>& state) {
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  Map<V>* buf = maps + (round & 1) * kMaxWarps * 32 + lane;
  Vec<V> before = state;
  buf[warp * 32] = own;
  __syncthreads();
  if constexpr (!CLUSTER) {
#pragma unroll
    for (int w = 0; w < kMaxWarps; ++w) {
      if (w >= warps) break;
      if (w == warp) before = state;
      state = apply<V, RESETS>(state, buf[w * 32]);
    }
    return before;
  }
  Map<V> all = {splat<V>(1.0f), splat<V>(0.0f)}, mine = all;
#pragma unroll
  for (int w = 0; w < kMaxWarps; ++w) {
    if (w >= warps) break;
    if (w == warp) mine = all;
    all = compose<V, RESETS>(all, buf[w * 32]);
  }
  // (a buffer is sent to again two rounds on: by then all have read it, or their maps of the round
  // between would not have come)
  Map<V>* in = blocks + (round & 1) * C * 32 + lane;
  const uint32_t full = x.full + 8 * (round & 1), slot = shared_address(in + rank * 32);
  for (int c = warp; c < C; c += warps) send<V>(in_block(slot, c), all, in_block(full, c));
  if (threadIdx.x == 0)
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(full), "r"(uint32_t(C * 32 * sizeof(Map<V>)))
                 : "memory");
  if (!x.gave_up && !wait_phase(full, uint32_t(round >> 1) & 1u)) {
    x.gave_up = true;
    state = splat<V>(NAN);
  }
  for (int c = 0; c < C; ++c) {
    if (c == rank) before = state;
    state = apply<V, RESETS>(state, in[c * 32]);
  }
  return apply<V, RESETS>(before, mine);
}

// A word of channels as V floats, and back.
template <typename E, int V>
__device__ __forceinline__ Vec<V> unpack(uint32_t w) {
  Vec<V> r;
  if constexpr (sizeof(E) == 4) {
    r.v[0] = __uint_as_float(w);
  } else if constexpr (std::is_same_v<E, __nv_bfloat16>) {
    r.v[0] = __uint_as_float(w << 16);
    if constexpr (V == 2) r.v[1] = __uint_as_float(w & 0xffff0000u);
  } else {
    const __half2 h = *reinterpret_cast<const __half2*>(&w);
    r.v[0] = __low2float(h);
    if constexpr (V == 2) r.v[1] = __high2float(h);
  }
  return r;
}

template <typename E, int V>
__device__ __forceinline__ uint32_t pack(const Vec<V>& a) {
  if constexpr (sizeof(E) == 4) {
    return __float_as_uint(a.v[0]);
  } else if constexpr (std::is_same_v<E, __nv_bfloat16>) {
    const __nv_bfloat162 w = __floats2bfloat162_rn(a.v[0], V == 2 ? a.v[V - 1] : 0.0f);
    return *reinterpret_cast<const uint32_t*>(&w);
  } else {
    const __half2 w = __floats2half2_rn(a.v[0], V == 2 ? a.v[V - 1] : 0.0f);
    return *reinterpret_cast<const uint32_t*>(&w);
  }
}

// A warp's tile of one tensor: kChunk rows of 32 words in shared memory, row k the channels of
// step k.  MODE: how the tensors' rows lie in memory.
//   kVector  every row starts at a 16-byte boundary and D fills whole 16-byte pieces: lane l moves
//            piece l % 8 of rows l / 8, l / 8 + 4, ...
//   kWord    rows start at 4-byte boundaries: lane l moves word l of each row
//   kHalf    16-bit rows start anywhere; a word holds one channel
enum Mode { kVector, kWord, kHalf };
constexpr int kTile = kChunk * 32;

__device__ __forceinline__ void fetch_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void fetch_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// Where a thread works: sequence b, its own channel word d.., and the channels it moves.
struct Place {
  int64_t b, d, move_d;
  int rank, warp, warps, lane;
  bool on, moves;
};

template <typename E, int V, Mode MODE>
__device__ __forceinline__ Place place_of(const GlrArgs& p, int C) {
  Place w;
  const int64_t slabs = (p.D + 32 * V - 1) / (32 * V);
  const int64_t id = blockIdx.x / C;
  w.rank = blockIdx.x % C;
  w.lane = threadIdx.x % 32;
  w.warp = threadIdx.x / 32;
  w.warps = blockDim.x / 32;
  w.b = id / slabs;
  const int64_t first = id % slabs * 32 * V;
  w.d = first + w.lane * V;
  w.on = w.d < p.D;
  w.move_d = MODE == kVector ? first + w.lane % 8 * (16 / int(sizeof(E))) : w.d;
  w.moves = w.move_d < p.D;
  return w;
}

// Starts the copy of rows 0..m of a tile; from: the row of step 0 at the lane's channels (move_d).
template <typename E, Mode MODE>
__device__ __forceinline__ void fetch_tile(uint32_t* tile, const E* from, int64_t stride, int m, int lane) {
  if constexpr (MODE == kVector) {
    const uint32_t s = static_cast<uint32_t>(__cvta_generic_to_shared(tile)) + lane * 16;
    from += lane / 8 * stride;
#pragma unroll
    for (int i = 0; i < kChunk / 4; ++i) {
      if (lane / 8 + 4 * i < m)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(s + i * 512), "l"(from) : "memory");
      from += 4 * stride;
    }
  } else {
#pragma unroll
    for (int k = 0; k < kChunk; ++k) {
      if (k < m) {
        if constexpr (MODE == kWord) {
          const uint32_t s = static_cast<uint32_t>(__cvta_generic_to_shared(tile + k * 32 + lane));
          asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(s), "l"(from) : "memory");
        } else {
          *reinterpret_cast<E*>(tile + k * 32 + lane) = *from;
        }
      }
      from += stride;
    }
  }
}

// Stores rows 0..m of a tile that the warp has written (all lanes call; the tile is free after).
template <typename E, Mode MODE>
__device__ __forceinline__ void store_tile(const uint32_t* tile, E* to, int64_t stride, int m, int lane, bool moves) {
  __syncwarp();
  if constexpr (MODE == kVector) {
    const uint4* t = reinterpret_cast<const uint4*>(tile) + lane;
    to += lane / 8 * stride;
#pragma unroll
    for (int i = 0; i < kChunk / 4; ++i) {
      if (moves && lane / 8 + 4 * i < m) *reinterpret_cast<uint4*>(to) = t[i * 32];
      to += 4 * stride;
    }
  } else {
#pragma unroll
    for (int k = 0; k < kChunk; ++k) {
      if (moves && k < m) {
        if constexpr (MODE == kWord)
          *reinterpret_cast<uint32_t*>(to) = tile[k * 32 + lane];
        else
          *to = *reinterpret_cast<const E*>(tile + k * 32 + lane);
      }
      to += stride;
    }
  }
  __syncwarp();
}

// Zeros to rows t, t + step, ... below T (steps past a sequence's end).
template <typename E, int V>
__device__ __forceinline__ void store_zeros(E* to, int64_t stride, int64_t t, int64_t step, int64_t T) {
  for (; t < T; t += step)
#pragma unroll
    for (int v = 0; v < V; ++v) to[t * stride + v] = from_f32<E>(0.0f);
}

// Bit k: a reset at step t0 + k (k < m).  All lanes of the warp call.
__device__ __forceinline__ uint32_t reset_bits(const GlrArgs& p, int64_t b, int64_t t0, int m) {
  if (!p.reset) return 0;
  const int lane = threadIdx.x % 32;
  const bool r = lane < m && p.reset[b * p.T + t0 + lane] != 0;
  return __ballot_sync(~0u, r);
}

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

template <typename E, int V, Mode MODE, bool LERP, bool CLUSTER>
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
  const bool resets = p.reset != nullptr;
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
  for (int round = 0; round < rounds; ++round) {
    issue(round + kForwardStages<MODE> - 1, stage == 0 ? kForwardStages<MODE> - 1 : stage - 1);
    const int64_t c = first + round * per_round, t0 = c * kChunk;
    const bool busy = c < chunks;
    const int m = busy ? int(n - t0 < kChunk ? n - t0 : kChunk) : 0;
    const uint32_t fresh = reset_bits(p, w.b, t0, m);
    const bool plain = m == kChunk && fresh == 0;
    fetch_wait<kForwardStages<MODE> - 1>();
    __syncwarp();
    uint32_t* const tile = ring + stage * kStage;
    stage = stage == kForwardStages<MODE> - 1 ? 0 : stage + 1;
    Vec<V> a[kChunk], u[kChunk];
    const Map<V> own = plain ? forward_map<E, V, LERP, true>(tile + w.lane, tile + kTile + w.lane, m, fresh, a, u)
                             : forward_map<E, V, LERP, false>(tile + w.lane, tile + kTile + w.lane, m, fresh, a, u);
    const Vec<V> h = resets ? scan_round<V, true, CLUSTER>(own, round, w.warps, w.rank, C, maps, blocks, exchange, state)
                            : scan_round<V, false, CLUSTER>(own, round, w.warps, w.rank, C, maps, blocks, exchange, state);
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

// Backward: the same scan from the end.  A step's map is g -> a (dh + g), g being what the step
// after it hands back.  A chunk's map is sum_k (a_0 .. a_k) dh_k + (a_0 .. a_15) g, so it is
// composed in the same pass over the steps that computes the states before them again, from the
// saved one; nothing counts from the first reset on.  q: what the gate's gradient multiplies,
// h_{t-1} - x_t or h_{t-1}.  The gates are kept in registers for one channel a thread; for two they would
// take 64 (and spilled: 173 us instead of 116 at 8 x 4096 x 2048 bf16), and are computed again.
template <int V>
constexpr int kKeep = V == 1 ? kChunk : 1;

template <typename E, int V, bool LERP, bool PLAIN>
__device__ __forceinline__ Map<V> backward_map(const uint32_t* x, const uint32_t* f, const uint32_t* dh, int m, uint32_t fresh,
                                               Vec<V> h, Vec<V> (&q)[kChunk], Vec<V> (&gates)[2][kKeep<V>]) {
  Map<V> own = {splat<V>(1.0f), splat<V>(0.0f)};
  bool counts = true;
#pragma unroll
  for (int k = 0; k < kChunk; ++k) {
    if (!PLAIN && k >= m) continue;
    Vec<V> a, b;
    const Vec<V> xv = unpack<E, V>(x[k * 32]);
    gate<E, V>(unpack<E, V>(f[k * 32]), a, b);
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
      own.H = fma<V>(own.A, unpack<E, V>(dh[k * 32]), own.H);
    }
  }
  if (!PLAIN && fresh) own.A = splat<V>(-1.0f);
  return own;
}

template <typename E, int V, bool LERP, bool PLAIN>
__device__ __forceinline__ void backward_apply(uint32_t* dx, uint32_t* df, const uint32_t* dh, int m, uint32_t fresh,
                                               const Vec<V> (&q)[kChunk], const Vec<V> (&gates)[2][kKeep<V>], Vec<V> g) {
#pragma unroll
  for (int k = kChunk - 1; k >= 0; --k) {
    if (!PLAIN && k >= m) continue;
    g = g + unpack<E, V>(dh[k * 32]);
    Vec<V> a, b;
    if constexpr (V == 1) {
      a = gates[0][k];
      b = gates[1][k];
    } else {
      gate<E, V>(unpack<E, V>(df[k * 32]), a, b);   // again from f (its slot is df's)
    }
    dx[k * 32] = pack<E, V>(LERP ? b * g : g);
    g = a * g;
    df[k * 32] = pack<E, V>(g * (q[k] * b));
    if (!PLAIN && (fresh >> k & 1)) g = splat<V>(0.0f);
  }
}

constexpr int kBackwardStages = 2;

template <typename E, int V, Mode MODE, bool LERP, bool CLUSTER>
__global__ void __launch_bounds__(kMaxWarps * 32, 2) glr_backward_kernel(const GlrArgs p, int blocks_of_cluster) {
  const int C = CLUSTER ? blocks_of_cluster : 1;
  extern __shared__ __align__(16) uint32_t tiles[];   // [warp][stage][x, f, dh][kTile], then the blocks' maps
  __shared__ Map<V> maps[2 * kMaxWarps * 32];
  __shared__ uint64_t mbarriers[2];
  pdl_entry();
  Exchange exchange = start_exchange<CLUSTER>(mbarriers);
  const Place w = place_of<E, V, MODE>(p, C);
  constexpr int kStage = 3 * kTile;
  uint32_t* const ring = tiles + w.warp * kBackwardStages * kStage;
  Map<V>* const blocks = reinterpret_cast<Map<V>*>(tiles + w.warps * kBackwardStages * kStage);
  const int64_t n = steps_of(p, w.b);
  const int64_t chunks = (n + kChunk - 1) / kChunk, all_chunks = (p.T + kChunk - 1) / kChunk;
  const int64_t per_round = int64_t(w.warps) * C;
  const int rounds = int((chunks + per_round - 1) / per_round);
  const int64_t first = int64_t(w.rank) * w.warps + w.warp;   // chunks are counted from the end
  const bool resets = p.reset != nullptr;
  const E* x = at<const E>(p.x, w.b, 0, w.move_d);
  const E* f = at<const E>(p.f, w.b, 0, w.move_d);
  const E* dh = at<const E>(p.dh, w.b, 0, w.move_d);
  E* dx_out = at<E>(p.dx, w.b, 0, w.move_d);
  E* df_out = at<E>(p.df, w.b, 0, w.move_d);
  const int64_t state_at = w.b * p.D + w.d;
  Vec<V> state, saved = splat<V>(0.0f);
#pragma unroll
  for (int v = 0; v < V; ++v) state.v[v] = p.dh_last && w.on ? p.dh_last[state_at + v] : 0.0f;

  auto issue = [&](int round, int stage) {
    const int64_t l = first + round * per_round;
    if (round < rounds && l < chunks && w.moves) {
      const int64_t t0 = (chunks - 1 - l) * kChunk;
      const int m = int(n - t0 < kChunk ? n - t0 : kChunk);
      uint32_t* tile = ring + stage * kStage;
      fetch_tile<E, MODE>(tile, x + t0 * p.x.stride_t, p.x.stride_t, m, w.lane);
      fetch_tile<E, MODE>(tile + kTile, f + t0 * p.f.stride_t, p.f.stride_t, m, w.lane);
      fetch_tile<E, MODE>(tile + 2 * kTile, dh + t0 * p.dh.stride_t, p.dh.stride_t, m, w.lane);
    }
    fetch_commit();
  };
  // the saved state of a round, read one round ahead
  auto load_saved = [&](int round) {
    const int64_t l = first + round * per_round;
    if (l < chunks && w.on) {
      const float* s = p.saved_in + (w.b * all_chunks + chunks - 1 - l) * p.D + w.d;
#pragma unroll
      for (int v = 0; v < V; ++v) saved.v[v] = s[v];
    }
  };
#pragma unroll
  for (int r = 0; r < kBackwardStages - 1; ++r) issue(r, r);
  load_saved(0);

  int stage = 0;
  for (int round = 0; round < rounds; ++round) {
    issue(round + kBackwardStages - 1, stage == 0 ? kBackwardStages - 1 : stage - 1);
    const int64_t l = first + round * per_round, t0 = (chunks - 1 - l) * kChunk;
    const bool busy = l < chunks;
    const int m = busy ? int(n - t0 < kChunk ? n - t0 : kChunk) : 0;
    const uint32_t fresh = reset_bits(p, w.b, t0, m);
    const bool plain = m == kChunk && fresh == 0;
    fetch_wait<kBackwardStages - 1>();
    __syncwarp();
    uint32_t* const tile = ring + stage * kStage;
    const uint32_t* const dhs = tile + 2 * kTile + w.lane;
    stage = stage == kBackwardStages - 1 ? 0 : stage + 1;
    Vec<V> q[kChunk], gates[2][kKeep<V>];
    const Vec<V> h = saved;
    load_saved(round + 1);
    const Map<V> own = plain ? backward_map<E, V, LERP, true>(tile + w.lane, tile + kTile + w.lane, dhs, m, fresh, h, q, gates)
                             : backward_map<E, V, LERP, false>(tile + w.lane, tile + kTile + w.lane, dhs, m, fresh, h, q, gates);
    const Vec<V> g = resets ? scan_round<V, true, CLUSTER>(own, round, w.warps, w.rank, C, maps, blocks, exchange, state)
                            : scan_round<V, false, CLUSTER>(own, round, w.warps, w.rank, C, maps, blocks, exchange, state);
    if (!busy) continue;
    if (plain)
      backward_apply<E, V, LERP, true>(tile + w.lane, tile + kTile + w.lane, dhs, m, fresh, q, gates, g);
    else
      backward_apply<E, V, LERP, false>(tile + w.lane, tile + kTile + w.lane, dhs, m, fresh, q, gates, g);
    store_tile<E, MODE>(tile, dx_out + t0 * p.dx.stride_t, p.dx.stride_t, m, w.lane, w.moves);
    store_tile<E, MODE>(tile + kTile, df_out + t0 * p.df.stride_t, p.df.stride_t, m, w.lane, w.moves);
  }
  CLUSTER ? cg::this_cluster().sync() : __syncthreads();
  if (!w.on) return;
  store_zeros<E, V>(at<E>(p.dx, w.b, 0, w.d), p.dx.stride_t, n + first, per_round, p.T);
  store_zeros<E, V>(at<E>(p.df, w.b, 0, w.d), p.df.stride_t, n + first, per_round, p.T);
  if (p.dh0 && first == 0) {
#pragma unroll
    for (int v = 0; v < V; ++v) p.dh0[state_at + v] = state.v[v];
  }
}

// How the work is cut.  About 16 warps fit an SM (128 registers a thread).  Few slabs of channels:
// clusters share a slab's time, as large ones as leave all slabs resident at once; many: blocks of
// fewer warps, so that all slabs are resident.  Neither goes past the chunks there are.
template <typename E, int V, Mode MODE, bool LERP>
cudaError_t launch_form(const GlrArgs& p, bool backward, cudaStream_t stream) {
  constexpr int kSms = 152;
  const int64_t chunks = (p.T + kChunk - 1) / kChunk;
  const int64_t slabs = (p.D + 32 * V - 1) / (32 * V) * p.B;
  const int stage = kTile * 4 * (backward ? kBackwardStages * 3 : kForwardStages<MODE> * 2);   // bytes of a warp's tiles
  auto clip = [](int64_t v, int64_t lo, int64_t hi) { return v < lo ? lo : v > hi ? hi : v; };
  const int blocks_per_sm = backward ? 2 : kForwardBlocks<MODE>;
  int cluster = int(clip(blocks_per_sm * kSms / slabs, 1, clip((chunks + kMaxWarps - 1) / kMaxWarps, 1, kMaxCluster)));
  if (cluster > 1) {
    constexpr auto kForward = glr_forward_kernel<E, V, MODE, LERP, true>;
    constexpr auto kBackward = glr_backward_kernel<E, V, MODE, LERP, true>;
    cudaError_t e = backward ? allow_shared<kBackward, true>(kMaxShared) : allow_shared<kForward, true>(kMaxShared);
    if (e != cudaSuccess) return e;
    auto* kernel = backward ? kBackward : kForward;
    for (; cluster > 1; --cluster) {
      const size_t shared = size_t(kMaxWarps) * stage + size_t(2) * cluster * 32 * sizeof(Map<V>);
      int fit = 0;
      e = resident_clusters(reinterpret_cast<const void*>(kernel), cluster, kMaxWarps * 32, shared, &fit);
      if (e != cudaSuccess) return e;
      if (fit >= slabs)
        return launch_cluster_pdl(kernel, unsigned(slabs * cluster), unsigned(kMaxWarps * 32), unsigned(cluster), shared, stream, p, cluster);
    }
  }
  constexpr auto kForward = glr_forward_kernel<E, V, MODE, LERP, false>;
  constexpr auto kBackward = glr_backward_kernel<E, V, MODE, LERP, false>;
  const int warps = int(clip(blocks_per_sm * kMaxWarps / ((slabs + kSms - 1) / kSms), 1, clip(chunks, 1, kMaxWarps)));
  const size_t shared = size_t(warps) * stage;
  const cudaError_t e = backward ? allow_shared<kBackward>(shared) : allow_shared<kForward>(shared);
  if (e != cudaSuccess) return e;
  return launch_cluster_pdl(backward ? kBackward : kForward, unsigned(slabs), unsigned(warps * 32), 1, shared, stream, p, 1);
}

template <typename E, int V, Mode MODE>
cudaError_t launch_tiles(const GlrArgs& p, bool lerp, bool backward, cudaStream_t stream) {
  return lerp ? launch_form<E, V, MODE, true>(p, backward, stream) : launch_form<E, V, MODE, false>(p, backward, stream);
}

template <typename E>
cudaError_t launch(const GlrArgs& p, int form, bool backward, cudaStream_t stream) {
  const bool lerp = form == GEM_GLR_LERP;
  if (!backward && p.T <= kStepT) {
    const int64_t blocks = (p.B * p.D + 127) / 128;
    return launch_pdl(lerp ? glr_step_kernel<E, true> : glr_step_kernel<E, false>, dim3(unsigned(blocks)), dim3(128), 0, stream, p);
  }
  // the largest power of two up to 16 bytes on which every row of every tensor starts and D ends
  uint64_t bits = 16 | uint64_t(p.D) * sizeof(E);
  for (const gem_seq_t* s : {&p.x, &p.f, backward ? &p.dh : &p.h, backward ? &p.dx : &p.h, backward ? &p.df : &p.h}) {
    bits |= reinterpret_cast<uintptr_t>(s->data);
    if (p.B > 1) bits |= uint64_t(s->stride_b) * sizeof(E);
    if (p.T > 1) bits |= uint64_t(s->stride_t) * sizeof(E);
  }
  constexpr int kWordV = 4 / sizeof(E);
  if (bits % 16 == 0) return launch_tiles<E, kWordV, kVector>(p, lerp, backward, stream);
  if constexpr (sizeof(E) == 2) {
    if (bits % 4 != 0) return launch_tiles<E, 1, kHalf>(p, lerp, backward, stream);
  }
  return launch_tiles<E, kWordV, kWord>(p, lerp, backward, stream);
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
