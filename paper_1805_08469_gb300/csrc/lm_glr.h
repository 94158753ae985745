// Gated linear recurrence (include/gem_lm.h): what its forward and backward kernels share (internal).
#pragma once

#include <cooperative_groups.h>

#include <type_traits>

#include "lm_internal.h"

namespace gem {
namespace lm {
namespace glr {

namespace cg = cooperative_groups;

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
// The copies of a warp's next rounds are in flight while it works (cp.async into tiles of its own,
// which need no block barrier), so memory does not wait for the scan.
//
// Forward moves 3, backward 5 elements a step and channel and a 16th of a float of saved state each;
// about 25 instructions an element of 16 bits are near what the SMs issue in that time.  Measured (bf16,
// 8 x 4096 x 2048): 69 us and 118 us, 5.8 and 5.7 TB/s; fp32, 1 x 100,003 x 1024 without resets: 243 and 342 us
// (5.1 and 6.0 TB/s), 2.8 and 3.9 us a round of 72 chunks, of which scan and exchange are waited for (with a reset
// in 700 steps 259 and 412: a chunk with one takes the path that tests every step).
// Steps that made it so: 16-byte copies through the warp's tile instead of 4-byte ones (157 -> 75 us
// forward), sums and products of two channels in one instruction, gates computed again instead of spilled
// (backward 173 -> 116).
//
// A is 2^-149 at least (at_least_some): gates are above 0, so that a state of infinity stays one, while 0 times
// it is NaN.  (Of a finite state that lets through 5e-7 at the most.)
//
// A map whose steps contain a reset has A = -1: it forgets the state whatever that holds (0 times
// an infinity would not).

constexpr int kMaxWarps = 8;
constexpr int kMaxCluster = 16;   // (more than 8 blocks are for this GPU only)

template <int V>
struct Map {
  Vec<V> A, H;
};

// (RESETS: A may be -1.  NaN stays)
template <int V, bool RESETS>
__device__ __forceinline__ void at_least_some(Vec<V>& A) {
#pragma unroll
  for (int k = 0; k < V; ++k) {
    if constexpr (RESETS)
      A.v[k] = A.v[k] == 0.0f ? __uint_as_float(1u) : A.v[k];
    else
      asm("max.NaN.f32 %0, %0, 0f00000001;" : "+f"(A.v[k]));
  }
}

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
  uint64_t full[2];    // mbarriers, one for each parity of the round
  uint32_t gave_up;    // a wait of the block passed its limit: no more of the exchange, and NaN from there on
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

// Waits until the phase of this parity is complete; false after two seconds (a round takes microseconds).
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
__device__ __forceinline__ void start_exchange(Exchange& x) {
  if constexpr (CLUSTER) {
    if (threadIdx.x == 0) {
      for (int b = 0; b < 2; ++b) asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(shared_address(&x.full[b])) : "memory");
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
      x.gave_up = 0;
    }
    cg::this_cluster().sync();
  }
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
  at_least_some<V, RESETS>(all.A);
  at_least_some<V, RESETS>(mine.A);
  // (a map that forgets the state must not bring back what rests on a map that did not come; the mbarriers'
  // phases stay open, so nobody arrives on them again, and the other blocks give up in their turn)
  volatile uint32_t& gave_up = x.gave_up;
  if (gave_up) return state = splat<V>(NAN);
  // (a buffer is sent to again two rounds on: by then all have read it, or their maps of the round
  // between would not have come)
  Map<V>* in = blocks + (round & 1) * C * 32 + lane;
  const uint32_t full = shared_address(&x.full[round & 1]), slot = shared_address(in + rank * 32);
  for (int c = warp; c < C; c += warps) send<V>(in_block(slot, c), all, in_block(full, c));
  if (threadIdx.x == 0)
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(full), "r"(uint32_t(C * 32 * sizeof(Map<V>)))
                 : "memory");
  if (!wait_phase(full, uint32_t(round >> 1) & 1u)) {
    gave_up = 1;
    return state = splat<V>(NAN);
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

// A warp's tile of one tensor: kChunk rows of 32 words of channels in shared memory, row k those of
// step k.  MODE: how the tensors' rows lie in memory.
//   kVector  every row starts at a 16-byte boundary and D fills whole 16-byte pieces: lane l moves
//            piece l % 8 of rows l / 8, l / 8 + 4, ...
//   kWord    rows start at 4-byte boundaries and D fills whole words: lane l moves word l of each row
//   kOdd     16-bit rows that start at any element: lane l moves the aligned word l that covers the
//            row's channels 2 l and 2 l + 1 or, where the row starts in the middle of a word, 2 l - 1 and
//            2 l; a row has one word more
enum Mode { kVector, kWord, kOdd };
template <Mode MODE>
constexpr int kPitch = MODE == kOdd ? 33 : 32;
template <Mode MODE>
constexpr int kTile = kChunk * kPitch<MODE>;

// Bit k: row k of a tile starts in the middle of a word.
template <typename E, Mode MODE>
__device__ __forceinline__ uint32_t odd_rows(const E* row0, int64_t stride) {
  if constexpr (MODE != kOdd) return 0;
  const uint32_t first = uint32_t(reinterpret_cast<uintptr_t>(row0) >> 1 & 1);
  return ((stride & 1) ? 0xAAAAu : 0u) ^ (first ? 0xFFFFu : 0u);
}

// The lane's word of channels of row k; tile points to the lane's word of row 0.
template <Mode MODE>
__device__ __forceinline__ uint32_t read_word(const uint32_t* tile, int k, uint32_t odd) {
  const uint32_t w = tile[k * kPitch<MODE>];
  if constexpr (MODE == kOdd) return (odd >> k & 1) ? __funnelshift_r(w, tile[k * kPitch<MODE> + 1], 16) : w;
  return w;
}

__device__ __forceinline__ void fetch_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void fetch_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// Where a thread works: sequence b, its own channel word d.., and the channels it moves.
struct Place {
  int64_t b, d, move_d;
  int rank, warp, warps, lane;
  int own;      // channels of the thread's word that exist: 0..V
  int slab;     // and of the warp's slab (kOdd)
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
  w.own = int(w.d + V <= p.D ? V : w.d < p.D ? p.D - w.d : 0);
  w.slab = int(p.D - first < 32 * V ? p.D - first : 32 * V);
  w.on = w.own > 0;
  w.move_d = MODE == kVector ? first + w.lane % 8 * (16 / int(sizeof(E))) : MODE == kOdd ? first : w.d;
  w.moves = w.move_d < p.D;
  return w;
}

// Multiples of a stride are computed anew in each round: 16 of them held in registers over the rounds
// make the rest spill.
__device__ __forceinline__ void keep_out_of_registers(int64_t& stride) { asm volatile("" : "+l"(stride)); }

// Copies a word, or its first BYTES bytes.
template <int BYTES>
__device__ __forceinline__ void copy_word(uint32_t* slot, const void* from) {
  const uint32_t s = static_cast<uint32_t>(__cvta_generic_to_shared(slot));
  if constexpr (BYTES == 4)
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(s), "l"(from) : "memory");
  else
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(s), "l"(from), "n"(BYTES) : "memory");
}

// Starts the copy of rows 0..m of a tile; from: the row of step 0 at the lane's channels (move_d); data:
// the tensor's first element, slab: its channels (kOdd).
template <typename E, Mode MODE>
__device__ __forceinline__ void fetch_tile(uint32_t* tile, const E* from, int64_t stride, int m, int lane, const void* data, int slab) {
  keep_out_of_registers(stride);
  if constexpr (MODE == kVector) {
    const uint32_t s = static_cast<uint32_t>(__cvta_generic_to_shared(tile)) + lane * 16;
    from += lane / 8 * stride;
#pragma unroll
    for (int i = 0; i < kChunk / 4; ++i) {
      if (lane / 8 + 4 * i < m)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(s + i * 512), "l"(from) : "memory");
      from += 4 * stride;
    }
  } else if constexpr (MODE == kWord) {
#pragma unroll
    for (int k = 0; k < kChunk; ++k) {
      if (k < m) copy_word<4>(tile + k * 32 + lane, from);
      from += stride;
    }
  } else {
    const uint32_t odd = odd_rows<E, MODE>(from, stride);
    if ((odd & 1) && from == data) {
      // the first word would start before the tensor: its second half alone
      if (lane == 0)
        for (int k = 0; k < m; ++k)
          if (from + k * stride == data) reinterpret_cast<E*>(tile + k * kPitch<MODE>)[1] = *from;
    }
    // every other row starts alike: in a word's middle or not
    const int c = 2 * lane;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const E* word = from + r * stride + c;
      if (odd >> r & 1) {
        const bool full = c < slab, half = c == slab, one_more = lane == 0 && slab == 64;
        const bool before = lane == 0 && from == data, all_before = before && stride == 0;   // (copied above)
#pragma unroll
        for (int k = r; k < kChunk; k += 2) {
          uint32_t* const row = tile + k * kPitch<MODE>;
          if (k < m) {
            if (full && !(k == 0 ? before : all_before)) copy_word<4>(row + lane, word - 1);
            if (half) copy_word<2>(row + lane, word - 1);
            if (one_more) copy_word<2>(row + 32, word + 63);
          }
          word += 2 * stride;
        }
      } else {
        const bool full = c + 1 < slab, half = c + 1 == slab;
#pragma unroll
        for (int k = r; k < kChunk; k += 2) {
          uint32_t* const row = tile + k * kPitch<MODE>;
          if (k < m) {
            if (full) copy_word<4>(row + lane, word);
            if (half) copy_word<2>(row + lane, word);
          }
          word += 2 * stride;
        }
      }
    }
  }
}

// Stores rows 0..m of a tile that the warp has written, word by word of its own channels (all lanes
// call; the tile is free after).
template <typename E, Mode MODE>
__device__ __forceinline__ void store_tile(const uint32_t* tile, E* to, int64_t stride, int m, int lane, bool moves, int slab) {
  keep_out_of_registers(stride);
  __syncwarp();
  if constexpr (MODE == kVector) {
    const uint4* t = reinterpret_cast<const uint4*>(tile) + lane;
    to += lane / 8 * stride;
#pragma unroll
    for (int i = 0; i < kChunk / 4; ++i) {
      if (moves && lane / 8 + 4 * i < m) *reinterpret_cast<uint4*>(to) = t[i * 32];
      to += 4 * stride;
    }
  } else if constexpr (MODE == kWord) {
#pragma unroll
    for (int k = 0; k < kChunk; ++k) {
      if (moves && k < m) *reinterpret_cast<uint32_t*>(to) = tile[k * 32 + lane];
      to += stride;
    }
  } else {
    const uint32_t odd = odd_rows<E, MODE>(to, stride);
    const int c = 2 * lane;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      E* word = to + r * stride + c;
      if (odd >> r & 1) {
        // the aligned word of channels c + 1 and c + 2; the slab's first channel and an even last one alone
        const bool full = c + 2 < slab, half = c + 2 == slab;
#pragma unroll
        for (int k = r; k < kChunk; k += 2) {
          const uint32_t* const row = tile + k * kPitch<MODE> + lane;
          if (k < m) {
            const uint32_t w = row[0];
            const E* const halves = reinterpret_cast<const E*>(&w);
            if (full) *reinterpret_cast<uint32_t*>(word + 1) = __funnelshift_r(w, row[1], 16);
            if (half) word[1] = halves[1];
            if (lane == 0) word[0] = halves[0];
          }
          word += 2 * stride;
        }
      } else {
        const bool full = c + 1 < slab, half = c + 1 == slab;
#pragma unroll
        for (int k = r; k < kChunk; k += 2) {
          const uint32_t w = tile[k * kPitch<MODE> + lane];
          const E* const halves = reinterpret_cast<const E*>(&w);
          if (k < m) {
            if (full) *reinterpret_cast<uint32_t*>(word) = w;
            if (half) word[0] = halves[0];
          }
          word += 2 * stride;
        }
      }
    }
  }
  __syncwarp();
}

// A tile of zeros for store_zeros.  All lanes call.
template <typename E, Mode MODE>
__device__ __forceinline__ void clear_tile(uint32_t* tile) {
  __syncwarp();
  for (int i = threadIdx.x % 32; i < kTile<MODE>; i += 32) tile[i] = 0;
}

// Zeros from such a tile to the rows of chunks c, c + step, ... of `all` (steps past a sequence's end), stored as
// wide as values are (24 x 1777 x 1000 fp16 of random lengths, forward: 44 us; element by element 60).  All lanes call.
template <typename E, Mode MODE>
__device__ __forceinline__ void store_zeros(const uint32_t* tile, E* to, int64_t stride, int64_t c, int64_t step, int64_t all, int64_t T,
                                            int lane, bool moves, int slab) {
  for (; c < all; c += step) {
    const int64_t t0 = c * kChunk;
    store_tile<E, MODE>(tile, to + t0 * stride, stride, int(T - t0 < kChunk ? T - t0 : kChunk), lane, moves, slab);
  }
}

// Bit k: a reset at step k of a chunk (k < m), from the lanes' bytes.  The bytes are read a round ahead.
template <bool RESETS>
__device__ __forceinline__ uint8_t load_reset(const GlrArgs& p, int64_t b, int64_t t) {
  return RESETS && t < p.T && threadIdx.x % 32 < kChunk ? p.reset[b * p.T + t] : 0;
}
template <bool RESETS>
__device__ __forceinline__ uint32_t reset_bits(uint8_t lane_byte, int m) {
  return RESETS ? __ballot_sync(~0u, int(threadIdx.x % 32) < m && lane_byte != 0) : 0;
}

// How the work is cut.  About 16 warps fit an SM (128 registers a thread).  Few slabs of channels:
// clusters share a slab's time, as large ones as leave all slabs resident at once; many: blocks of
// fewer warps, so that all slabs are resident.  Neither goes past the chunks there are.  A slab for two
// SMs in three or more: no clusters, whose rounds take longer (bf16, forward: 128 slabs of 4,096 steps
// 45 us without and 52 in clusters of two; 96 slabs of 8,000 steps 84 and 70 in threes).
//
// DIRECTION names the kernel, its tensors copied in and their stages.
template <typename DIRECTION, typename E, int V, Mode MODE, bool LERP, bool RESETS>
cudaError_t launch_form(const GlrArgs& p, cudaStream_t stream) {
  constexpr int kSms = 152, kBlocks = 2;   // (of an SM)
  constexpr size_t kWarpBytes = size_t(kTile<MODE>) * 4 * DIRECTION::kTensors * DIRECTION::kStages;
  const int64_t chunks = (p.T + kChunk - 1) / kChunk;
  const int64_t slabs = (p.D + 32 * V - 1) / (32 * V) * p.B;
  auto clip = [](int64_t v, int64_t lo, int64_t hi) { return v < lo ? lo : v > hi ? hi : v; };
  int cluster = int(clip(3 * slabs > 2 * kSms ? 1 : kBlocks * kSms / slabs, 1, clip((chunks + kMaxWarps - 1) / kMaxWarps, 1, kMaxCluster)));
  if (cluster > 1) {
    constexpr auto kKernel = DIRECTION::template kernel<E, V, MODE, LERP, true, RESETS>();
    cudaError_t e = allow_shared<kKernel, true>(kMaxShared);
    if (e != cudaSuccess) return e;
    for (; cluster > 1; --cluster) {
      const size_t shared = kMaxWarps * kWarpBytes + size_t(2) * cluster * 32 * sizeof(Map<V>);
      int fit = 0;
      e = resident_clusters(reinterpret_cast<const void*>(kKernel), cluster, kMaxWarps * 32, shared, &fit);
      if (e != cudaSuccess) return e;
      if (fit >= slabs)
        return launch_cluster_pdl(kKernel, unsigned(slabs * cluster), unsigned(kMaxWarps * 32), unsigned(cluster), shared, stream, p,
                                  cluster);
    }
  }
  constexpr auto kKernel = DIRECTION::template kernel<E, V, MODE, LERP, false, RESETS>();
  const int warps = int(clip(kBlocks * kMaxWarps / ((slabs + kSms - 1) / kSms), 1, clip(chunks, 1, kMaxWarps)));
  const size_t shared = warps * kWarpBytes;
  const cudaError_t e = allow_shared<kKernel>(shared);
  if (e != cudaSuccess) return e;
  return launch_cluster_pdl(kKernel, unsigned(slabs), unsigned(warps * 32), 1, shared, stream, p, 1);
}

template <typename DIRECTION, typename E, int V, Mode MODE>
cudaError_t launch_mode(const GlrArgs& p, int form, cudaStream_t stream) {
  if (form == GEM_GLR_LERP)
    return p.reset ? launch_form<DIRECTION, E, V, MODE, true, true>(p, stream) : launch_form<DIRECTION, E, V, MODE, true, false>(p, stream);
  return p.reset ? launch_form<DIRECTION, E, V, MODE, false, true>(p, stream) : launch_form<DIRECTION, E, V, MODE, false, false>(p, stream);
}

// By the largest power of two, 16 bytes at most, on which every row of every tensor starts and D ends.
template <typename DIRECTION, typename E>
cudaError_t launch_tiles(const GlrArgs& p, int form, cudaStream_t stream) {
  uint64_t bits = 16 | uint64_t(p.D) * sizeof(E);
  for (const gem_seq_t* s : DIRECTION::tensors(p)) {
    bits |= reinterpret_cast<uintptr_t>(s->data);
    if (p.B > 1) bits |= uint64_t(s->stride_b) * sizeof(E);
    if (p.T > 1) bits |= uint64_t(s->stride_t) * sizeof(E);
  }
  constexpr int kWordV = 4 / sizeof(E);
  if (bits % 16 == 0) return launch_mode<DIRECTION, E, kWordV, kVector>(p, form, stream);
  if constexpr (sizeof(E) == 2) {
    if (bits % 4 != 0) return launch_mode<DIRECTION, E, kWordV, kOdd>(p, form, stream);
  }
  return launch_mode<DIRECTION, E, kWordV, kWord>(p, form, stream);
}

// The directions' launches for one element type each, compiled apart (lm_glr_f32.cu and so on).
template <typename E>
cudaError_t launch_forward(const GlrArgs& p, int form, cudaStream_t stream);
template <typename E>
cudaError_t launch_backward(const GlrArgs& p, int form, cudaStream_t stream);

}  // namespace glr
}  // namespace lm
}  // namespace gem
