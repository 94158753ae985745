// Rows of logits: how the operators over a vocabulary hold a row on chip, take its statistics and are
// launched (internal).
#pragma once

#include <cooperative_groups.h>

#include <type_traits>

#include "lm_internal.h"

namespace gem {
namespace lm {

namespace cg = cooperative_groups;

constexpr int kThreads = 512;

struct Sum {
  __device__ float operator()(float a, float b) const { return a + b; }
  static constexpr float start = 0.0f;
};
struct Max {
  __device__ float operator()(float a, float b) const { return fmaxf(a, b); }
  static constexpr float start = -INFINITY;
};

// ---- rows longer than a cluster's shared memory: a block streams the row, once for each statistic ----

// The block's value of every thread's v, in an order that the block size fixes.
template <typename Op>
__device__ float block_reduce(float v, float* buf, Op op) {
  for (int s = 16; s > 0; s >>= 1) v = op(v, __shfl_xor_sync(~0u, v, s));
  __syncthreads();
  if (threadIdx.x % 32 == 0) buf[threadIdx.x / 32] = v;
  __syncthreads();
  v = Op::start;
  for (int w = 0; w < int(blockDim.x) / 32; ++w) v = op(v, buf[w]);
  return v;
}

// The row's largest logit and sum of exp((z - m) / tau).  A row without a finite or larger
// logit has m = -inf and a sum of 0.
template <typename E>
__device__ void row_stats(const E* z, int V, float inv_tau, float* buf, float& m, float& s) {
  float v = -INFINITY;
  for (int j = threadIdx.x; j < V; j += blockDim.x) v = fmaxf(v, to_f32(z[j]));
  m = block_reduce(v, buf, Max());
  const float ref = m == -INFINITY ? 0.0f : m;
  float t = 0.0f;
  for (int j = threadIdx.x; j < V; j += blockDim.x) t += expf((to_f32(z[j]) - ref) * inv_tau);
  s = block_reduce(t, buf, Sum());
}

// ---- rows on chip ----
//
// A row is read once into the shared memory of a cluster of C blocks; all later passes read it
// there.  It is taken as its whole 16-byte pieces in memory, cut evenly over the blocks, and up to 14
// edge elements before and after them.  A thread copies pieces t, t + T, ... of its block's slice and
// is the one that reads them, so the passes over a slice need no barrier between.
//
// Clusters stay and take row after row.  The last pass over a row copies the next row's piece into
// each slot as soon as it has read it, and one or two warps of the block beside the T threads (side warps)
// do what is short and serial: the teacher's entries, the loss, the choice of alternatives, the
// edge elements.  They work on the next or the previous row while the others stream, so that
// memory and the passes seldom wait for them.  One cluster barrier per row keeps them in step.
//
// The distillation reads and writes each logit once, the scores read it once.  Per element that is
// about 18 instructions (scores: 10) and 2 exponentials (1), of which an SM issues 128 and 16 a cycle.
// Measured, bf16, 4096 x 131072: distillation with 128 entries 429 us (5.0 TB/s), scores 207 us (5.2 TB/s)
// without alternatives, 255 with one, 259 with 20 and 356 with 64, where a row's chain of barrier, search
// and sort is longer than its stream.  A block's slice of 64 KB and 256 threads was the best of 16 to
// 64 KB and 128 to 256; one pass of blocks without prefetch took 672 and 260 us.
//
// Maximum and sum in one go: every thread takes the maximum of its own pieces, then the sum
// relative to that; warps and blocks join (m, s) pairs by m = max m_i, s = sum s_i exp((m_i - m) / tau),
// in the order that the sizes fix.  The warps write their pairs to every block of the cluster.

constexpr int kRowThreads = 256;                 // most threads beside the side warp
constexpr int kRowParts = kRowThreads / 32 + 1;  // most warps of a block
constexpr int kRowCluster = 8;
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float exp2_fast(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// For gradients: fp32 ones keep probabilities below 2^-126, 16-bit ones let them go to 0.
template <typename E>
__device__ __forceinline__ float exp2_grad(float x) {
  float r;
  if constexpr (sizeof(E) == 4)
    asm("ex2.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
  else
    r = exp2_fast(x);
  return r;
}

template <typename E>
constexpr int kPer = 16 / int(sizeof(E));   // elements of a piece

// A row and the block's slice of its whole pieces.
template <typename E>
struct Slice {
  const E* row;
  int V;
  int lead;     // elements before the first whole piece
  int whole;    // whole pieces of the row
  int first;    // first one of the slice
  int pieces;   // number of the slice's
  __device__ int index(int i) const { return lead + (first + i) * kPer<E>; }   // first element of the slice's piece i
  __device__ const uint4* data() const { return reinterpret_cast<const uint4*>(row + index(0)); }
  __device__ int edges() const { return V - whole * kPer<E>; }
  __device__ int edge(int e) const { return e < lead ? e : e + whole * kPer<E>; }   // index of an edge element
};

template <typename E>
__device__ __forceinline__ Slice<E> slice_of(const E* row, int V, int rank, int C) {
  Slice<E> s;
  s.row = row;
  s.V = V;
  s.lead = min(int((16 - reinterpret_cast<uintptr_t>(row) % 16) % 16 / sizeof(E)), V);
  s.whole = (V - s.lead) / kPer<E>;
  const int per = (s.whole + C - 1) / C;
  s.first = min(rank * per, s.whole);
  s.pieces = min(per, s.whole - s.first);
  return s;
}

__device__ __forceinline__ void load_piece(uint4* slot, const uint4* from) {
  const uint32_t to = static_cast<uint32_t>(__cvta_generic_to_shared(slot));
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void load_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void load_wait() { asm volatile("cp.async.wait_group 0;" ::: "memory"); }

// The cluster barrier, in two halves.  cluster_started: the first half of one that only tells that all
// blocks have started, which they must have before another writes to them.
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }
__device__ __forceinline__ void cluster_started() { asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory"); }
// A barrier of `threads` threads of the block.
__device__ __forceinline__ void part_sync(int id, int threads) {
  asm volatile("barrier.sync %0, %1;" ::"r"(id), "r"(threads) : "memory");
}

// The variable of another block of the cluster (this block's own where rank is its own).
template <typename X>
__device__ __forceinline__ X* of_block(X* x, int rank) {
  return cg::this_cluster().map_shared_rank(x, rank);
}

// A piece's elements as pairs of floats, and back.
template <typename E>
constexpr int kPairs = kPer<E> / 2;

template <typename E>
__device__ __forceinline__ void unpack(const uint4& w, Vec<2> (&v)[kPairs<E>]) {
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int k = 0; k < kPairs<E>; ++k) {
    if constexpr (sizeof(E) == 4) {
      v[k] = {__uint_as_float(u[2 * k]), __uint_as_float(u[2 * k + 1])};
    } else if constexpr (std::is_same_v<E, __nv_bfloat16>) {
      v[k] = {__uint_as_float(u[k] << 16), __uint_as_float(u[k] & 0xffff0000u)};
    } else {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&u[k]));
      v[k] = {f.x, f.y};
    }
  }
}

template <typename E>
__device__ __forceinline__ uint4 pack(const Vec<2> (&v)[kPairs<E>]) {
  uint32_t u[4];
#pragma unroll
  for (int k = 0; k < kPairs<E>; ++k) {
    if constexpr (sizeof(E) == 4) {
      u[2 * k] = __float_as_uint(v[k].v[0]);
      u[2 * k + 1] = __float_as_uint(v[k].v[1]);
    } else if constexpr (std::is_same_v<E, __nv_bfloat16>) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(v[k].v[0], v[k].v[1]);
      u[k] = *reinterpret_cast<const uint32_t*>(&h);
    } else {
      const __half2 h = __floats2half2_rn(v[k].v[0], v[k].v[1]);
      u[k] = *reinterpret_cast<const uint32_t*>(&h);
    }
  }
  return make_uint4(u[0], u[1], u[2], u[3]);
}

// The piece's largest element (NaN is passed over: the sum finds it).
template <typename E>
__device__ __forceinline__ float piece_max(const uint4& w) {
  if constexpr (sizeof(E) == 4) {
    return fmaxf(fmaxf(__uint_as_float(w.x), __uint_as_float(w.y)), fmaxf(__uint_as_float(w.z), __uint_as_float(w.w)));
  } else {
    using P = std::conditional_t<std::is_same_v<E, __nv_bfloat16>, __nv_bfloat162, __half2>;
    const P* p = reinterpret_cast<const P*>(&w);
    const P m = __hmax2(__hmax2(p[0], p[1]), __hmax2(p[2], p[3]));
    return fmaxf(to_f32(m.x), to_f32(m.y));
  }
}

// Sums of a set of elements relative to their maximum m: s = sum exp((z - m) / tau), e = sum
// exp((z - m) / tau) (z - m) log2(e) / tau, s1 as s with tau = 1.  An empty or all -inf set has m = -inf.
struct Stats {
  float m, s, e, s1;
};
__device__ __forceinline__ Stats no_stats() { return {-INFINITY, 0.0f, 0.0f, 0.0f}; }

// a relative to m >= a.m instead (c = log2(e) / tau); an empty set stays one.
__device__ __forceinline__ void rebase(Stats& a, float m, float c) {
  const float d = a.m - (m == -INFINITY ? 0.0f : m), f = exp2_fast(d * c);
  // (far below m nothing is left of a set, and its e must not be infinite by then)
  a.e = (a.e + fmaxf(d * c, -1000.0f) * a.s) * f;
  a.s *= f;
  a.s1 *= exp2_fast(d * kLog2e);
  a.m = m;
}

// Joins b to a.
__device__ __forceinline__ void join(Stats& a, Stats b, float c) {
  const float m = fmaxf(a.m, b.m);
  rebase(a, m, c);
  rebase(b, m, c);
  a.s += b.s;
  a.e += b.e;
  a.s1 += b.s1;
}

// The warp's set from its lanes', in every lane with the same bits.
__device__ __forceinline__ Stats warp_join(Stats a, float c) {
  float m = a.m;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(~0u, m, o));
  rebase(a, m, c);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    a.s += __shfl_xor_sync(~0u, a.s, o);
    a.e += __shfl_xor_sync(~0u, a.e, o);
    a.s1 += __shfl_xor_sync(~0u, a.s1, o);
  }
  return a;
}

// What the second softmax, that with tau = 1, costs: nothing where there are no labels or tau is 1 itself;
// where tau is 2, exp(d) = exp(d / 2)^2; else exponentials of its own (4 a logit in both passes, at 16 a
// cycle and SM: 124 us instead of 110 at 4096 x 32000 with 64 entries).
enum Hard { kNoLabels, kOwnExponential, kTau1, kTau2 };

template <Hard HARD>
__device__ __forceinline__ Vec<2> second_exponential(const Vec<2>& first, const Vec<2>& d) {
  if constexpr (HARD == kTau1) return first;
  if constexpr (HARD == kTau2) return first * first;
  const Vec<2> y = d * splat<2>(kLog2e);
  return {exp2_fast(y.v[0]), exp2_fast(y.v[1])};
}

// A thread's sums over its pieces (t, t + T, ...), relative to a.m.  after(i) runs when piece i has
// been read.
template <typename E, bool ENTROPY, Hard HARD, bool CLAMP, typename F>
__device__ __forceinline__ void thread_sums(const uint4* data, int pieces, int t, int T, float c, Stats& a, F after) {
  const Vec<2> ref = splat<2>(a.m == -INFINITY ? -0.0f : -a.m), scale = splat<2>(c);
  Vec<2> s = splat<2>(0.0f), e = s, s1 = s;
#pragma unroll 2
  for (int i = t; i < pieces; i += T) {
    Vec<2> v[kPairs<E>];
    unpack<E>(data[i], v);
    after(i);
#pragma unroll
    for (int k = 0; k < kPairs<E>; ++k) {
      const Vec<2> d = v[k] + ref;
      Vec<2> x = d * scale;
      const Vec<2> p = {exp2_fast(x.v[0]), exp2_fast(x.v[1])};
      s = s + p;
      if constexpr (ENTROPY) {
        if constexpr (CLAMP) x = {fmaxf(x.v[0], -1000.0f), fmaxf(x.v[1], -1000.0f)};
        e = fma<2>(p, x, e);
      }
      if constexpr (HARD == kOwnExponential || HARD == kTau2) s1 = s1 + second_exponential<HARD>(p, d);
    }
  }
  a.s = s.v[0] + s.v[1];
  a.e = e.v[0] + e.v[1];
  a.s1 = HARD == kTau1 ? a.s : s1.v[0] + s1.v[1];
}

template <typename E>
__device__ __forceinline__ float thread_max(const uint4* data, int pieces, int t, int T) {
  float m = -INFINITY;
#pragma unroll 4
  for (int i = t; i < pieces; i += T) m = fmaxf(m, piece_max<E>(data[i]));
  return m;
}

// An edge element alone.
__device__ __forceinline__ Stats one_element(float z) {
  if (isnan(z)) return {-INFINITY, z, z, z};
  return z == -INFINITY ? no_stats() : Stats{z, 1.0f, 0.0f, 1.0f};
}

// A warp's set to every block of the cluster (all: [C * parts]), and the row's set from them.
__device__ __forceinline__ void publish_stats(const Stats& mine, Stats* all, int rank, int C, int parts, float c) {
  const Stats a = warp_join(mine, c);
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  if (lane < C) of_block(all, lane)[rank * parts + warp] = a;
}
// A warp's edge elements to every block, which most rows have none of.
__device__ __forceinline__ void publish_edges(const Stats& mine, bool any, Stats* all, int rank, int C, int parts, float c) {
  const Stats a = any ? warp_join(mine, c) : no_stats();
  const int lane = threadIdx.x % 32;
  if (lane < C) of_block(all, lane)[rank * parts + parts - 1] = a;
}
__device__ __forceinline__ Stats collect_stats(const Stats* all, int C, int parts, float c) {
  const int lane = threadIdx.x % 32, n = C * parts;
  Stats a = lane < n ? all[lane] : no_stats();
  for (int i = lane + 32; i < n; i += 32) join(a, all[i], c);
  return warp_join(a, c);
}

// ---- short rows: a warp for each, nothing shared between warps ----

constexpr int kShortWarps = 4;          // rows of a block
constexpr int kShortPieces = 512;       // most whole pieces of a row (8 KB)

// The warp's part of dynamic shared memory.
template <typename X>
__device__ __forceinline__ X* warp_part(uint4* shared, size_t bytes_of_warp) {
  return reinterpret_cast<X*>(reinterpret_cast<char*>(shared) + threadIdx.x / 32 * bytes_of_warp);
}

// Copies the row's pieces to the slots and waits for them (the lane's own, and after the warp's barrier all).
template <typename E>
__device__ __forceinline__ void load_row(const Slice<E>& s, uint4* slots) {
  for (int i = threadIdx.x % 32; i < s.pieces; i += 32) load_piece(slots + i, s.data() + i);
  load_commit();
}

// How a row is held: blocks of a cluster, threads of a block (the side warps' too) and bytes of
// shared memory.  Slices of up to 65 KB let three blocks share an SM, so that one waits while others
// work; few rows are cut further, down to 8 KB, as long as all their blocks are resident at two an SM (64
// x 50,001 fp16: 4 blocks a row 8.8 us, 8 of which some wait 12.5).  cluster = 0: the row does not fit on
// chip.
struct RowCut {
  int cluster, threads, slots;
  size_t smem;
};

inline RowCut row_cut(int dtype, int64_t N, int64_t V, int side_warps) {
  constexpr int64_t kSlice = 65 << 10, kLeast = 8 << 10, kMost = 188 << 10;
  const int64_t bytes = V * dtype_size(dtype);
  RowCut c = {1, kRowThreads, 0, 0};
  while (c.cluster < kRowCluster && bytes > kSlice * c.cluster) c.cluster *= 2;
  while (c.cluster < kRowCluster && N * c.cluster * 2 <= 2 * 152 && bytes >= 2 * kLeast * c.cluster) c.cluster *= 2;
  c.slots = int((bytes / 16 + c.cluster - 1) / c.cluster);
  c.smem = size_t(c.slots) * 16;
  if (int64_t(c.smem) > kMost) return {0, 0, 0, 0};
  c.threads += 32 * side_warps;
  return c;
}

template <auto KERNEL, typename... Args>
cudaError_t launch_rows(const RowCut& c, int64_t N, cudaStream_t stream, const Args&... args) {
  cudaError_t e = allow_shared<KERNEL>(c.smem);
  int clusters = 0;
  if (e == cudaSuccess) e = resident_clusters(reinterpret_cast<const void*>(KERNEL), c.cluster, c.threads, c.smem, &clusters);
  if (e == cudaSuccess && clusters < 1) e = cudaErrorInvalidConfiguration;
  if (e != cudaSuccess) return e;
  const int64_t grid = (N < clusters ? N : clusters) * c.cluster;
  return launch_cluster_pdl(KERNEL, unsigned(grid), unsigned(c.threads), unsigned(c.cluster), c.smem, stream, args...);
}

// Rows of up to 8 KB take a warp each (8192 x 1000 bf16, 8 entries: 16 us against 48 in blocks that stay).
inline int row_slots(int dtype, int64_t V) { return int(V * dtype_size(dtype) / 16); }
template <auto KERNEL, typename Args, typename... More>
cudaError_t launch_short(const Args& p, int dtype, int64_t N, size_t more_bytes, cudaStream_t stream, const More&... more) {
  const unsigned warp_bytes = unsigned((size_t(row_slots(dtype, p.V)) * 16 + more_bytes + 15) / 16 * 16);
  const size_t shared = size_t(warp_bytes) * kShortWarps;
  const cudaError_t e = allow_shared<KERNEL>(shared);
  if (e != cudaSuccess) return e;
  return launch_pdl(KERNEL, dim3(unsigned((N + kShortWarps - 1) / kShortWarps)), dim3(kShortWarps * 32), shared, stream, p, N,
                    warp_bytes, more...);
}
inline bool row_is_short(int dtype, int64_t V) { return V * dtype_size(dtype) <= kShortPieces * 16; }

// Grids of up to 8 blocks a row, and element indices of a row with room past its end.
constexpr int64_t kMaxRows = int64_t(1) << 27, kMaxVocabulary = int64_t(1) << 30;

inline bool rows_ok(int dtype, int64_t N, int64_t V, const void* z, int64_t ld) {
  if (!dtype_ok(dtype) || N < 0 || N > kMaxRows || V < 1 || V > kMaxVocabulary) return false;
  if (N == 0) return true;
  return z && aligned_to(z, size_t(dtype_size(dtype))) && (ld == 0 || ld >= V) && ld <= kMaxStride;
}

inline bool grad_ok(int dtype, int64_t V, const void* g, int64_t ld) {
  return g && aligned_to(g, size_t(dtype_size(dtype))) && ld >= V && ld <= kMaxStride;
}

// Within these limits neither 1 / tau nor a difference of equal logits over tau leaves fp32.
inline bool temperature_ok(float tau) { return tau >= 1.0e-20f && tau <= 1.0e20f; }

}  // namespace lm
}  // namespace gem
