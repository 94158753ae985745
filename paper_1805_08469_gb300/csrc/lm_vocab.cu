// Losses and scores over rows of logits (include/gem_lm.h): distillation from a teacher's top
// logits, log probabilities of tokens with entropy and top alternatives, and their gradients.
#include <cooperative_groups.h>

#include <type_traits>

#include "lm_internal.h"

namespace cg = cooperative_groups;

namespace gem {
namespace lm {
namespace {

constexpr int kThreads = 512;
static_assert(kThreads >= GEM_TOP_MAX, "a thread per top entry");

struct DistillArgs {
  const void* logits;
  void* grad;
  int64_t ld, grad_ld;
  int V, K;
  const int32_t* top_idx;
  const float* top_logits;
  const float* teacher_lse;
  const int32_t* labels;
  const float* row_scale;
  float tau, alpha;
  float* loss;
};

struct LogpArgs {
  const void* logits;
  int64_t ld;
  int V, K;
  const int32_t* tokens;
  float tau;
  float* logp;
  float* entropy;
  float* lse;
  int32_t* top_idx;
  float* top_logp;
};

struct LogpGradArgs {
  const void* logits;
  void* grad;
  int64_t ld, grad_ld;
  int V;
  const int32_t* tokens;
  float tau;
  const float* lse;
  const float* entropy;
  const float* dlogp;
  const float* dentropy;
};

struct Sum {
  __device__ float operator()(float a, float b) const { return a + b; }
  static constexpr float start = 0.0f;
};
struct Max {
  __device__ float operator()(float a, float b) const { return fmaxf(a, b); }
  static constexpr float start = -INFINITY;
};

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

template <typename E>
__global__ void __launch_bounds__(kThreads) distill_stream_kernel(const DistillArgs p) {
  pdl_entry();
  __shared__ float buf[kThreads / 32];
  __shared__ int at[GEM_TOP_MAX];
  __shared__ float qs[GEM_TOP_MAX];
  const int64_t n = blockIdx.x;
  const E* z = static_cast<const E*>(p.logits) + n * p.ld;
  E* grad = p.grad ? static_cast<E*>(p.grad) + n * p.grad_ld : nullptr;
  const int tid = threadIdx.x;
  const float w = p.row_scale ? p.row_scale[n] : 1.0f;
  if (w == 0.0f) {
    if (grad)
      for (int j = tid; j < p.V; j += blockDim.x) grad[j] = from_f32<E>(0.0f);
    if (tid == 0) p.loss[n] = 0.0f;
    return;
  }
  const float inv_tau = 1.0f / p.tau;

  // the teacher: thread k holds entry k
  int j = -1;
  float t = -INFINITY;
  if (tid < p.K) {
    j = p.top_idx[n * p.K + tid];
    if (j >= 0 && j < p.V) t = p.top_logits[n * p.K + tid] * inv_tau;
    if (t == -INFINITY) j = -1;
    at[tid] = j;
  }
  const bool there = tid < p.K && j >= 0;
  float lse;
  if (p.teacher_lse) {
    lse = p.teacher_lse[n];
  } else {
    const float mt = block_reduce(t, buf, Max());
    const float st = block_reduce(there ? expf(t - mt) : 0.0f, buf, Sum());
    lse = mt + logf(st);
  }
  const float logq = t - lse;
  const float q = there ? expf(logq) : 0.0f;
  if (tid < p.K) qs[tid] = q;
  const float mass = block_reduce(q, buf, Sum());   // (its barriers also publish at and qs)
  // entries with the same index: the first of them stands for all in the gradient
  bool first = there;
  float q_here = 0.0f;
  if (there)
    for (int k = 0; k < p.K; ++k)
      if (at[k] == j) {
        q_here += qs[k];
        if (k < tid) first = false;
      }

  float m, s;
  row_stats(z, p.V, inv_tau, buf, m, s);
  const float ref = m == -INFINITY ? 0.0f : m;
  const float inv_s = s == 0.0f ? 0.0f : 1.0f / s;
  const float zk = there ? to_f32(z[j]) : 0.0f;
  const float logp = (zk - ref) * inv_tau - logf(s == 0.0f ? 1.0f : s);
  float kl = block_reduce(q > 0.0f ? q * (logq - logp) : 0.0f, buf, Sum());
  float inside = mass, outside = mass;   // factors of p_j in the gradient
  if (p.teacher_lse) {
    // the mass outside the entries, summed by itself: 1 - sum p_k would cancel
    float r = 0.0f;
    for (int i = tid; i < p.V; i += blockDim.x) {
      bool top = false;
      for (int k = 0; k < p.K; ++k) top |= at[k] == i;
      if (!top) r += expf((to_f32(z[i]) - ref) * inv_tau);
    }
    r = block_reduce(r, buf, Sum());
    const float qr = r > 0.0f ? fmaxf(1.0f - mass, 0.0f) : 0.0f;
    if (qr > 0.0f) {
      kl += qr * (logf(qr) - logf(r * inv_s));
      inside += qr;
      outside = inside - qr * s / r;
    }
  }
  const float soft = (1.0f - p.alpha) * p.tau;
  float loss = soft * p.tau * kl;
  int label = -1;
  float inv_s1 = 0.0f;
  const bool hard = p.alpha > 0.0f && (label = p.labels[n]) >= 0;
  if (hard) {
    float m1, s1;
    row_stats(z, p.V, 1.0f, buf, m1, s1);
    inv_s1 = s1 == 0.0f ? 0.0f : 1.0f / s1;
    const float lp = label < p.V ? (to_f32(z[label]) - ref) - logf(s1 == 0.0f ? 1.0f : s1) : NAN;
    loss -= p.alpha * lp;
    if (label >= p.V) inv_s1 = NAN;
  }
  if (tid == 0) p.loss[n] = loss;
  if (!grad) return;
  auto value = [&](float zj, float factor, float qj, bool is_label) {
    const float d = zj - ref;
    float g = soft * (expf(d * inv_tau) * inv_s * factor - qj);
    if (hard) g += p.alpha * (expf(d) * inv_s1 - (is_label ? 1.0f : 0.0f));
    return from_f32<E>(w * g);
  };
  // the entries' logits are read before any of the row is replaced (grad may be logits)
  const E top_grad = first ? value(zk, inside, q_here, j == label) : from_f32<E>(0.0f);
  __syncthreads();
  for (int i = tid; i < p.V; i += blockDim.x) grad[i] = value(to_f32(z[i]), outside, 0.0f, i == label);
  __syncthreads();
  if (first) grad[j] = top_grad;
}

// (value, index) order of the alternatives: larger logits first, NaN above all, equal ones
// by index.
__device__ __forceinline__ unsigned long long order_key(float v, int j) {
  unsigned u = __float_as_uint(v == 0.0f ? 0.0f : v);
  u = isnan(v) ? 0xFFFFFFF0u : (u & 0x80000000u) ? ~u : u | 0x80000000u;
  return static_cast<unsigned long long>(u) << 32 | ~unsigned(j);
}

template <typename E>
__global__ void __launch_bounds__(kThreads) token_logp_stream_kernel(const LogpArgs p) {
  pdl_entry();
  __shared__ float buf[kThreads / 32];
  __shared__ unsigned long long best[kThreads / 32];
  const int64_t n = blockIdx.x;
  const E* z = static_cast<const E*>(p.logits) + n * p.ld;
  const int tid = threadIdx.x;
  const float inv_tau = 1.0f / p.tau;
  float m, s;
  row_stats(z, p.V, inv_tau, buf, m, s);
  const bool empty = m == -INFINITY && s == 0.0f;
  const float ref = m == -INFINITY ? 0.0f : m;
  const float log_s = empty ? 0.0f : logf(s);
  if (p.entropy) {
    float e = 0.0f;
    for (int j = tid; j < p.V; j += blockDim.x) {
      const float d = (to_f32(z[j]) - ref) * inv_tau;
      e += expf(d) * fmaxf(d, -1000.0f);
    }
    e = block_reduce(e, buf, Sum());
    if (tid == 0) p.entropy[n] = empty ? 0.0f : log_s - e / s;
  }
  if (tid == 0) {
    if (p.lse) p.lse[n] = empty ? -INFINITY : ref * inv_tau + log_s;
    if (p.logp) {
      const int y = p.tokens[n];
      p.logp[n] = y < 0 ? 0.0f : y >= p.V ? NAN : (to_f32(z[y]) - ref) * inv_tau - log_s;
    }
  }
  unsigned long long last = ~0ull;
  for (int k = 0; k < p.K; ++k) {
    unsigned long long b = 0;
    for (int j = tid; j < p.V; j += blockDim.x) {
      const unsigned long long key = order_key(to_f32(z[j]), j);
      if (key < last && key > b) b = key;
    }
    for (int o = 16; o > 0; o >>= 1) {
      const unsigned long long other = __shfl_xor_sync(~0u, b, o);
      b = other > b ? other : b;
    }
    __syncthreads();
    if (tid % 32 == 0) best[tid / 32] = b;
    __syncthreads();
    for (int i = 0; i < int(blockDim.x) / 32; ++i) b = best[i] > b ? best[i] : b;
    last = b;
    if (tid == 0) {
      const int j = int(~unsigned(b));
      p.top_idx[n * p.K + k] = j;
      p.top_logp[n * p.K + k] = (to_f32(z[j]) - ref) * inv_tau - log_s;
    }
  }
}

// ---- rows on chip ----
//
// A row is read once into the shared memory of a cluster of C blocks, each holding a slice of it as
// 16-byte pieces at the alignment they have in memory; all later passes read it there.  Elements of
// the first and last piece that lie outside the row are -inf.  A thread copies pieces t, t + T, ...
// of its block's slice and is the one that reads them, so the passes need no barrier between.
//
// Maximum and sum in one go: every thread takes the maximum of its own pieces, then the sum
// relative to that; warps and blocks join (m, s) pairs by m = max m_i, s = sum s_i exp((m_i - m) / tau),
// in the order that the sizes fix.  The blocks' warps write their pairs to every block of the
// cluster, which joins all of them after one cluster barrier.

constexpr int kRowThreads = 256;
constexpr int kRowWarps = kRowThreads / 32;
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

// A block's slice of a row.
template <typename E>
struct Slice {
  const E* row;
  int V;
  int shift;    // elements between the 16-byte boundary below the row's start and the row
  int piece0;   // first piece
  int pieces;   // number of pieces
  // index in the row of the slice's piece i's first element (may be negative, or past V)
  __device__ int index(int i) const { return (piece0 + i) * kPer<E> - shift; }
};

template <typename E>
__device__ __forceinline__ Slice<E> slice_of(const E* row, int V, int rank, int C) {
  Slice<E> s;
  s.row = row;
  s.V = V;
  s.shift = int(reinterpret_cast<uintptr_t>(row) % 16 / sizeof(E));
  const int all = (s.shift + V + kPer<E> - 1) / kPer<E>;
  const int per = (all + C - 1) / C;
  s.piece0 = min(rank * per, all);
  s.pieces = min(per, all - s.piece0);
  return s;
}

template <typename E>
__device__ __forceinline__ void load_slice(const Slice<E>& s, uint4* data) {
  for (int i = threadIdx.x; i < s.pieces; i += blockDim.x) {
    const int j = s.index(i);
    if (j >= 0 && j + kPer<E> <= s.V) {
      const uint32_t to = static_cast<uint32_t>(__cvta_generic_to_shared(data + i));
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(s.row + j) : "memory");
    } else {
      E e[kPer<E>];
      for (int k = 0; k < kPer<E>; ++k) e[k] = j + k >= 0 && j + k < s.V ? s.row[j + k] : from_f32<E>(-INFINITY);
      data[i] = *reinterpret_cast<const uint4*>(e);
    }
  }
  asm volatile("cp.async.commit_group;" ::: "memory");
}
__device__ __forceinline__ void load_wait() { asm volatile("cp.async.wait_group 0;" ::: "memory"); }

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

// A thread's sums over its pieces, relative to a.m.
template <typename E, bool ENTROPY, bool HARD, bool CLAMP>
__device__ __forceinline__ void thread_sums(const uint4* data, int pieces, float c, Stats& a) {
  const Vec<2> ref = splat<2>(a.m == -INFINITY ? -0.0f : -a.m), scale = splat<2>(c);
  Vec<2> s = splat<2>(0.0f), e = s, s1 = s;
#pragma unroll 2
  for (int i = threadIdx.x; i < pieces; i += blockDim.x) {
    Vec<2> v[kPairs<E>];
    unpack<E>(data[i], v);
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
      if constexpr (HARD) {
        const Vec<2> y = d * splat<2>(kLog2e);
        s1 = s1 + Vec<2>{exp2_fast(y.v[0]), exp2_fast(y.v[1])};
      }
    }
  }
  a.s = s.v[0] + s.v[1];
  a.e = e.v[0] + e.v[1];
  a.s1 = s1.v[0] + s1.v[1];
}

// A thread's statistics over its pieces.
template <typename E, bool ENTROPY, bool HARD>
__device__ __forceinline__ Stats thread_stats(const uint4* data, int pieces, float c) {
  Stats a = no_stats();
#pragma unroll 4
  for (int i = threadIdx.x; i < pieces; i += blockDim.x) a.m = fmaxf(a.m, piece_max<E>(data[i]));
  thread_sums<E, ENTROPY, HARD, false>(data, pieces, c, a);
  // 0 times -inf, from logits of -inf or far below the others: again with their x bounded
  if (ENTROPY && isnan(a.e)) thread_sums<E, ENTROPY, HARD, true>(data, pieces, c, a);
  return a;
}

// Blocks of a cluster may write to one another once all have started: row_start early, and
// row_started before the first write.
__device__ __forceinline__ void row_start(int C) {
  if (C > 1) asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory");
}
__device__ __forceinline__ void row_started(int C) {
  if (C > 1) asm volatile("barrier.cluster.wait;" ::: "memory");
}

// A cluster barrier (the block's alone where there is one block).
__device__ __forceinline__ void row_sync(int C) {
  if (C == 1)
    __syncthreads();
  else
    cg::this_cluster().sync();
}

// The row's statistics, from every thread's.  all: [kRowCluster * kRowWarps] in every block.
__device__ __forceinline__ void publish_stats(const Stats& mine, Stats* all, int rank, int C, float c) {
  const Stats a = warp_join(mine, c);
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, warps = blockDim.x / 32;
  if (C == 1) {
    if (lane == 0) all[warp] = a;
  } else if (lane < C) {
    cg::this_cluster().map_shared_rank(all, lane)[rank * warps + warp] = a;
  }
}
__device__ __forceinline__ Stats collect_stats(const Stats* all, int C, float c) {
  const int lane = threadIdx.x % 32, n = C * int(blockDim.x / 32);
  Stats a = lane < n ? all[lane] : no_stats();
  if (n > 32) join(a, lane + 32 < n ? all[lane + 32] : no_stats(), c);
  return warp_join(a, c);
}

// Writes f of every pair of elements of the slice to out: whole pieces where the output has the
// logits' alignment, else element by element.
template <typename E, typename F>
__device__ __forceinline__ void write_slice(const Slice<E>& s, const uint4* data, E* out, F f) {
  const bool same = int(reinterpret_cast<uintptr_t>(out) % 16 / sizeof(E)) == s.shift;
#pragma unroll 2
  for (int i = threadIdx.x; i < s.pieces; i += blockDim.x) {
    const int j = s.index(i);
    Vec<2> v[kPairs<E>];
    unpack<E>(data[i], v);
#pragma unroll
    for (int k = 0; k < kPairs<E>; ++k) v[k] = f(v[k]);
    const uint4 w = pack<E>(v);
    if (same && j >= 0 && j + kPer<E> <= s.V) {
      *reinterpret_cast<uint4*>(out + j) = w;
    } else {
      const E* e = reinterpret_cast<const E*>(&w);
#pragma unroll
      for (int k = 0; k < kPer<E>; ++k)
        if (j + k >= 0 && j + k < s.V) out[j + k] = e[k];
    }
  }
}

// The teacher's side of a row, taken by a block's first warp (lane l holds entries l, l + 32, ...)
// while the others go ahead with the student's row.
constexpr int kTableBits = 9;
struct Teacher {
  int at[GEM_TOP_MAX];      // index of an entry; -1: absent, or another entry has it
  float q[GEM_TOP_MAX];     // mass there, that of all entries with the index
  float z[GEM_TOP_MAX];     // the student's logit there
  int table[1 << kTableBits];
  float mass;               // sum of q
  Stats top;                // the student's entries
  int label_is_entry;
};

constexpr int kPerLane = GEM_TOP_MAX / 32;

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
  return v;
}

// Fills t; q and logq: the lane's own entries (0 and anything where absent).
template <typename E>
__device__ __forceinline__ void read_teacher(const DistillArgs& p, int64_t n, const E* z, int label, float c, Teacher& t,
                                             float (&q)[kPerLane], float (&logq)[kPerLane], float (&zk)[kPerLane]) {
  const int lane = threadIdx.x % 32;
  const float inv_tau = 1.0f / p.tau;
  int j[kPerLane];
  float most = -INFINITY;
#pragma unroll
  for (int e = 0; e < kPerLane; ++e) {
    const int k = e * 32 + lane;
    j[e] = -1;
    logq[e] = -INFINITY;
    if (k < p.K) {
      const int a = p.top_idx[n * p.K + k];
      if (a >= 0 && a < p.V) {
        logq[e] = p.top_logits[n * p.K + k] * inv_tau;
        if (logq[e] != -INFINITY) j[e] = a;
      }
    }
    zk[e] = j[e] >= 0 ? to_f32(z[j[e]]) : -INFINITY;
    most = fmaxf(most, logq[e]);
  }
  for (int i = lane; i < 1 << kTableBits; i += 32) t.table[i] = -1;
  float lse;
  if (p.teacher_lse) {
    lse = p.teacher_lse[n];
  } else {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(~0u, most, o));
    float sum = 0.0f;
#pragma unroll
    for (int e = 0; e < kPerLane; ++e)
      if (e * 32 < p.K && j[e] >= 0) sum += expf(logq[e] - most);
    lse = most + logf(warp_sum(sum));
  }
  __syncwarp();
  float mass = 0.0f;
  bool again = false, label_here = false;
  Stats top = no_stats();
#pragma unroll
  for (int e = 0; e < kPerLane; ++e) {
    q[e] = 0.0f;
    if (e * 32 >= p.K) continue;
    const int k = e * 32 + lane;
    if (j[e] >= 0) {
      logq[e] -= lse;
      q[e] = expf(logq[e]);
      mass += q[e];
      label_here |= j[e] == label;
      // a table of the indices seen: who finds an index there is not its first entry
      unsigned h = unsigned(j[e]) * 2654435761u >> (32 - kTableBits);
      for (;;) {   // (at most half of the table is ever taken)
        const int other = atomicCAS(&t.table[h], -1, j[e]);
        if (other == -1) break;
        if (other == j[e]) {
          again = true;
          break;
        }
        h = (h + 1) & ((1 << kTableBits) - 1);
      }
    }
    if (k < p.K) {
      t.at[k] = j[e];
      t.q[k] = q[e];
      t.z[k] = zk[e];
    }
  }
  mass = warp_sum(mass);
  label_here = __any_sync(~0u, label_here);
  if (__any_sync(~0u, again)) {
    // entries with the same index add up in the first of them; the others leave
    float sum[kPerLane];
    bool first[kPerLane];
    __syncwarp();
#pragma unroll
    for (int e = 0; e < kPerLane; ++e) {
      const int k = e * 32 + lane;
      sum[e] = 0.0f;
      first[e] = true;
      if (j[e] < 0) continue;
      for (int i = 0; i < p.K; ++i)
        if (t.at[i] == j[e]) {
          sum[e] += t.q[i];
          if (i < k) first[e] = false;
        }
    }
    __syncwarp();
#pragma unroll
    for (int e = 0; e < kPerLane; ++e)
      if (j[e] >= 0) {
        if (first[e])
          t.q[e * 32 + lane] = sum[e];
        else
          t.at[e * 32 + lane] = j[e] = -1;
      }
  }
  if (p.teacher_lse) {
#pragma unroll
    for (int e = 0; e < kPerLane; ++e)
      if (e * 32 < p.K) {
        Stats one = no_stats();
        if (j[e] >= 0 && !(zk[e] == -INFINITY)) one = {zk[e], 1.0f, 0.0f, 1.0f};
        if (isnan(zk[e])) one = {-INFINITY, zk[e], 0.0f, zk[e]};
        join(top, one, c);
      }
    top = warp_join(top, c);
  }
  if (lane == 0) {
    t.mass = mass;
    t.top = top;
    t.label_is_entry = label_here;
  }
}

template <typename E, bool HARD>
__global__ void __launch_bounds__(kRowThreads, 3) distill_kernel(const DistillArgs p, int C) {
  extern __shared__ uint4 data[];
  __shared__ Stats all[kRowCluster * kRowWarps];
  __shared__ Teacher teacher;
  pdl_entry();
  const int64_t n = blockIdx.x / C;
  const int rank = blockIdx.x % C, tid = threadIdx.x;
  const E* z = static_cast<const E*>(p.logits) + n * p.ld;
  E* grad = p.grad ? static_cast<E*>(p.grad) + n * p.grad_ld : nullptr;
  const Slice<E> s = slice_of(z, p.V, rank, C);
  const float w = p.row_scale ? p.row_scale[n] : 1.0f;
  if (w == 0.0f) {
    if (grad) write_slice<E>(s, data, grad, [](Vec<2>) { return splat<2>(0.0f); });
    if (rank == 0 && tid == 0) p.loss[n] = 0.0f;
    return;
  }
  row_start(C);
  load_slice(s, data);
  const float inv_tau = 1.0f / p.tau, c = kLog2e * inv_tau;
  int label = -1;
  float zl = 0.0f;
  if constexpr (HARD) {
    label = p.labels[n];
    if (label >= 0 && label < p.V) zl = to_f32(z[label]);
  }
  float q[kPerLane], logq[kPerLane], zk[kPerLane];
  if (tid < 32) read_teacher<E>(p, n, z, label, c, teacher, q, logq, zk);
  // where this block holds an element, or -1
  auto place = [&](int e) {
    const int k = e + s.shift - s.piece0 * kPer<E>;
    return e >= 0 && k >= 0 && k < s.pieces * kPer<E> ? k : -1;
  };
  const bool tail = p.teacher_lse != nullptr;
  load_wait();
  if (tail) {
    // the mass outside the entries is summed by itself (1 - sum p_k would cancel): they leave the row
    __syncthreads();
    const int k = tid < p.K ? place(teacher.at[tid]) : -1;   // (blocks have K threads or more)
    if (k >= 0) reinterpret_cast<E*>(data)[k] = from_f32<E>(-INFINITY);
    __syncthreads();
  }
  const Stats mine = thread_stats<E, false, HARD>(data, s.pieces, c);
  row_started(C);
  publish_stats(mine, all, rank, C, c);
  row_sync(C);
  const Stats rest = collect_stats(all, C, c);
  Stats r = rest;
  if (tail) join(r, teacher.top, c);
  const float ref = r.m == -INFINITY ? 0.0f : r.m;
  const float inv_s = r.s == 0.0f ? 0.0f : 1.0f / r.s;
  const float log_s = r.s == 0.0f ? 0.0f : logf(r.s);
  // With q_rest the factor of p_j outside the entries is mass + q_rest - q_rest / p_rest.  Exponentials
  // outside are taken relative to the largest logit there, low: p_j = exp((z_j - low) / tau) to_low.
  const float low = tail && rest.s > 0.0f ? rest.m : ref;
  const float to_low = exp2_fast((low - ref) * c) * inv_s;
  const float mass = teacher.mass;
  float factor = mass, rest_share = 0.0f, kl_rest = 0.0f;
  if (tail && rest.s > 0.0f) {
    const float qr = fmaxf(1.0f - mass, 0.0f);
    factor += qr;
    rest_share = qr / rest.s;
    if (qr > 0.0f) kl_rest = qr * (logf(qr) - (logf(rest.s) + (low - ref) * inv_tau - log_s));
  }
  const float soft = (1.0f - p.alpha) * p.tau;
  bool hard = false;
  float inv_s1 = 0.0f;
  if constexpr (HARD) {
    hard = label >= 0;
    inv_s1 = label >= p.V ? NAN : hard && r.s1 != 0.0f ? 1.0f / r.s1 : 0.0f;
  }
  if (rank == 0 && tid < 32) {
    float kl = 0.0f;
#pragma unroll
    for (int e = 0; e < kPerLane; ++e)
      if (e * 32 < p.K && !(q[e] == 0.0f)) kl += q[e] * (logq[e] - ((zk[e] - ref) * inv_tau - log_s));
    kl = warp_sum(kl);
    if (tid == 0) {
      float loss = soft * p.tau * (kl + kl_rest);
      if (hard) loss -= p.alpha * (label < p.V ? (zl - ref) - (r.s1 == 0.0f ? 0.0f : logf(r.s1)) : NAN);
      p.loss[n] = loss;
    }
  }
  if (!grad) return;
  const float k_soft = w * soft, k_hard = w * p.alpha * inv_s1 * exp2_fast((low - ref) * kLog2e);
  const float k_out = k_soft * (to_low * factor - rest_share);
  const Vec<2> neg_low = splat<2>(-low);
  auto outside = [&](Vec<2> v) {
    const Vec<2> d = v + neg_low, x = d * splat<2>(c);
    Vec<2> g = splat<2>(k_out) * Vec<2>{exp2_grad<E>(x.v[0]), exp2_grad<E>(x.v[1])};
    if constexpr (HARD) {
      const Vec<2> y = d * splat<2>(kLog2e);
      g = fma<2>(splat<2>(k_hard), Vec<2>{exp2_grad<E>(y.v[0]), exp2_grad<E>(y.v[1])}, g);
    }
    return g;
  };
  write_slice<E>(s, data, grad, outside);
  // the entries' and the label's own values, over what was just written
  __syncthreads();
  for (int k = tid; k < p.K; k += blockDim.x) {
    const int j = teacher.at[k];
    if (place(j) < 0) continue;
    const float d = teacher.z[k] - ref;
    float g = k_soft * (exp2_grad<E>(d * c) * inv_s * factor - teacher.q[k]);
    if (HARD && hard) g += w * p.alpha * (inv_s1 * exp2_grad<E>(d * kLog2e) - (j == label ? 1.0f : 0.0f));
    grad[j] = from_f32<E>(g);
  }
  if (HARD && tid == 0 && hard && label < p.V && !teacher.label_is_entry && place(label) >= 0)
    grad[label] = from_f32<E>(outside(splat<2>(zl)).v[0] - w * p.alpha);
}

// Top K of a row on chip.  The blocks' threads are cut into G groups of neighbours; the K-th largest
// of the groups' maxima is a bound that K elements reach, and few others do (about G ln(G / (G - K))
// for elements in no order).  Those that do are collected and ranked against one another.  Where
// more reach it than the lists hold (ties, adverse orders), and in rows that are not finite, K
// rounds each find the next element instead.
constexpr int kMaxGroups = 1024;
constexpr int kList = 512;

struct TopShared {
  float group_max[kMaxGroups];
  unsigned long long list[kList];
  unsigned long long best[kRowWarps];
  unsigned long long round_best[2][kRowCluster];
  int count, counts[kRowCluster];
  float bound;
};

// A value that at least K of the G (at least K) values reach, and hardly more do: bisection over the
// floats in their order, ended when at most K / 4 too many remain.  One warp calls.
__device__ __forceinline__ float group_bound(const float* values, int G, int K) {
  const int lane = threadIdx.x % 32;
  auto order = [](float v) {
    const int u = __float_as_int(v);
    return u ^ (u >> 31 & 0x7fffffff);
  };
  int lo = INT32_MAX, hi = INT32_MIN;
  for (int i = lane; i < G; i += 32) {
    const int v = order(values[i]);
    lo = min(lo, v);
    hi = max(hi, v);
  }
  lo = __reduce_min_sync(~0u, lo);
  hi = __reduce_max_sync(~0u, hi);
  // K values reach lo; fewer than K reach hi + 1
  int reach = G;
  while (lo < hi && reach > K + K / 4) {
    const int mid = int((int64_t(lo) + hi + 1) >> 1);
    int n = 0;
    for (int i = lane; i < G; i += 32) n += order(values[i]) >= mid;
    n = __reduce_add_sync(~0u, n);
    if (n >= K) {
      lo = mid;
      reach = n;
    } else {
      hi = mid - 1;
    }
  }
  return __int_as_float(lo ^ (lo >> 31 & 0x7fffffff));
}

__device__ __forceinline__ int key_index(unsigned long long key) { return int(~unsigned(key)); }

// Calls f(key) for every element of the thread's pieces.
template <typename E, typename F>
__device__ __forceinline__ void each_key(const Slice<E>& s, const uint4* data, F f) {
  for (int i = threadIdx.x; i < s.pieces; i += blockDim.x) {
    const uint4 w = data[i];
    const int j = s.index(i);
    Vec<2> v[kPairs<E>];
    unpack<E>(w, v);
#pragma unroll
    for (int k = 0; k < kPer<E>; ++k)
      if (j + k >= 0 && j + k < s.V) f(order_key(v[k / 2].v[k % 2], j + k));
  }
}

template <typename E>
__global__ void __launch_bounds__(kRowThreads, 3) token_logp_kernel(const LogpArgs p, int C, int group_lanes) {
  extern __shared__ uint4 data[];
  __shared__ Stats all[kRowCluster * kRowWarps];
  __shared__ TopShared top;
  pdl_entry();
  const int64_t n = blockIdx.x / C;
  const int rank = blockIdx.x % C, tid = threadIdx.x, T = blockDim.x, lane = tid % 32;
  const E* z = static_cast<const E*>(p.logits) + n * p.ld;
  const Slice<E> s = slice_of(z, p.V, rank, C);
  row_start(C);
  load_slice(s, data);
  const float inv_tau = 1.0f / p.tau, c = kLog2e * inv_tau;
  int y = -1;
  float zy = 0.0f;
  if (rank == 0 && tid == 0 && p.logp) {
    y = p.tokens[n];
    if (y >= 0 && y < p.V) zy = to_f32(z[y]);
  }
  if (tid == 0) top.count = 0;
  load_wait();
  const Stats mine = thread_stats<E, true, false>(data, s.pieces, c);
  row_started(C);
  publish_stats(mine, all, rank, C, c);
  const int per_block = T / group_lanes, groups = per_block * C;
  if (p.K > 0) {
    float g = mine.m;
    for (int o = 1; o < group_lanes; o <<= 1) g = fmaxf(g, __shfl_xor_sync(~0u, g, o));
    const int id = rank * per_block + tid / group_lanes;
    for (int k = tid % group_lanes; k < C; k += group_lanes)
      (C == 1 ? &top : cg::this_cluster().map_shared_rank(&top, k))->group_max[id] = g;
  }
  row_sync(C);
  const Stats r = collect_stats(all, C, c);
  const bool empty = r.m == -INFINITY && r.s == 0.0f;
  const float ref = r.m == -INFINITY ? 0.0f : r.m;
  const float log_s = empty ? 0.0f : logf(r.s);
  if (rank == 0 && tid == 0) {
    if (p.entropy) p.entropy[n] = empty ? 0.0f : log_s - r.e / r.s * (1.0f / kLog2e);
    if (p.lse) p.lse[n] = empty ? -INFINITY : ref * inv_tau + log_s;
    if (p.logp) p.logp[n] = y < 0 ? 0.0f : y >= p.V ? NAN : (zy - ref) * inv_tau - log_s;
  }
  if (p.K == 0) return;
  auto write = [&](int k, unsigned long long key) {
    p.top_idx[n * p.K + k] = key_index(key);
    p.top_logp[n * p.K + k] = (to_f32(z[key_index(key)]) - ref) * inv_tau - log_s;
  };
  bool listed = !isnan(r.s);
  if (listed) {
    if (tid < 32) {
      const float bound = group_bound(top.group_max, groups, p.K);
      if (tid == 0) top.bound = bound;
    }
    __syncthreads();
    const float bound = top.bound;
    // a thread whose maximum reaches the bound: its pieces are searched by the warp together
    for (unsigned hit = __ballot_sync(~0u, mine.m >= bound); hit; hit &= hit - 1) {
      const int owner = tid - lane + __ffs(hit) - 1;
      for (int i = owner + lane * T; i < s.pieces; i += 32 * T) {
        const uint4 w = data[i];
        if (piece_max<E>(w) < bound) continue;
        const int j = s.index(i);
        Vec<2> v[kPairs<E>];
        unpack<E>(w, v);
#pragma unroll
        for (int k = 0; k < kPer<E>; ++k) {
          const float x = v[k / 2].v[k % 2];
          if (x >= bound && j + k >= 0 && j + k < s.V) {
            const int at = atomicAdd(&top.count, 1);   // (the order in the list does not matter)
            if (at < kList) top.list[at] = order_key(x, j + k);
          }
        }
      }
    }
    __syncthreads();
    if (C > 1 && tid < C) cg::this_cluster().map_shared_rank(&top, tid)->counts[rank] = top.count;
    if (C == 1 && tid == 0) top.counts[0] = top.count;
    row_sync(C);
    int total = 0;
    for (int k = 0; k < C; ++k) total += top.counts[k] > kList ? kList * kRowCluster + 1 : top.counts[k];
    listed = total <= kList;
    if (listed) {
      // the first block takes the lists together: its own stays, the others' follow
      if (rank == 0 && C > 1) {
        int from = top.counts[0];
        for (int b = 1; b < C; ++b) {
          const unsigned long long* theirs = cg::this_cluster().map_shared_rank(&top, b)->list;
          for (int k = tid; k < top.counts[b]; k += T) top.list[from + k] = theirs[k];
          from += top.counts[b];
        }
      }
      row_sync(C);
      if (rank == 0)
        for (int i = tid; i < total; i += T) {
          const unsigned long long key = top.list[i];
          int above = 0;
          for (int k = 0; k < total; ++k) above += top.list[k] > key;
          if (above < p.K) write(above, key);
        }
      return;
    }
  }
  unsigned long long last = ~0ull;
  for (int k = 0; k < p.K; ++k) {
    unsigned long long b = 0;
    each_key<E>(s, data, [&](unsigned long long key) {
      if (key < last && key > b) b = key;
    });
    for (int o = 16; o > 0; o >>= 1) {
      const unsigned long long other = __shfl_xor_sync(~0u, b, o);
      b = other > b ? other : b;
    }
    if (lane == 0) top.best[tid / 32] = b;
    __syncthreads();
    for (int i = 0; i < T / 32; ++i) b = top.best[i] > b ? top.best[i] : b;
    if (C > 1) {
      if (tid < C) cg::this_cluster().map_shared_rank(&top, tid)->round_best[k & 1][rank] = b;
      row_sync(C);
      for (int i = 0; i < C; ++i) b = top.round_best[k & 1][i] > b ? top.round_best[k & 1][i] : b;
    } else {
      __syncthreads();
    }
    last = b;
    if (rank == 0 && tid == 0) write(k, b);
  }
  row_sync(C);   // no block leaves while another may still write to it
}

// ---- gradient of log probability and entropy: one pass, block by block of a row's pieces ----

constexpr int kGradPieces = 4;   // of a thread

template <typename E>
__global__ void __launch_bounds__(kRowThreads) token_logp_grad_kernel(const LogpGradArgs p, int blocks_per_row) {
  pdl_entry();
  const int64_t n = blockIdx.x / blocks_per_row;
  const int part = blockIdx.x % blocks_per_row;
  const E* z = static_cast<const E*>(p.logits) + n * p.ld;
  E* grad = static_cast<E*>(p.grad) + n * p.grad_ld;
  const Slice<E> s = slice_of(z, p.V, 0, 1);
  const bool same = int(reinterpret_cast<uintptr_t>(grad) % 16 / sizeof(E)) == s.shift;
  const int first = part * kGradPieces * kRowThreads + threadIdx.x;
  uint4 w[kGradPieces];
#pragma unroll
  for (int i = 0; i < kGradPieces; ++i) {
    const int j = s.index(first + i * kRowThreads);
    if (j >= 0 && j + kPer<E> <= s.V) {
      w[i] = *reinterpret_cast<const uint4*>(z + j);
    } else {
      E e[kPer<E>];
      for (int k = 0; k < kPer<E>; ++k) e[k] = j + k >= 0 && j + k < s.V ? z[j + k] : from_f32<E>(0.0f);
      w[i] = *reinterpret_cast<const uint4*>(e);
    }
  }
  const float inv_tau = 1.0f / p.tau;
  const float lse = p.lse[n];
  int y = -1;
  float dl = 0.0f;
  if (p.dlogp) {
    y = p.tokens[n];
    if (y >= 0) dl = y < p.V ? p.dlogp[n] : NAN;
  }
  const float dh = p.dentropy ? p.dentropy[n] : 0.0f;
  const float H = p.dentropy ? p.entropy[n] : 0.0f;
  const float none = lse == -INFINITY ? 0.0f : 1.0f;   // a row without mass: p = 0
  const float off = lse == -INFINITY ? 0.0f : lse;
#pragma unroll
  for (int i = 0; i < kGradPieces; ++i) {
    const int j = s.index(first + i * kRowThreads);
    if (j >= s.V) break;
    Vec<2> v[kPairs<E>];
    unpack<E>(w[i], v);
#pragma unroll
    for (int k = 0; k < kPairs<E>; ++k) {
      const Vec<2> lp = fma<2>(v[k], splat<2>(inv_tau), splat<2>(-off)), x = lp * splat<2>(kLog2e);
      const Vec<2> e = Vec<2>{exp2_grad<E>(x.v[0]), exp2_grad<E>(x.v[1])} * splat<2>(-none);
      const Vec<2> bounded = {fmaxf(lp.v[0], -1000.0f), fmaxf(lp.v[1], -1000.0f)};
      Vec<2> g = e * fma<2>(splat<2>(dh), bounded, splat<2>(fmaf(dh, H, dl)));
#pragma unroll
      for (int m = 0; m < 2; ++m)
        if (j + 2 * k + m == y) g.v[m] += dl;
      v[k] = g * splat<2>(inv_tau);
    }
    const uint4 o = pack<E>(v);
    if (same && j >= 0 && j + kPer<E> <= s.V) {
      *reinterpret_cast<uint4*>(grad + j) = o;
    } else {
      const E* e = reinterpret_cast<const E*>(&o);
#pragma unroll
      for (int k = 0; k < kPer<E>; ++k)
        if (j + k >= 0 && j + k < s.V) grad[j + k] = e[k];
    }
  }
}

// How a row is held: blocks of a cluster, threads of a block and bytes of shared memory.  Slices of
// up to 64 KB let three blocks share an SM, so that one loads or stores while another computes; few
// rows are cut further, down to 8 KB, to use more SMs.  cluster = 0: the row does not fit on chip.
struct RowCut {
  int cluster, threads;
  size_t smem;
};

RowCut row_cut(int dtype, int64_t N, int64_t V, int K) {
  constexpr int64_t kSlice = 65 << 10, kLeast = 8 << 10, kMost = 200 << 10;
  const int64_t bytes = V * dtype_size(dtype) + 32;   // with the pieces at both ends
  RowCut c = {1, kRowThreads, 0};
  while (c.cluster < kRowCluster && bytes > kSlice * c.cluster) c.cluster *= 2;
  while (c.cluster < kRowCluster && N * c.cluster < 2 * 152 && bytes >= 2 * kLeast * c.cluster) c.cluster *= 2;
  c.smem = size_t((bytes / 16 + c.cluster) / c.cluster + 1) * 16;
  if (int64_t(c.smem) > kMost) return {0, 0, 0};
  if (c.smem <= 8192 && K <= 128) c.threads = 128;
  return c;
}

template <typename Kernel, typename... Args>
cudaError_t launch_rows(Kernel kernel, const RowCut& c, int64_t N, cudaStream_t stream, Args... args) {
  const cudaError_t e = allow_smem(kernel, c.smem);
  if (e != cudaSuccess) return e;
  return launch_cluster_pdl(kernel, unsigned(N * c.cluster), unsigned(c.threads), unsigned(c.cluster), c.smem, stream, args...);
}

template <typename E>
cudaError_t launch_distill(const DistillArgs& p, int dtype, int64_t N, cudaStream_t stream) {
  const RowCut c = row_cut(dtype, N, p.V, p.K);
  if (c.cluster == 0) return launch_pdl(distill_stream_kernel<E>, dim3(unsigned(N)), dim3(kThreads), 0, stream, p);
  return p.alpha > 0.0f ? launch_rows(distill_kernel<E, true>, c, N, stream, p, c.cluster)
                        : launch_rows(distill_kernel<E, false>, c, N, stream, p, c.cluster);
}

template <typename E>
cudaError_t launch_logp(const LogpArgs& p, int dtype, int64_t N, cudaStream_t stream) {
  const RowCut c = row_cut(dtype, N, p.V, p.K);
  if (c.cluster == 0) return launch_pdl(token_logp_stream_kernel<E>, dim3(unsigned(N)), dim3(kThreads), 0, stream, p);
  // the widest groups of which there are at least 2 K with elements
  const int64_t pieces = (int64_t(p.V) * sizeof(E) / 16 + c.cluster) / c.cluster;
  const int64_t busy = (pieces < c.threads ? pieces : c.threads) * c.cluster;
  int lanes = 32;
  while (lanes > 1 && (busy < int64_t(2) * p.K * lanes || c.threads * c.cluster > kMaxGroups * lanes * 8)) lanes /= 2;
  while (c.threads * c.cluster > kMaxGroups * lanes) lanes *= 2;
  return launch_rows(token_logp_kernel<E>, c, N, stream, p, c.cluster, lanes);
}

template <typename E>
cudaError_t launch_logp_grad(const LogpGradArgs& p, int64_t N, cudaStream_t stream) {
  const int64_t per_block = int64_t(kGradPieces) * kRowThreads * kPer<E>;
  const int64_t blocks = (p.V + 16 + per_block - 1) / per_block;
  return launch_pdl(token_logp_grad_kernel<E>, dim3(unsigned(N * blocks)), dim3(kRowThreads), 0, stream, p, int(blocks));
}

// Grids of up to 8 blocks a row, and element indices of a row with room past its end.
constexpr int64_t kMaxRows = int64_t(1) << 27, kMaxVocabulary = int64_t(1) << 30;

bool rows_ok(int dtype, int64_t N, int64_t V, const void* z, int64_t ld) {
  if (!dtype_ok(dtype) || N < 0 || N > kMaxRows || V < 1 || V > kMaxVocabulary) return false;
  if (N == 0) return true;
  return z && aligned_to(z, size_t(dtype_size(dtype))) && (ld == 0 || ld >= V) && ld <= kMaxStride;
}

bool grad_ok(int dtype, int64_t V, const void* g, int64_t ld) {
  return g && aligned_to(g, size_t(dtype_size(dtype))) && ld >= V && ld <= kMaxStride;
}

// Within these limits neither 1 / tau nor a difference of equal logits over tau leaves fp32.
bool temperature_ok(float tau) { return tau >= 1.0e-20f && tau <= 1.0e20f; }

}  // namespace
}  // namespace lm
}  // namespace gem

using namespace gem;
using namespace gem::lm;

// Calls LAUNCH<E>(...) for the element type.
#define LAUNCH_BY_TYPE(LAUNCH, ...)                                  \
  launch_status(dtype == GEM_F32    ? LAUNCH<float>(__VA_ARGS__)         \
                : dtype == GEM_BF16 ? LAUNCH<__nv_bfloat16>(__VA_ARGS__) \
                                    : LAUNCH<__half>(__VA_ARGS__))

extern "C" {

int gem_distill(int dtype, int64_t N, int64_t V, const void* logits, int64_t ld, int K,
                const int32_t* top_idx, const float* top_logits, const float* teacher_lse,
                const int32_t* labels, const float* row_scale, float temperature, float alpha,
                float* loss, void* grad, int64_t grad_ld, void* stream) {
  if (!rows_ok(dtype, N, V, logits, ld) || !temperature_ok(temperature)) return GEM_EINVAL;
  if (K < 0 || K > GEM_TOP_MAX || !(alpha >= 0.0f && alpha <= 1.0f)) return GEM_EINVAL;
  if (N == 0) return GEM_OK;
  if (K > 0 && (!array_ok(top_idx) || !array_ok(top_logits))) return GEM_EINVAL;
  if (!optional_ok(teacher_lse) || !optional_ok(row_scale) || !array_ok(loss)) return GEM_EINVAL;
  if (alpha > 0.0f && !array_ok(labels)) return GEM_EINVAL;
  if (grad && (!grad_ok(dtype, V, grad, grad_ld) || (grad == logits && grad_ld != ld))) return GEM_EINVAL;
  const DistillArgs p = {logits, grad, ld, grad_ld, int(V), K, top_idx, top_logits, teacher_lse,
                         labels, row_scale, temperature, alpha, loss};
  return LAUNCH_BY_TYPE(launch_distill, p, dtype, N, static_cast<cudaStream_t>(stream));
}

int gem_token_logp(int dtype, int64_t N, int64_t V, const void* logits, int64_t ld,
                   const int32_t* tokens, float temperature, int K, float* logp,
                   float* entropy, float* lse, int32_t* top_idx, float* top_logp, void* stream) {
  if (!rows_ok(dtype, N, V, logits, ld) || !temperature_ok(temperature)) return GEM_EINVAL;
  if (K < 0 || K > GEM_TOP_MAX || K > V) return GEM_EINVAL;
  if (N == 0) return GEM_OK;
  if (K > 0 && (!array_ok(top_idx) || !array_ok(top_logp))) return GEM_EINVAL;
  if (!optional_ok(logp) || !optional_ok(entropy) || !optional_ok(lse)) return GEM_EINVAL;
  if (logp && !array_ok(tokens)) return GEM_EINVAL;
  const LogpArgs p = {logits, ld, int(V), K, tokens, temperature, logp, entropy, lse, top_idx, top_logp};
  return LAUNCH_BY_TYPE(launch_logp, p, dtype, N, static_cast<cudaStream_t>(stream));
}

int gem_token_logp_grad(int dtype, int64_t N, int64_t V, const void* logits, int64_t ld,
                        const int32_t* tokens, float temperature, const float* lse,
                        const float* entropy, const float* dlogp, const float* dentropy,
                        void* grad, int64_t grad_ld, void* stream) {
  if (!rows_ok(dtype, N, V, logits, ld) || !temperature_ok(temperature)) return GEM_EINVAL;
  if (N == 0) return GEM_OK;
  if (!grad_ok(dtype, V, grad, grad_ld) || (grad == logits && grad_ld != ld)) return GEM_EINVAL;
  if (!array_ok(lse) || !optional_ok(dlogp) || !optional_ok(dentropy)) return GEM_EINVAL;
  if ((dlogp && !array_ok(tokens)) || (dentropy && !array_ok(entropy))) return GEM_EINVAL;
  const LogpGradArgs p = {logits, grad, ld, grad_ld, int(V), tokens, temperature, lse, entropy, dlogp, dentropy};
  return LAUNCH_BY_TYPE(launch_logp_grad, p, N, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
