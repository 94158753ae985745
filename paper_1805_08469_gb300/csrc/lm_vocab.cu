// Losses and scores over rows of logits (include/gem_lm.h): distillation from a teacher's top
// logits, log probabilities of tokens with entropy and top alternatives, and their gradients.
#include "lm_rows.h"

namespace gem {
namespace lm {
namespace {

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
    if (j >= 0 && j < p.V) t = p.top_logits[n * p.K + tid];
    if (t == -INFINITY) j = -1;
    at[tid] = j;
  }
  const bool there = tid < p.K && j >= 0;
  float logq;
  if (p.teacher_lse) {
    logq = t * inv_tau - p.teacher_lse[n];
  } else {
    // (differences first: an offset that the logits share would round q away)
    const float d = (t - block_reduce(there ? t : -INFINITY, buf, Max())) * inv_tau;
    logq = d - logf(block_reduce(there ? expf(d) : 0.0f, buf, Sum()));
  }
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
  const float log_s = logf(s == 0.0f ? 1.0f : s);
  const float zk = there ? to_f32(z[j]) : 0.0f;
  const float logp = (zk - ref) * inv_tau - log_s;
  float kl = block_reduce(q > 0.0f ? q * (logq - logp) : 0.0f, buf, Sum()) + 0.0f * log_s;   // (NaN of a row without entries)
  float inside = mass;             // the factor of p_j in the gradient
  float low = ref, share = 0.0f;   // outside the entries also -share exp((z_j - low) / tau)
  if (p.teacher_lse) {
    // the mass outside the entries, summed by itself (1 - sum p_k would cancel) and relative to the largest
    // logit there (relative to the row's it may leave fp32)
    float top_z = -INFINITY, r = 0.0f;
    for (int i = tid; i < p.V; i += blockDim.x) {
      bool top = false;
      for (int k = 0; k < p.K; ++k) top |= at[k] == i;
      const float zi = to_f32(z[i]);
      if (top || zi == -INFINITY) continue;
      const float e = expf(-fabsf(zi - top_z) * inv_tau);
      r = zi > top_z ? r * e + 1.0f : r + e;
      top_z = fmaxf(top_z, zi);
    }
    const float most = block_reduce(top_z, buf, Max());
    if (most != -INFINITY) low = most;
    r = block_reduce(r * expf((top_z - low) * inv_tau), buf, Sum());
    const float qr = r == 0.0f ? 0.0f : fmaxf(1.0f - mass, 0.0f);
    if (qr > 0.0f) {
      kl += qr * (logf(qr) - (logf(r) + (low - ref) * inv_tau - log_s));
      inside += qr;
      share = qr / r;
    }
  }
  const float soft = (1.0f - p.alpha) * p.tau;
  float loss = soft * (p.tau * kl);   // (tau^2 may leave fp32)
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
  const float scale = expf((low - ref) * inv_tau) * inv_s * inside - share;
  auto value = [&](float zj, bool top, float qj, bool is_label) {
    float g = soft * (top ? expf((zj - ref) * inv_tau) * inv_s * inside - qj : expf((zj - low) * inv_tau) * scale);
    if (hard) g += p.alpha * (expf(zj - ref) * inv_s1 - (is_label ? 1.0f : 0.0f));
    return from_f32<E>(w * g);
  };
  // the entries' logits are read before any of the row is replaced (grad may be logits)
  const E top_grad = first ? value(zk, true, q_here, j == label) : from_f32<E>(0.0f);
  __syncthreads();
  for (int i = tid; i < p.V; i += blockDim.x) grad[i] = value(to_f32(z[i]), false, 0.0f, i == label);
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

// The teacher's side of a row, taken by the side warp (lane l holds entries l, l + 32, ...).  Arrays of
// K values in dynamic shared memory.
struct Teacher {
  int* at;          // index of an entry; -1: absent, or another entry has it
  float* q;         // mass there, that of all entries with the index
  float* z;         // the student's logit there
  uint8_t* table;   // entries by hashes of their indices, [kTable]
};
constexpr int kTableBits = 10, kTable = 1 << kTableBits;
static_assert(GEM_TOP_MAX <= 256, "an entry's number is a byte");
// What a block needs of them: 3 K words for each of two rows, and the table.
inline size_t teacher_bytes(int K) { return size_t(6) * K * 4 + kTable; }
__device__ __forceinline__ Teacher teacher_at(void* shared, int K, int b) {
  int* w = static_cast<int*>(shared);
  Teacher t;
  t.at = w + (3 * b) * K;
  t.q = reinterpret_cast<float*>(w + (3 * b + 1) * K);
  t.z = reinterpret_cast<float*>(w + (3 * b + 2) * K);
  t.table = reinterpret_cast<uint8_t*>(w + 6 * K);
  return t;
}

constexpr int kPerLane = GEM_TOP_MAX / 32;

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
  return v;
}

// The entries' part of the loss: sum q (log q - log p) = cross + mass (log S + (m - base) / tau), with base
// the entries' largest logit, so that the sum is done before m and S are known and no large terms cancel.
struct Entries {
  float mass, cross, base;
  Stats top;               // the student's statistics of the entries (where the rest is a class)
  bool label_here;         // the label is one of them
  unsigned edges_here;     // bit e: edge element e is one of them (asked for where the rest is a class)
};

template <typename E>
__device__ __forceinline__ Entries read_teacher(const DistillArgs& p, int64_t n, const Slice<E>& s, int label, float c,
                                                const Teacher& t) {
  const E* z = s.row;
  const int lane = threadIdx.x % 32;
  const float inv_tau = 1.0f / p.tau;
  int j[kPerLane];
  float logq[kPerLane], zk[kPerLane];
  float most = -INFINITY, base = -INFINITY;
  // (all loads of a kind together: their latencies overlap)
#pragma unroll
  for (int e = 0; e < kPerLane; ++e) {
    const int k = e * 32 + lane;
    j[e] = k < p.K ? p.top_idx[n * p.K + k] : -1;
    logq[e] = k < p.K ? p.top_logits[n * p.K + k] : -INFINITY;
  }
#pragma unroll
  for (int e = 0; e < kPerLane; ++e) {
    if (j[e] < 0 || j[e] >= p.V || logq[e] == -INFINITY) {
      j[e] = -1;
      logq[e] = -INFINITY;
    }
    zk[e] = j[e] >= 0 ? to_f32(z[j[e]]) : -INFINITY;
    most = fmaxf(most, logq[e]);
    base = fmaxf(base, zk[e]);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) base = fmaxf(base, __shfl_xor_sync(~0u, base, o));
  if (base == -INFINITY) base = 0.0f;
  // log q = (logit - most) / tau - lse: without the teacher's own log-sum-exp relative to the largest entry (an
  // offset that the logits share would round q away)
  float lse;
  if (p.teacher_lse) {
    most = 0.0f;
    lse = p.teacher_lse[n];
  } else {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(~0u, most, o));
    float sum = 0.0f;
#pragma unroll
    for (int e = 0; e < kPerLane; ++e)
      if (e * 32 < p.K && j[e] >= 0) sum += expf((logq[e] - most) * inv_tau);
    lse = logf(warp_sum(sum));
  }
  Entries r = {0.0f, 0.0f, base, no_stats(), false, 0u};
#pragma unroll
  for (int e = 0; e < kPerLane; ++e) {
    if (e * 32 >= p.K) continue;
    const int k = e * 32 + lane;
    float q = 0.0f;
    if (j[e] >= 0) {
      logq[e] = (logq[e] - most) * inv_tau - lse;
      q = expf(logq[e]);
      r.mass += q;
      if (q != 0.0f) r.cross += q * (logq[e] - (zk[e] - base) * inv_tau);
      r.label_here |= j[e] == label;
    }
    if (k < p.K) {
      t.at[k] = j[e];
      t.q[k] = q;
      t.z[k] = zk[e];
    }
  }
  r.mass = warp_sum(r.mass);
  r.cross = warp_sum(r.cross);
  r.label_here = __any_sync(~0u, r.label_here);
  // Do two entries have the same index?  All write their number to their index's place in the table;
  // who finds another index's number there tries again with another hash, together with those that have
  // its index, if any (they met the same).
  __syncwarp();
  bool again = false;
  unsigned open = 0;   // bit e: entry e is not settled
#pragma unroll
  for (int e = 0; e < kPerLane; ++e) open |= unsigned(j[e] >= 0) << e;
  unsigned odd = 2654435761u;
  for (int round = 0; __any_sync(~0u, open); ++round, odd = odd * 0x9E3779B1u) {
    if (round == 8) {   // (not seen: then the slow way)
      again = true;
      break;
    }
#pragma unroll
    for (int e = 0; e < kPerLane; ++e)
      if (e * 32 < p.K && (open >> e & 1)) t.table[unsigned(j[e]) * odd >> (32 - kTableBits)] = uint8_t(e * 32 + lane);
    __syncwarp();
    unsigned settled = 0;
#pragma unroll
    for (int e = 0; e < kPerLane; ++e)
      if (e * 32 < p.K && (open >> e & 1)) {
        const int there = t.table[unsigned(j[e]) * odd >> (32 - kTableBits)];
        if (t.at[there] == j[e]) {
          settled |= 1u << e;
          again |= there != e * 32 + lane;
        }
      }
    open &= ~settled;
    __syncwarp();
  }
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
        join(r.top, one, c);
      }
    r.top = warp_join(r.top, c);
    for (int i = 0; i < s.edges(); ++i) {
      bool here = false;
#pragma unroll
      for (int e = 0; e < kPerLane; ++e) here |= j[e] == s.edge(i);
      r.edges_here |= unsigned(__any_sync(~0u, here)) << i;
    }
  }
  __syncwarp();
  return r;
}

// What the gradient of a row needs beside its elements.
struct Coefficients {
  float ref, log_s, inv_s;   // largest logit (0 where there is none), log and inverse of the sum
  float factor;              // of p_j at the entries
  float low, k_out, k_hard;  // outside: k_out exp((z - low) / tau) + k_hard exp(z - low)
  float k_soft, k_one, inv_s1, kl_rest;
};

template <Hard HARD>
__device__ __forceinline__ Coefficients coefficients(const DistillArgs& p, const Stats& rest, const Stats& top, float mass,
                                                     float w, int label, float c) {
  const bool tail = p.teacher_lse != nullptr;
  Stats r = rest;
  if (tail) join(r, top, c);
  Coefficients k;
  k.ref = r.m == -INFINITY ? 0.0f : r.m;
  k.inv_s = r.s == 0.0f ? 0.0f : 1.0f / r.s;
  k.log_s = r.s == 0.0f ? 0.0f : logf(r.s);
  // With q_rest the factor of p_j outside the entries is mass + q_rest - q_rest / p_rest.  Exponentials
  // outside are taken relative to the largest logit there, low.
  // (a NaN logit makes the rest's sum NaN, and with it all of the row)
  const bool rest_left = tail && !(rest.s == 0.0f);
  k.low = rest_left ? rest.m : k.ref;
  k.factor = mass;
  k.kl_rest = 0.0f;
  float rest_share = 0.0f;
  if (rest_left) {
    const float qr = fmaxf(1.0f - mass, 0.0f);
    k.factor += qr;
    rest_share = qr / rest.s;
    if (qr > 0.0f) k.kl_rest = qr * (logf(qr) - (logf(rest.s) + (k.low - k.ref) * (1.0f / p.tau) - k.log_s));
  }
  k.k_soft = w * (1.0f - p.alpha) * p.tau;
  k.k_one = w * p.alpha;
  k.inv_s1 = !HARD ? 0.0f : label >= p.V ? NAN : label >= 0 && r.s1 != 0.0f ? 1.0f / r.s1 : 0.0f;
  k.k_out = k.k_soft * (exp2_fast((k.low - k.ref) * c) * k.inv_s * k.factor - rest_share);
  k.k_hard = !HARD ? 0.0f : k.k_one * k.inv_s1 * exp2_fast((k.low - k.ref) * kLog2e);
  return k;
}

template <typename E, Hard HARD>
__device__ __forceinline__ Vec<2> outside_grad(Vec<2> v, const Coefficients& k, float c) {
  const Vec<2> d = v + splat<2>(-k.low), x = d * splat<2>(c);
  const Vec<2> e = {exp2_grad<E>(x.v[0]), exp2_grad<E>(x.v[1])};
  if constexpr (HARD == kNoLabels) return splat<2>(k.k_out) * e;
  if constexpr (HARD == kTau1) return splat<2>(k.k_out + k.k_hard) * e;
  if constexpr (HARD == kTau2) return fma<2>(splat<2>(k.k_hard), e, splat<2>(k.k_out)) * e;
  const Vec<2> y = d * splat<2>(kLog2e);
  return fma<2>(splat<2>(k.k_hard), Vec<2>{exp2_grad<E>(y.v[0]), exp2_grad<E>(y.v[1])}, splat<2>(k.k_out) * e);
}

// Writes the gradient of one piece (LIVE: of a row whose scale is not 0) to out, at any alignment.
template <typename E, Hard HARD, bool LIVE>
__device__ __forceinline__ void write_piece(const uint4& w, E* out, bool aligned, const Coefficients& k, float c) {
  uint4 g = make_uint4(0, 0, 0, 0);
  if constexpr (LIVE) {
    Vec<2> v[kPairs<E>];
    unpack<E>(w, v);
#pragma unroll
    for (int m = 0; m < kPairs<E>; ++m) v[m] = outside_grad<E, HARD>(v[m], k, c);
    g = pack<E>(v);
  }
  if (aligned) {
    *reinterpret_cast<uint4*>(out) = g;
  } else {
    const E* e = reinterpret_cast<const E*>(&g);
#pragma unroll
    for (int m = 0; m < kPer<E>; ++m) out[m] = e[m];
  }
}

// The entries' and the label's own values of a row (zl: the label's logit), over what was written there.
// One warp calls.
template <typename E, Hard HARD>
__device__ __forceinline__ void write_entries(const DistillArgs& p, const Teacher& t, const Coefficients& k, float c, int label,
                                              bool label_is_entry, float zl, E* out) {
  const int lane = threadIdx.x % 32;
  for (int i = lane; i < p.K; i += 32) {
    const int j = t.at[i];
    if (j < 0) continue;
    const float d = t.z[i] - k.ref;
    float g = k.k_soft * (exp2_grad<E>(d * c) * k.inv_s * k.factor - t.q[i]);
    if (HARD && label >= 0) g += k.k_one * (k.inv_s1 * exp2_grad<E>(d * kLog2e) - (j == label ? 1.0f : 0.0f));
    out[j] = from_f32<E>(g);
  }
  if (HARD && lane == 0 && label >= 0 && label < p.V && !label_is_entry)
    out[label] = from_f32<E>(outside_grad<E, HARD>(splat<2>(zl), k, c).v[0] - k.k_one);
}

// A row's loss.
template <Hard HARD>
__device__ __forceinline__ float row_loss(const DistillArgs& p, const Coefficients& k, const Entries& entries, int label, float zl) {
  // (a NaN in the row makes log_s NaN, which a row without entries keeps)
  const float kl = entries.mass == 0.0f ? 0.0f * k.log_s : entries.cross + entries.mass * ((k.ref - entries.base) * (1.0f / p.tau) + k.log_s);
  float loss = (1.0f - p.alpha) * p.tau * (p.tau * (kl + k.kl_rest));   // (tau^2 may leave fp32)
  if (HARD && label >= 0)
    loss -= p.alpha * (label < p.V ? (zl - k.ref) + (k.inv_s1 == 0.0f ? 0.0f : logf(k.inv_s1)) : NAN);
  return loss;
}

template <typename E, Hard HARD>
__global__ void __launch_bounds__(kRowThreads + 32, 3) distill_kernel(const DistillArgs p, int64_t N, int C, int slots) {
  extern __shared__ uint4 data[];
  __shared__ Stats all[2][kRowCluster * kRowParts];
  __shared__ Stats tops[2];
  __shared__ float masses[2];
  pdl_entry();
  const int rank = blockIdx.x % C, tid = threadIdx.x, T = blockDim.x - 32, parts = blockDim.x / 32, lane = tid % 32;
  const int64_t step = gridDim.x / C;
  void* const teachers = data + slots;
  const float c = kLog2e * (1.0f / p.tau);
  const bool tail = p.teacher_lse != nullptr;
  const E* const logits = static_cast<const E*>(p.logits);
  E* const grads = static_cast<E*>(p.grad);
  auto scale = [&](int64_t n) { return n < N ? p.row_scale ? p.row_scale[n] : 1.0f : 0.0f; };
  auto label_of = [&](int64_t n) { return HARD && n < N ? p.labels[n] : -1; };
  int64_t n = blockIdx.x / C;
  float w = scale(n);
  int label = label_of(n);
  cluster_started();

  if (tid < T) {
    Slice<E> s = slice_of(logits + n * p.ld, p.V, rank, C);
    if (w != 0.0f)
      for (int i = tid; i < s.pieces; i += T) load_piece(data + i, s.data() + i);
    load_commit();
    cluster_wait();
    for (int b = 0; n < N; n += step, b ^= 1) {
      // the next row, whose pieces follow this one's
      const float next_w = scale(n + step);
      const int next_label = label_of(n + step);
      const Slice<E> next = slice_of(logits + (n + step) * p.ld, p.V, rank, C);
      const int next_pieces = n + step < N && next_w != 0.0f ? next.pieces : 0;
      load_wait();
      if (tail) {
        // the mass outside the entries is summed by itself (1 - sum p_k would cancel): they leave the row
        part_sync(1, T + 32);
        const int j = tid < p.K && w != 0.0f ? teacher_at(teachers, p.K, b).at[tid] : -1;   // (T >= K)
        const int at = j - s.index(0);
        if (j >= 0 && at >= 0 && at < s.pieces * kPer<E>) reinterpret_cast<E*>(data)[at] = from_f32<E>(-INFINITY);
        part_sync(2, T);
      }
      Stats mine = no_stats();
      if (w != 0.0f) {
        mine.m = thread_max<E>(data, s.pieces, tid, T);
        thread_sums<E, false, HARD, false>(data, s.pieces, tid, T, c, mine, [](int) {});
      }
      publish_stats(mine, all[b], rank, C, parts, c);
      cluster_arrive();
      cluster_wait();
      const Coefficients k = coefficients<HARD>(p, collect_stats(all[b], C, parts, c), tops[b], masses[b], w, label, c);
      E* const out = grads ? grads + n * p.grad_ld + s.index(0) : nullptr;
      const bool aligned = reinterpret_cast<uintptr_t>(out) % 16 == 0;
      const int most = max(s.pieces, next_pieces);
      auto write = [&](auto live) {
#pragma unroll 2
        for (int i = tid; i < most; i += T) {
          if (i < s.pieces) write_piece<E, HARD, decltype(live)::value>(data[i], out + int64_t(i) * kPer<E>, aligned, k, c);
          if (i < next_pieces) load_piece(data + i, next.data() + i);
        }
      };
      if (!grads) {
        for (int i = tid; i < next_pieces; i += T) load_piece(data + i, next.data() + i);
      } else if (w != 0.0f) {
        write(std::true_type());
      } else {
        write(std::false_type());
      }
      load_commit();
      s = next;
      w = next_w;
      label = next_label;
    }
    cluster_arrive();
    cluster_wait();
    return;
  }

  // the side warp.  The first block's does the row's loss, edges and entries; the others' know the
  // teacher only where the entries leave their slices.
  Coefficients k = {};
  E* out = nullptr;
  float zl = 0.0f;
  int last_label = -1;
  bool label_is_entry = false;
  bool pending = false;   // the entries' and the label's own values of the row before, over what was written there
  auto finish = [&](const Teacher& t) { write_entries<E, HARD>(p, t, k, c, last_label, label_is_entry, zl, out); };
  cluster_wait();
  int b = 0;
  for (; n < N; n += step, b ^= 1) {
    const E* z = logits + n * p.ld;
    const Slice<E> s = slice_of(z, p.V, rank, C);
    const Teacher t = teacher_at(teachers, p.K, b);
    Entries entries = {0.0f, 0.0f, 0.0f, no_stats(), false, 0u};
    const bool live = w != 0.0f;
    Stats edge = no_stats();
    float ze = 0.0f, next_zl = 0.0f;
    const int je = lane < s.edges() ? s.edge(lane) : -1;
    if (live) {
      if (HARD && label >= 0 && label < p.V) next_zl = to_f32(z[label]);
      if (rank == 0 && je >= 0) ze = to_f32(z[je]);
      if (rank == 0 || tail) entries = read_teacher<E>(p, n, s, label, c, t);
      if (rank == 0 && je >= 0 && !(entries.edges_here >> lane & 1)) edge = one_element(ze);
    }
    if (tail) {
      if (lane == 0) tops[b] = entries.top;
      part_sync(1, T + 32);
    }
    if (rank == 0 && lane < C) *of_block(&masses[b], lane) = entries.mass;
    publish_edges(edge, s.edges() > 0, all[b], rank, C, parts, c);
    cluster_arrive();
    cluster_wait();
    if (rank == 0) {
      if (pending) finish(teacher_at(teachers, p.K, b ^ 1));
      pending = live && grads;
      out = grads + n * p.grad_ld;
      last_label = label;
      label_is_entry = entries.label_here;
      zl = next_zl;
      float loss = 0.0f;
      if (live) {
        const Stats rest = collect_stats(all[b], C, parts, c);
        k = coefficients<HARD>(p, rest, entries.top, entries.mass, w, label, c);
        loss = row_loss<HARD>(p, k, entries, label, zl);
      }
      if (lane == 0) p.loss[n] = loss;
      if (grads && je >= 0) out[je] = from_f32<E>(live ? outside_grad<E, HARD>(splat<2>(ze), k, c).v[0] : 0.0f);
      __syncwarp();
    }
    w = scale(n + step);
    label = label_of(n + step);
  }
  cluster_arrive();
  cluster_wait();
  if (rank == 0 && pending) finish(teacher_at(teachers, p.K, b ^ 1));
}

// Top K of a row on chip.  Threads record the largest element of their pieces, the piece it is in, and
// the largest of their other pieces.  They are cut into G groups of neighbours; the K-th largest of the
// groups' maxima is a bound that K elements reach, and few others do (about G ln(G / (G - K)) for
// elements in no order).  A block's search warp looks for them: in the recorded piece of each thread
// whose maximum reaches the bound (read again, from L2), and in all pieces of the few whose second
// value does.  It sends them to one block of the cluster, whose rank warp sorts them.  Where more
// reach the bound than the list holds (ties, adverse orders), and in rows that are not finite, that warp
// finds the K-th element exactly, by bisection over the row.
//
// Dynamic shared memory after the slots, twice each (rows take turns):
//   list [entries]       the block that ranks the row: keys of the elements that reached the bound, a
//                        share for each block
//   group_max [groups]   (the last group is the edge elements)
//   counts [C]           the block that ranks the row: elements of each block that reached the bound
//   best, second [T]     threads' recorded values, and
//   where [T]            their pieces
// and owners [T].
__host__ __device__ inline int top_entries(int K) { return K < 64 ? 256 : 4 * K; }
template <typename E>
size_t top_bytes(int K, int groups, int T) {
  return K == 0 ? 0 : size_t(2) * (top_entries(K) * 8 + (groups + kRowCluster) * 4 + T * (2 * sizeof(E) + 1)) + T;
}
template <typename E>
struct TopShared {
  unsigned long long* lists;
  int entries, groups, T;
  __device__ TopShared(void* shared, int K, int groups, int T)
      : lists(static_cast<unsigned long long*>(shared)), entries(top_entries(K)), groups(groups), T(T) {}
  __device__ unsigned long long* list(int b) const { return lists + b * entries; }
  __device__ float* group_max(int b) const { return reinterpret_cast<float*>(list(2)) + b * groups; }
  __device__ int* counts(int b) const { return reinterpret_cast<int*>(group_max(2)) + b * kRowCluster; }
  __device__ E* best(int b) const { return reinterpret_cast<E*>(counts(2)) + 2 * b * T; }
  __device__ E* second(int b) const { return best(b) + T; }
  __device__ uint8_t* where(int b) const { return reinterpret_cast<uint8_t*>(best(2)) + b * T; }
  __device__ uint8_t* owners() const { return where(2); }
};
static_assert(kRowThreads <= 256, "a thread's number is a byte");

// Order of the alternatives in 32 bits: larger logits above, NaN above all, -0 as 0.
__device__ __forceinline__ unsigned value_order(float v) { return unsigned(order_key(v, 0) >> 32); }
__device__ __forceinline__ float key_value(unsigned long long key) {
  const unsigned u = unsigned(key >> 32);
  return u == 0xFFFFFFF0u ? NAN : __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u);
}
__device__ __forceinline__ int key_index(unsigned long long key) { return int(~unsigned(key)); }

// Group maxima that may reach a bound: 8 or K / 4 more than the K it takes, but no more than two thirds of the
// groups (the elements that do grow without limit towards all of them), and K at least.
__device__ __forceinline__ int bound_reach(int G, int K) { return max(K, min(K + (K < 32 ? 8 : K / 4), 2 * G / 3)); }

// A value that at least K of the G (at least K) values reach, and hardly more do: bisection over the
// floats in their order, ended when few too many remain.  One warp calls.
__device__ __forceinline__ float group_bound(const float* values, int G, int K) {
  const int lane = threadIdx.x % 32;
  auto order = [](float v) {
    const int u = __float_as_int(v);
    return u ^ (u >> 31 & 0x7fffffff);
  };
  constexpr int kKept = 4;   // values of a lane in registers; there are hardly ever more
  int kept[kKept], lo = INT32_MAX, hi = INT32_MIN;
#pragma unroll
  for (int e = 0; e < kKept; ++e) kept[e] = lane + 32 * e < G ? order(values[lane + 32 * e]) : INT32_MIN;
  auto each = [&](auto f) {
#pragma unroll
    for (int e = 0; e < kKept; ++e)
      if (lane + 32 * e < G) f(kept[e]);
    for (int i = lane + 32 * kKept; i < G; i += 32) f(order(values[i]));
  };
  each([&](int v) {
    lo = min(lo, v);
    hi = max(hi, v);
  });
  lo = __reduce_min_sync(~0u, lo);
  hi = __reduce_max_sync(~0u, hi);
  // K values reach lo; fewer than K reach hi + 1
  int reach = G;
  // groups without an element (often the edges') would stretch the range: eight steps more, a tenth of the
  // time of 4096 x 131072 bf16 with 64 alternatives
  const int least = order(-INFINITY);
  if (lo == least) {
    int n = 0, low = INT32_MAX;
    each([&](int v) {
      n += v > least;
      low = v > least ? min(low, v) : low;
    });
    n = __reduce_add_sync(~0u, n);
    low = __reduce_min_sync(~0u, low);
    if (n >= K) {
      lo = low;
      reach = n;
    }
  }
  const int enough = bound_reach(G, K);
  while (lo < hi && reach > enough) {
    const int mid = int((int64_t(lo) + hi + 1) >> 1);
    int n = 0;
    each([&](int v) { n += v >= mid; });
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

// Takes a warp over a row in ascending index: f(orders, first, count) gets each lane's next `count`
// elements from index `first` on, lanes side by side, and returns whether to go on (the same in all).
template <typename E, typename F>
__device__ __forceinline__ void walk_row(const E* z, int V, F f) {
  const int lane = threadIdx.x % 32;
  const Slice<E> s = slice_of(z, V, 0, 1);
  unsigned o[kPer<E>] = {};
  if (lane < s.lead) o[0] = value_order(to_f32(z[lane]));
  if (!f(o, lane, lane < s.lead ? 1 : 0)) return;
  constexpr int kAhead = 4;
  for (int i0 = 0; i0 < s.pieces; i0 += 32 * kAhead) {
    uint4 w[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (i0 + 32 * u + lane < s.pieces) w[u] = s.data()[i0 + 32 * u + lane];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int i = i0 + 32 * u + lane;
      Vec<2> v[kPairs<E>] = {};
      if (i < s.pieces) unpack<E>(w[u], v);
#pragma unroll
      for (int k = 0; k < kPer<E>; ++k) o[k] = value_order(v[k / 2].v[k % 2]);
      if (!f(o, s.index(i), i < s.pieces ? kPer<E> : 0)) return;
    }
  }
  const int j = s.lead + s.whole * kPer<E> + lane;
  if (j < V) o[0] = value_order(to_f32(z[j]));
  f(o, j, j < V ? 1 : 0);
}

// The K largest elements of a row by (value, index), into list [entries] in no order.  At least K
// elements have an order of lo or above, none one above hi.  One warp calls.
template <typename E>
__device__ __noinline__ void exact_top(const E* z, int V, int K, unsigned lo, unsigned hi, unsigned long long* list, int entries) {
  const int lane = threadIdx.x % 32;
  int have = 0;
  auto collect = [&](bool ties, int most) {
    walk_row<E>(z, V, [&](const unsigned (&o)[kPer<E>], int first, int count) {
      int mine = 0;
#pragma unroll
      for (int k = 0; k < kPer<E>; ++k) mine += k < count && (ties ? o[k] == lo : o[k] > lo);
      if (!__any_sync(~0u, mine)) return true;
      int at = mine;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int other = __shfl_up_sync(~0u, at, d);
        if (lane >= d) at += other;
      }
      const int all = __shfl_sync(~0u, at, 31);
      at += have - mine;
#pragma unroll
      for (int k = 0; k < kPer<E>; ++k)
        if (k < count && (ties ? o[k] == lo : o[k] > lo)) {
          if (at < most) list[at] = static_cast<unsigned long long>(o[k]) << 32 | ~unsigned(first + k);
          ++at;
        }
      have += all;
      return have < most;
    });
  };
  // most often few elements are above lo (what reaches it is ties); else the K-th order by bisection
  collect(false, entries);
  if (have >= K) {
    while (lo < hi) {
      const unsigned mid = lo + (hi - lo) / 2 + 1;
      int n = 0;
      walk_row<E>(z, V, [&](const unsigned (&o)[kPer<E>], int, int count) {
#pragma unroll
        for (int k = 0; k < kPer<E>; ++k) n += k < count && o[k] >= mid;
        return true;
      });
      if (__reduce_add_sync(~0u, n) >= K)
        lo = mid;
      else
        hi = mid - 1;
    }
    have = 0;
    collect(false, entries);
  }
  collect(true, K);
  __syncwarp();
}

// Bitonic sort of 32 N keys, N a lane, descending: key e of lane l is number 32 e + l.  The merges into
// runs of FROM * 2, ..., TO keys, of which those of 32 N are sorted.
template <int N, int FROM, int TO>
__device__ __forceinline__ void warp_sort(unsigned long long (&v)[N]) {
  const int lane = threadIdx.x % 32;
#pragma unroll
  for (int k = 2 * FROM; k <= TO; k <<= 1)
#pragma unroll
    for (int j = k >> 1; j > 0; j >>= 1) {
      if (j >= 32) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const int o = e ^ (j / 32);
          if (o > e) {
            const bool descending = (e * 32 & k) == 0;
            const unsigned long long hi = v[e] > v[o] ? v[e] : v[o], lo = v[e] > v[o] ? v[o] : v[e];
            v[e] = descending ? hi : lo;
            v[o] = descending ? lo : hi;
          }
        }
      } else {
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const unsigned long long other = __shfl_xor_sync(~0u, v[e], j);
          const bool descending = ((e * 32 + lane) & k) == 0, lower = (lane & j) == 0;
          v[e] = (v[e] > other) == (descending == lower) ? v[e] : other;
        }
      }
    }
}

// The list's `total` keys (at most 32 N), sorted: f(rank, key) for the first K.
template <int N, typename F>
__device__ __forceinline__ void write_sorted(const unsigned long long* list, int total, int K, F f) {
  const int lane = threadIdx.x % 32;
  unsigned long long v[N];
#pragma unroll
  for (int e = 0; e < N; ++e) v[e] = e * 32 + lane < total ? list[e * 32 + lane] : 0ull;
  warp_sort<N, 1, 32 * N>(v);
#pragma unroll
  for (int e = 0; e < N; ++e)
    if (e * 32 + lane < K) f(e * 32 + lane, v[e]);
}

template <typename E>
__global__ void __launch_bounds__(kRowThreads + 64, 3) token_logp_kernel(const LogpArgs p, int64_t N, int C, int slots, int group_lanes) {
  extern __shared__ uint4 data[];
  __shared__ Stats all[2][kRowCluster * kRowParts];
  __shared__ float bounds[2];
  pdl_entry();
  // T threads stream; then there are the search warp and the rank warp
  const int rank = blockIdx.x % C, tid = threadIdx.x, T = blockDim.x - 64, parts = T / 32 + 1, lane = tid % 32;
  const int64_t step = gridDim.x / C;
  const float inv_tau = 1.0f / p.tau, c = kLog2e * inv_tau;
  const E* const logits = static_cast<const E*>(p.logits);
  const int per_block = T / group_lanes, groups = per_block * C + 1;
  const TopShared<E> top(data + slots, p.K, groups, T);
  const int share = top.entries / C;
  int64_t n = blockIdx.x / C;
  // rows' rankings go round the cluster's blocks
  int turn = 0;
  auto next_turn = [&] { turn = turn + 1 == C ? 0 : turn + 1; };
  cluster_started();

  if (tid < T) {
    Slice<E> s = slice_of(logits + n * p.ld, p.V, rank, C);
    for (int i = tid; i < s.pieces; i += T) load_piece(data + i, s.data() + i);
    load_commit();
    cluster_wait();
    for (int b = 0, row = 0; n < N; n += step, b ^= 1, ++row) {
      const Slice<E> next = slice_of(logits + (n + step) * p.ld, p.V, rank, C);
      const int next_pieces = n + step < N ? next.pieces : 0;
      load_wait();
      Stats mine = no_stats();
      float second = -INFINITY;
      int where = 0;
      if (p.K == 0) {
        mine.m = thread_max<E>(data, s.pieces, tid, T);
      } else {
#pragma unroll 4
        for (int i = tid, round = 0; i < s.pieces; i += T, ++round) {
          const float m = piece_max<E>(data[i]);
          second = fmaxf(second, fminf(mine.m, m));
          if (m > mine.m) where = round;
          mine.m = fmaxf(mine.m, m);
        }
      }
      const float m = mine.m;
      thread_sums<E, true, kNoLabels, false>(data, s.pieces, tid, T, c, mine, [&](int i) {
        if (i < next_pieces) load_piece(data + i, next.data() + i);
      });
      for (int i = s.pieces + (tid - s.pieces % T + T) % T; i < next_pieces; i += T) load_piece(data + i, next.data() + i);
      load_commit();
      // 0 times -inf, from logits of -inf or far below the others: again, with their x bounded
      if (isnan(mine.e)) thread_sums<E, true, kNoLabels, true>(s.data(), s.pieces, tid, T, c, mine, [](int) {});
      // the side warps have read what the row before last left in these buffers
      if (row > 0) cluster_wait();
      publish_stats(mine, all[b], rank, C, parts, c);
      if (p.K > 0) {
        top.best(b)[tid] = from_f32<E>(m);
        top.second(b)[tid] = from_f32<E>(second);
        top.where(b)[tid] = uint8_t(where);
        float g = m;
        for (int o = 1; o < group_lanes; o <<= 1) g = fmaxf(g, __shfl_xor_sync(~0u, g, o));
        for (int k = tid % group_lanes; k < C; k += group_lanes)
          of_block(top.group_max(b), k)[rank * per_block + tid / group_lanes] = g;
      }
      cluster_arrive();
      s = next;
    }
    cluster_wait();
    cluster_arrive();
    cluster_wait();
    return;
  }

  if (tid < T + 32) {
    // the search warp: the elements that reach a row's bound (and the edge elements' statistics)
    const unsigned below = (1u << lane) - 1;
    cluster_wait();
    for (int b = 0; n < N; n += step, b ^= 1, next_turn()) {
      const E* z = logits + n * p.ld;
      const Slice<E> s = slice_of(z, p.V, rank, C);
      const int je = rank == 0 && lane < s.edges() ? s.edge(lane) : -1;
      const float ze = je >= 0 ? to_f32(z[je]) : -INFINITY;
      const bool any = rank == 0 && s.edges() > 0;
      publish_edges(je >= 0 ? one_element(ze) : no_stats(), any, all[b], rank, C, parts, c);
      if (p.K > 0 && rank == 0) {
        float g = ze;
        if (any) {
#pragma unroll
          for (int o = 16; o > 0; o >>= 1) g = fmaxf(g, __shfl_xor_sync(~0u, g, o));
        }
        if (lane < C) of_block(top.group_max(b), lane)[groups - 1] = g;
      }
      cluster_arrive();
      cluster_wait();
      if (p.K == 0) continue;
      const float bound = group_bound(top.group_max(b), groups, p.K);
      if (rank == turn && lane == 0) bounds[b] = bound;
      unsigned long long* const to = of_block(top.list(b), turn) + rank * share;
      int count = 0;
      auto push = [&](bool want, float v, int j) {
        const unsigned votes = __ballot_sync(~0u, want);
        if (votes == 0) return;
        const int at = count + __popc(votes & below);
        if (want && at < share) to[at] = order_key(v, j);
        count += __popc(votes);
      };
      auto push_piece = [&](const uint4& w, int piece) {
        const bool in = piece < s.pieces;
        Vec<2> v[kPairs<E>] = {};
        if (in) unpack<E>(w, v);
        unsigned reach = 0;   // bit k: element k does; hardly ever two
#pragma unroll
        for (int k = 0; k < kPer<E>; ++k) reach |= unsigned(in && v[k / 2].v[k % 2] >= bound) << k;
        while (__any_sync(~0u, reach)) {
          const int k = __ffs(reach) - 1;
          float x = 0.0f;
#pragma unroll
          for (int i = 0; i < kPer<E>; ++i) x = i == k ? v[i / 2].v[i % 2] : x;
          push(reach != 0, x, s.index(piece) + k);
          reach &= reach - 1;
        }
      };
      if (any) push(je >= 0 && ze >= bound, ze, je);
      // the threads that have an element: a lane each
      int owners = 0, more = 0;
      uint8_t* const list = top.owners();
#pragma unroll 8
      for (int t = lane; t < T; t += 32) {
        const bool hit = to_f32(top.best(b)[t]) >= bound;
        const unsigned votes = __ballot_sync(~0u, hit);
        if (hit) list[owners + __popc(votes & below)] = uint8_t(t);
        owners += __popc(votes);
      }
      __syncwarp();
      for (int o0 = 0; o0 < owners && count <= share; o0 += 32) {
        const int t = o0 + lane < owners ? list[o0 + lane] : -1;
        // those with elements in several pieces are taken below instead, all their pieces
        const bool several = t >= 0 && to_f32(top.second(b)[t]) >= bound;
        const int piece = t >= 0 && !several ? t + top.where(b)[t] * T : s.pieces;
        uint4 w = {};
        if (piece < s.pieces) w = s.data()[piece];
        const unsigned votes = __ballot_sync(~0u, several);
        if (several) list[more + __popc(votes & below)] = uint8_t(t);   // (more <= o0: read already)
        more += __popc(votes);
        push_piece(w, piece);
      }
      __syncwarp();
      // lanes side by side take the pieces of one or more of them
      const int each = (s.pieces + T - 1) / T;
      int bits = 0;
      while (bits < 5 && (1 << bits) < each) ++bits;
      const int at_once = 32 >> bits, my_owner = lane >> bits, my_piece = lane & ((1 << bits) - 1);
      constexpr int kAhead = 4;
      for (int o0 = 0; o0 < more && count <= share; o0 += kAhead * at_once)
        for (int r = 0; r < each; r += 1 << bits) {
          uint4 w[kAhead];
          int piece[kAhead];
#pragma unroll
          for (int u = 0; u < kAhead; ++u) {
            const int o = o0 + u * at_once + my_owner;
            piece[u] = o < more && r + my_piece < each ? list[o] + (r + my_piece) * T : s.pieces;
            w[u] = {};
            if (piece[u] < s.pieces) w[u] = s.data()[piece[u]];
          }
#pragma unroll
          for (int u = 0; u < kAhead; ++u) {
            if (o0 + u * at_once >= more) break;
            if (__any_sync(~0u, piece[u] < s.pieces && piece_max<E>(w[u]) >= bound)) push_piece(w[u], piece[u]);
          }
        }
      if (lane == 0) of_block(top.counts(b), turn)[rank] = count;
    }
    cluster_arrive();
    cluster_wait();
    return;
  }

  // the rank warp: a row's values (the first block's), and the alternatives of the rows that are this
  // block's turn.  Other blocks have theirs before its next one, so with several blocks the sort goes
  // on over the next rows' barriers, a part after each.
  int64_t done = -1;   // the row being ranked
  Stats r = no_stats();
  int part = 0;
  constexpr int kKeys = 4;   // of a lane
  unsigned long long keys[kKeys];
  auto write = [&](int k, unsigned long long key) {
    const bool empty = r.m == -INFINITY && r.s == 0.0f;
    const float ref = r.m == -INFINITY ? 0.0f : r.m, log_s = empty ? 0.0f : logf(r.s);
    p.top_idx[done * p.K + k] = key_index(key);
    p.top_logp[done * p.K + k] = (key_value(key) - ref) * inv_tau - log_s;
  };
  // the first part takes the keys from list b
  auto rank_part = [&](int b) {
    if (part == 0) {
      unsigned long long* list = top.list(b);
      bool fits = !isnan(r.s);
      int total = 0;
      for (int k = 0; k < C; ++k) {
        const int count = top.counts(b)[k];
        fits = fits && count <= share;
        total += count;
      }
      // key number i of all shares one after the other, 0 past the last
      auto key = [&](int i) {
        if (i >= total) return 0ull;
        int k = 0;
        for (int count; i >= (count = top.counts(b)[k]); ++k) i -= count;
        return list[k * share + i];
      };
      if (fits && total <= 32) {
        unsigned long long one[1] = {key(lane)};
        warp_sort<1, 1, 32>(one);
        if (lane < p.K) write(lane, one[0]);
        done = -1;
      } else if (fits && total <= 32 * kKeys) {
#pragma unroll
        for (int e = 0; e < kKeys; ++e) keys[e] = key(e * 32 + lane);
        warp_sort<kKeys, 1, 32>(keys);
        part = 1;
      } else {
        if (fits) {
          // the shares moved together
          int to = top.counts(b)[0];
          for (int k = 1; k < C; ++k) {
            const int count = top.counts(b)[k];
            for (int i0 = 0; i0 < count; i0 += 32) {
              const unsigned long long key = i0 + lane < count ? list[k * share + i0 + lane] : 0;
              __syncwarp();
              if (i0 + lane < count) list[to + i0 + lane] = key;
            }
            to += count;
          }
        } else {
          const bool finite = !isnan(r.s);
          exact_top<E>(logits + done * p.ld, p.V, p.K, finite ? value_order(bounds[b]) : 1u,
                       finite ? value_order(r.m) : value_order(NAN), list, top.entries);
          total = p.K;
        }
        __syncwarp();
        for (int i = lane; i < total; i += 32) {
          const unsigned long long key = list[i];
          int above = 0;
#pragma unroll 8
          for (int k = 0; k < total; ++k) above += list[k] > key;
          if (above < p.K) write(above, key);
        }
        __syncwarp();
        done = -1;
      }
    } else if (part == 1) {
      warp_sort<kKeys, 32, 64>(keys);
      part = 2;
    } else {
      warp_sort<kKeys, 64, 128>(keys);
#pragma unroll
      for (int e = 0; e < kKeys; ++e)
        if (e * 32 + lane < p.K) write(e * 32 + lane, keys[e]);
      part = 0;
      done = -1;
    }
  };
  cluster_wait();
  for (int b = 0;; n += step, b ^= 1, next_turn()) {
    const bool live = n < N, mine = live && p.K > 0 && rank == turn;
    int y = -1;
    float zy = 0.0f;
    if (live && rank == 0 && p.logp) {
      y = p.tokens[n];
      if (y >= 0 && y < p.V) zy = to_f32(logits[n * p.ld + y]);
    }
    cluster_arrive();
    cluster_wait();
    while (done >= 0) {
      rank_part(b ^ 1);
      if (live && !mine) break;   // the next part after the next row
    }
    if (!live) return;
    if (rank != 0 && !mine) continue;
    const Stats now = collect_stats(all[b], C, parts, c);
    if (mine) {
      done = n;
      r = now;
    }
    if (rank == 0 && lane == 0) {
      const bool empty = now.m == -INFINITY && now.s == 0.0f;
      const float ref = now.m == -INFINITY ? 0.0f : now.m, log_s = empty ? 0.0f : logf(now.s);
      if (p.entropy) p.entropy[n] = empty ? 0.0f : log_s - now.e / now.s * (1.0f / kLog2e);
      if (p.lse) p.lse[n] = empty ? -INFINITY : ref * inv_tau + log_s;
      if (p.logp) p.logp[n] = y < 0 ? 0.0f : y >= p.V ? NAN : (zy - ref) * inv_tau - log_s;
    }
  }
}

// ---- short rows ----

constexpr int kShortOwn = kShortPieces / 32;
constexpr int kShortList = 256;
static_assert(kShortList >= GEM_TOP_MAX, "the list holds K");

// (eight blocks an SM, 64 registers a thread: 8192 x 1000 bf16 with 8 entries 15.6 us; without that bound 16.6)
template <typename E, Hard HARD>
__global__ void __launch_bounds__(kShortWarps * 32, 8) distill_short_kernel(const DistillArgs p, int64_t N, unsigned warp_bytes, int slots) {
  extern __shared__ uint4 shared[];
  pdl_entry();
  const int64_t n = int64_t(blockIdx.x) * kShortWarps + threadIdx.x / 32;
  if (n >= N) return;
  const int lane = threadIdx.x % 32;
  uint4* const data = warp_part<uint4>(shared, warp_bytes);
  const E* z = static_cast<const E*>(p.logits) + n * p.ld;
  E* const grad = p.grad ? static_cast<E*>(p.grad) + n * p.grad_ld : nullptr;
  const Slice<E> s = slice_of(z, p.V, 0, 1);
  const float w = p.row_scale ? p.row_scale[n] : 1.0f;
  const bool live = w != 0.0f, tail = p.teacher_lse != nullptr;
  const float c = kLog2e * (1.0f / p.tau);
  const int je = lane < s.edges() ? s.edge(lane) : -1;
  Coefficients k = {};
  Entries entries = {};
  const Teacher t = teacher_at(data + slots, p.K, 0);
  float ze = 0.0f, zl = 0.0f, loss = 0.0f;
  int label = -1;
  if (live) {
    load_row(s, data);
    if (je >= 0) ze = to_f32(z[je]);
    if constexpr (HARD) {
      label = p.labels[n];
      if (label >= 0 && label < p.V) zl = to_f32(z[label]);
    }
    entries = read_teacher<E>(p, n, s, label, c, t);
    load_wait();
    __syncwarp();
    if (tail) {
      for (int i = lane; i < p.K; i += 32) {
        const int at = t.at[i] - s.index(0);
        if (t.at[i] >= 0 && at >= 0 && at < s.pieces * kPer<E>) reinterpret_cast<E*>(data)[at] = from_f32<E>(-INFINITY);
      }
      __syncwarp();
    }
    Stats mine = no_stats();
    mine.m = thread_max<E>(data, s.pieces, lane, 32);
    thread_sums<E, false, HARD, false>(data, s.pieces, lane, 32, c, mine, [](int) {});
    if (je >= 0 && !(entries.edges_here >> lane & 1)) join(mine, one_element(ze), c);
    k = coefficients<HARD>(p, warp_join(mine, c), entries.top, entries.mass, w, label, c);
    loss = row_loss<HARD>(p, k, entries, label, zl);
  }
  if (lane == 0) p.loss[n] = loss;
  if (!grad) return;
  E* const out = grad + s.index(0);
  const bool aligned = reinterpret_cast<uintptr_t>(out) % 16 == 0;
  for (int i = lane; i < s.pieces; i += 32) {
    if (live)
      write_piece<E, HARD, true>(data[i], out + i * kPer<E>, aligned, k, c);
    else
      write_piece<E, HARD, false>(data[i], out + i * kPer<E>, aligned, k, c);
  }
  if (je >= 0) grad[je] = from_f32<E>(live ? outside_grad<E, HARD>(splat<2>(ze), k, c).v[0] : 0.0f);
  if (!live) return;
  __syncwarp();
  write_entries<E, HARD>(p, t, k, c, label, entries.label_here, zl, grad);
}

template <typename E>
__global__ void __launch_bounds__(kShortWarps * 32) token_logp_short_kernel(const LogpArgs p, int64_t N, unsigned warp_bytes, int slots) {
  extern __shared__ uint4 shared[];
  pdl_entry();
  const int64_t n = int64_t(blockIdx.x) * kShortWarps + threadIdx.x / 32;
  if (n >= N) return;
  const int lane = threadIdx.x % 32;
  uint4* const data = warp_part<uint4>(shared, warp_bytes);
  const E* z = static_cast<const E*>(p.logits) + n * p.ld;
  const Slice<E> s = slice_of(z, p.V, 0, 1);
  load_row(s, data);
  const float inv_tau = 1.0f / p.tau, c = kLog2e * inv_tau;
  const int je = lane < s.edges() ? s.edge(lane) : -1;
  const float ze = je >= 0 ? to_f32(z[je]) : -INFINITY;
  int y = -1;
  float zy = 0.0f;
  if (p.logp) {
    y = p.tokens[n];
    if (y >= 0 && y < p.V) zy = to_f32(z[y]);
  }
  load_wait();
  Stats mine = no_stats();
  mine.m = thread_max<E>(data, s.pieces, lane, 32);
  thread_sums<E, true, kNoLabels, false>(data, s.pieces, lane, 32, c, mine, [](int) {});
  if (isnan(mine.e)) thread_sums<E, true, kNoLabels, true>(data, s.pieces, lane, 32, c, mine, [](int) {});
  if (je >= 0) join(mine, one_element(ze), c);
  const Stats r = warp_join(mine, c);
  const bool empty = r.m == -INFINITY && r.s == 0.0f;
  const float ref = r.m == -INFINITY ? 0.0f : r.m, log_s = empty ? 0.0f : logf(r.s);
  if (lane == 0) {
    if (p.entropy) p.entropy[n] = empty ? 0.0f : log_s - r.e / r.s * (1.0f / kLog2e);
    if (p.lse) p.lse[n] = empty ? -INFINITY : ref * inv_tau + log_s;
    if (p.logp) p.logp[n] = y < 0 ? 0.0f : y >= p.V ? NAN : (zy - ref) * inv_tau - log_s;
  }
  if (p.K == 0) return;
  unsigned long long* const list = reinterpret_cast<unsigned long long*>(data + slots);
  // a bound as in the kernel above, with the lanes' pieces as groups where there are 2 K of them, else the
  // elements themselves
  auto order = [](float v) {
    const int u = __float_as_int(v);
    return u ^ (u >> 31 & 0x7fffffff);
  };
  float best[kShortOwn];
  int lo = INT32_MAX, hi = INT32_MIN;
#pragma unroll
  for (int e = 0; e < kShortOwn; ++e) {
    best[e] = lane + 32 * e < s.pieces ? piece_max<E>(data[lane + 32 * e]) : -INFINITY;
    if (lane + 32 * e < s.pieces) lo = min(lo, order(best[e]));
  }
  hi = order(r.m);
  const bool by_piece = s.pieces >= 2 * p.K;
  lo = by_piece ? __reduce_min_sync(~0u, lo) : order(-INFINITY);
  int reach = by_piece ? s.pieces : p.V;
  const int enough = by_piece ? bound_reach(s.pieces, p.K) : max(p.K, min(p.K + 64, kShortList));
  auto value = [](int o) { return __int_as_float(o ^ (o >> 31 & 0x7fffffff)); };
  while (lo < hi && reach > enough) {
    const int mid = int((int64_t(lo) + hi + 1) >> 1);
    const float x = value(mid);
    int count = 0;
#pragma unroll
    for (int e = 0; e < kShortOwn; ++e) {
      if (32 * e >= s.pieces) break;
      if (by_piece) {
        count += best[e] >= x && lane + 32 * e < s.pieces;
      } else if (best[e] >= x && lane + 32 * e < s.pieces) {
        Vec<2> v[kPairs<E>];
        unpack<E>(data[lane + 32 * e], v);
#pragma unroll
        for (int k = 0; k < kPer<E>; ++k) count += v[k / 2].v[k % 2] >= x;
      }
    }
    if (!by_piece) count += je >= 0 && ze >= x;
    count = __reduce_add_sync(~0u, count);
    if (count >= p.K) {
      lo = mid;
      reach = count;
    } else {
      hi = mid - 1;
    }
  }
  const float bound = value(lo);
  // the elements that reach it
  auto each_hit = [&](auto f) {
    if (je >= 0 && ze >= bound) f(ze, je);
    for (int i = lane; i < s.pieces; i += 32) {
      const uint4 w = data[i];
      if (piece_max<E>(w) < bound) continue;
      Vec<2> v[kPairs<E>];
      unpack<E>(w, v);
#pragma unroll
      for (int k = 0; k < kPer<E>; ++k)
        if (v[k / 2].v[k % 2] >= bound) f(v[k / 2].v[k % 2], s.index(i) + k);
    }
  };
  int hits = 0;
  each_hit([&](float, int) { ++hits; });
  int at = hits;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int other = __shfl_up_sync(~0u, at, d);
    if (lane >= d) at += other;
  }
  int total = __shfl_sync(~0u, at, 31);
  at -= hits;
  if (isnan(r.s) || total > kShortList) {
    const bool finite = !isnan(r.s);
    exact_top<E>(z, p.V, p.K, finite ? value_order(bound) : 1u, finite ? value_order(r.m) : value_order(NAN), list, kShortList);
    total = p.K;
  } else {
    each_hit([&](float v, int j) { list[at++] = order_key(v, j); });
  }
  __syncwarp();
  auto write = [&](int k, unsigned long long key) {
    p.top_idx[n * p.K + k] = key_index(key);
    p.top_logp[n * p.K + k] = (key_value(key) - ref) * inv_tau - log_s;
  };
  if (total <= 32)
    write_sorted<1>(list, total, p.K, write);
  else if (total <= 128)
    write_sorted<4>(list, total, p.K, write);
  else
    write_sorted<8>(list, total, p.K, write);
}

// ---- gradient of log probability and entropy: one pass over a row's pieces, cut over blocks ----
//
// lse and entropy come from the forward call, so an element is read, transformed and written: HBM
// bound (2048 x 32000 fp32: 76 us, 6.2 TB/s of reads and writes under the profiler).
//
// p = exp(z / tau - lse) has the rounding of lse as its relative error: up to 2^-18 below kFarLse.  Rows
// beyond it (low temperatures, logits with a common offset, an lse past fp32) are taken by their first block
// alone, which finds their maximum and sum again and forms (z - m) / tau - log s, where nothing cancels
// (2048 x 32000 fp32, every row such: 125 us; one row of 131072 bf16: 28.5 against 6.8).

constexpr int kGradPieces = 4;   // of a thread
constexpr float kFarLse = 128.0f;

// log p = (z - ref) / tau - off
struct GradRow {
  float inv_tau, ref, off;
  float none;        // 0: a row without mass, where p = 0
  float dl, dh, H;   // dlogp, dentropy, entropy
  int y;
};

// The gradients of elements j and j + 1.  FAR: ref is not 0.
template <typename E, bool FAR>
__device__ __forceinline__ Vec<2> score_grad(const GradRow& r, Vec<2> v, int j) {
  if constexpr (FAR) v = v + splat<2>(-r.ref);
  const Vec<2> lp = fma<2>(v, splat<2>(r.inv_tau), splat<2>(-r.off)), x = lp * splat<2>(kLog2e);
  const Vec<2> e = Vec<2>{exp2_grad<E>(x.v[0]), exp2_grad<E>(x.v[1])} * splat<2>(-r.none);
  const Vec<2> bounded = {fmaxf(lp.v[0], -1000.0f), fmaxf(lp.v[1], -1000.0f)};
  Vec<2> g = e * fma<2>(splat<2>(r.dh), bounded, splat<2>(fmaf(r.dh, r.H, r.dl)));
#pragma unroll
  for (int m = 0; m < 2; ++m)
    if (j + m == r.y) g.v[m] += r.dl;
  return g * splat<2>(r.inv_tau);
}

template <typename E, bool FAR>
__device__ __forceinline__ void write_score_grad(const GradRow& r, const uint4& w, E* grad, int j, bool aligned) {
  Vec<2> v[kPairs<E>];
  unpack<E>(w, v);
#pragma unroll
  for (int k = 0; k < kPairs<E>; ++k) v[k] = score_grad<E, FAR>(r, v[k], j + 2 * k);
  const uint4 o = pack<E>(v);
  if (aligned) {
    *reinterpret_cast<uint4*>(grad + j) = o;
  } else {
    const E* e = reinterpret_cast<const E*>(&o);
#pragma unroll
    for (int k = 0; k < kPer<E>; ++k) grad[j + k] = e[k];
  }
}

// A whole row by one block.  grad may be the row itself: all have read it before the first store, and then
// each thread reads a piece before it writes there.
template <typename E>
__device__ __noinline__ void far_row_grad(const E* z, int V, E* grad, GradRow r) {
  __shared__ Stats all[kRowThreads / 32];
  const int tid = threadIdx.x;
  const Slice<E> s = slice_of(z, V, 0, 1);
  const bool aligned = reinterpret_cast<uintptr_t>(grad + s.index(0)) % 16 == 0;
  const float c = kLog2e * r.inv_tau;
  const int je = tid < s.edges() ? s.edge(tid) : -1;
  const float ze = je >= 0 ? to_f32(z[je]) : 0.0f;
  Stats mine = no_stats();
  mine.m = thread_max<E>(s.data(), s.pieces, tid, kRowThreads);
  thread_sums<E, false, kNoLabels, false>(s.data(), s.pieces, tid, kRowThreads, c, mine, [](int) {});
  if (je >= 0) join(mine, one_element(ze), c);
  mine = warp_join(mine, c);
  if (tid % 32 == 0) all[tid / 32] = mine;
  __syncthreads();
  const Stats row = collect_stats(all, 1, kRowThreads / 32, c);
  r.ref = row.m == -INFINITY ? 0.0f : row.m;
  r.off = row.s == 0.0f ? 0.0f : logf(row.s);
  r.none = row.s == 0.0f ? 0.0f : 1.0f;
  for (int i = tid; i < s.pieces; i += kRowThreads) write_score_grad<E, true>(r, s.data()[i], grad, s.index(i), aligned);
  if (je >= 0) grad[je] = from_f32<E>(score_grad<E, true>(r, splat<2>(ze), je).v[0]);
}

template <typename E>
__global__ void __launch_bounds__(kRowThreads, 8) token_logp_grad_kernel(const LogpGradArgs p, int blocks_per_row) {
  pdl_entry();
  const int64_t n = blockIdx.x / blocks_per_row;
  const int part = blockIdx.x % blocks_per_row;
  const E* z = static_cast<const E*>(p.logits) + n * p.ld;
  const Slice<E> s = slice_of(z, p.V, 0, 1);
  E* const grad = static_cast<E*>(p.grad) + n * p.grad_ld;
  const bool aligned = reinterpret_cast<uintptr_t>(grad + s.index(0)) % 16 == 0;
  const int first = part * kGradPieces * kRowThreads + threadIdx.x;
  uint4 w[kGradPieces];
#pragma unroll
  for (int i = 0; i < kGradPieces; ++i)
    if (first + i * kRowThreads < s.pieces) w[i] = s.data()[first + i * kRowThreads];
  const int je = part == 0 && int(threadIdx.x) < s.edges() ? s.edge(threadIdx.x) : -1;
  const float ze = je >= 0 ? to_f32(z[je]) : 0.0f;
  const float lse = p.lse[n];
  int y = -1;
  float dl = 0.0f;
  if (p.dlogp) {
    y = p.tokens[n];
    if (y >= 0) dl = y < p.V ? p.dlogp[n] : NAN;
  }
  const GradRow r = {1.0f / p.tau, 0.0f, lse, 1.0f, dl, p.dentropy ? p.dentropy[n] : 0.0f, p.dentropy ? p.entropy[n] : 0.0f, y};
  if (fabsf(lse) >= kFarLse) {   // (not NaN)
    if (part == 0) far_row_grad<E>(z, p.V, grad, r);
    return;
  }
#pragma unroll
  for (int i = 0; i < kGradPieces; ++i) {
    const int piece = first + i * kRowThreads;
    if (piece >= s.pieces) break;
    write_score_grad<E, false>(r, w[i], grad, s.index(piece), aligned);
  }
  if (je >= 0) grad[je] = from_f32<E>(score_grad<E, false>(r, splat<2>(ze), je).v[0]);
}

template <typename E, Hard HARD>
cudaError_t launch_distill_as(const DistillArgs& p, int dtype, int64_t N, const RowCut& c, cudaStream_t stream) {
  if (row_is_short(dtype, p.V)) return launch_short<distill_short_kernel<E, HARD>>(p, dtype, N, teacher_bytes(p.K), stream, row_slots(dtype, p.V));
  return launch_rows<distill_kernel<E, HARD>>(c, N, stream, p, N, c.cluster, c.slots);
}

template <typename E>
cudaError_t launch_distill(const DistillArgs& p, int dtype, int64_t N, cudaStream_t stream) {
  RowCut c = row_cut(dtype, N, p.V, 1);
  if (c.cluster == 0) return launch_pdl(distill_stream_kernel<E>, dim3(unsigned(N)), dim3(kThreads), 0, stream, p);
  c.smem += teacher_bytes(p.K);
  if (p.alpha == 0.0f) return launch_distill_as<E, kNoLabels>(p, dtype, N, c, stream);
  if (p.tau == 1.0f) return launch_distill_as<E, kTau1>(p, dtype, N, c, stream);
  if (p.tau == 2.0f) return launch_distill_as<E, kTau2>(p, dtype, N, c, stream);
  return launch_distill_as<E, kOwnExponential>(p, dtype, N, c, stream);
}

template <typename E>
cudaError_t launch_logp(const LogpArgs& p, int dtype, int64_t N, cudaStream_t stream) {
  if (row_is_short(dtype, p.V))
    return launch_short<token_logp_short_kernel<E>>(p, dtype, N, p.K > 0 ? kShortList * sizeof(unsigned long long) : 0, stream,
                                                    row_slots(dtype, p.V));
  RowCut c = row_cut(dtype, N, p.V, 2);
  if (c.cluster == 0) return launch_pdl(token_logp_stream_kernel<E>, dim3(unsigned(N)), dim3(kThreads), 0, stream, p);
  // the widest groups of which there are at least 2 K with elements (T C of one lane: at least K)
  const int T = c.threads - 64, busy = (c.slots < T ? c.slots : T) * c.cluster;
  int lanes = 32;
  while (lanes > 1 && busy < 2 * p.K * lanes) lanes /= 2;
  c.smem += top_bytes<E>(p.K, T / lanes * c.cluster + 1, T);
  return launch_rows<token_logp_kernel<E>>(c, N, stream, p, N, c.cluster, c.slots, lanes);
}

template <typename E>
cudaError_t launch_logp_grad(const LogpGradArgs& p, int64_t N, cudaStream_t stream) {
  const int64_t per_block = int64_t(kGradPieces) * kRowThreads * kPer<E>;
  const int64_t blocks = (p.V + per_block - 1) / per_block;
  return launch_pdl(token_logp_grad_kernel<E>, dim3(unsigned(N * blocks)), dim3(kRowThreads), 0, stream, p, int(blocks));
}

}  // namespace
}  // namespace lm
}  // namespace gem

using namespace gem;
using namespace gem::lm;

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
  // labels only: 0 times a term that may be infinite is not 0, so the kernels get no teacher
  const bool teacher = alpha < 1.0f;
  const DistillArgs p = {logits, grad, ld, grad_ld, int(V), teacher ? K : 0, top_idx, top_logits, teacher ? teacher_lse : nullptr,
                         labels, row_scale, temperature, alpha, loss};
  return launch_status(BY_TYPE(launch_distill, p, dtype, N, static_cast<cudaStream_t>(stream)));
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
  return launch_status(BY_TYPE(launch_logp, p, dtype, N, static_cast<cudaStream_t>(stream)));
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
  return launch_status(BY_TYPE(launch_logp_grad, p, N, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
