// Losses and scores over rows of logits (include/gem_lm.h): distillation from a teacher's top
// logits, log probabilities of tokens with entropy and top alternatives, and their gradients.
#include "lm_internal.h"

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
__global__ void __launch_bounds__(kThreads) distill_kernel(const DistillArgs p) {
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
__global__ void __launch_bounds__(kThreads) token_logp_kernel(const LogpArgs p) {
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

template <typename E>
__global__ void __launch_bounds__(kThreads) token_logp_grad_kernel(const LogpGradArgs p) {
  pdl_entry();
  const int64_t n = blockIdx.x;
  const E* z = static_cast<const E*>(p.logits) + n * p.ld;
  E* grad = static_cast<E*>(p.grad) + n * p.grad_ld;
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
  for (int j = threadIdx.x; j < p.V; j += blockDim.x) {
    const float lp = lse == -INFINITY ? -INFINITY : to_f32(z[j]) * inv_tau - lse;
    const float e = expf(lp);
    float g = -e * (dl + dh * (fmaxf(lp, -1000.0f) + H));
    if (j == y) g += dl;
    grad[j] = from_f32<E>(g * inv_tau);
  }
}

bool rows_ok(int dtype, int64_t N, int64_t V, const void* z, int64_t ld) {
  if (!dtype_ok(dtype) || !extent_ok(N) || V < 1 || !extent_ok(V)) return false;
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

// Calls KERNEL<E> for the element type.
#define LAUNCH_BY_TYPE(KERNEL, args)                                                                        \
  launch_status(dtype == GEM_F32    ? launch_pdl(KERNEL<float>, grid, block, 0, st, args)                   \
                : dtype == GEM_BF16 ? launch_pdl(KERNEL<__nv_bfloat16>, grid, block, 0, st, args) \
                                    : launch_pdl(KERNEL<__half>, grid, block, 0, st, args))

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
  const dim3 grid{unsigned(N)}, block{kThreads};
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  return LAUNCH_BY_TYPE(distill_kernel, p);
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
  const dim3 grid{unsigned(N)}, block{kThreads};
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  return LAUNCH_BY_TYPE(token_logp_kernel, p);
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
  const dim3 grid{unsigned(N)}, block{kThreads};
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  return LAUNCH_BY_TYPE(token_logp_grad_kernel, p);
}

}  // extern "C"
