// The clipped policy loss of sampled tokens with its gradient (include/gem_lm.h), over rows of logits.
#include "lm_rows.h"

namespace gem {
namespace lm {
namespace {

struct PolicyArgs {
  const void* logits;
  void* grad;
  int64_t ld, grad_ld;
  int V;
  const int32_t* tokens;
  const float *old_logp, *advantage, *ref_logp, *row_scale;
  float tau, low, high, kl, bonus;
  float *loss, *logp, *entropy;
};

// A row's loss, and what its gradient needs: the element's is
//   e (k_one + k_log x), e = exp2(x), x = (z - ref) log2(e) / tau,
// and at the token k_token more.
struct PolicyRow {
  float ref, k_one, k_log, k_token;
  float loss, logp, entropy;
};

// From the statistics r of the row (e only where the bonus or the entropy is asked for), its token y and that one's
// logit zy; w is its scale.
__device__ __forceinline__ PolicyRow policy_row(const PolicyArgs& p, int64_t n, const Stats& r, int y, float zy, float w) {
  PolicyRow k;
  const float inv_tau = 1.0f / p.tau;
  k.ref = r.m == -INFINITY ? 0.0f : r.m;
  const float log_s = logf(r.s);   // (-inf for a row without mass, whose loss is NaN)
  k.entropy = log_s - r.e / r.s * (1.0f / kLog2e);
  k.logp = y < p.V ? (zy - k.ref) * inv_tau - log_s : NAN;
  const float A = p.advantage[n], ratio = expf(k.logp - p.old_logp[n]);
  const float plain = -ratio * A, clipped = -fminf(fmaxf(ratio, 1.0f - p.low), 1.0f + p.high) * A;
  // (written so that a NaN stays one)
  k.loss = plain >= clipped ? plain : isnan(plain) ? plain : clipped;
  float d = plain >= clipped ? plain : isnan(plain) ? plain : 0.0f;
  if (p.kl != 0.0f) {
    const float far = p.ref_logp[n] - k.logp, more = expm1f(far);
    k.loss += p.kl * (more - far);
    d -= p.kl * more;
  }
  const float scale = w * inv_tau / r.s;
  k.k_one = -scale * d;
  k.k_log = 0.0f;
  if (p.bonus != 0.0f) {
    k.loss -= p.bonus * k.entropy;
    k.k_one += scale * p.bonus * (k.entropy - log_s);
    k.k_log = scale * p.bonus * (1.0f / kLog2e);
  }
  k.k_token = w * inv_tau * d;
  return k;
}

// Whether the row is read at all.
__device__ __forceinline__ bool policy_live(const PolicyArgs& p, int y, float w) { return y >= 0 && w != 0.0f; }

__device__ __forceinline__ void write_policy(const PolicyArgs& p, int64_t n, const PolicyRow& k) {
  p.loss[n] = k.loss;
  if (p.logp) p.logp[n] = k.logp;
  if (p.entropy) p.entropy[n] = k.entropy;
}

// A block streams the row: rows longer than a cluster's shared memory.
template <typename E>
__global__ void __launch_bounds__(kThreads) policy_stream_kernel(const PolicyArgs p) {
  pdl_entry();
  __shared__ float buf[kThreads / 32];
  const int64_t n = blockIdx.x;
  const E* z = static_cast<const E*>(p.logits) + n * p.ld;
  E* const grad = p.grad ? static_cast<E*>(p.grad) + n * p.grad_ld : nullptr;
  const int tid = threadIdx.x, y = p.tokens[n];
  const float w = p.row_scale ? p.row_scale[n] : 1.0f, inv_tau = 1.0f / p.tau;
  if (!policy_live(p, y, w)) {
    if (grad)
      for (int j = tid; j < p.V; j += kThreads) grad[j] = from_f32<E>(0.0f);
    if (tid == 0) write_policy(p, n, PolicyRow{});
    return;
  }
  Stats r = no_stats();
  row_stats(z, p.V, inv_tau, buf, r.m, r.s);
  const float ref = r.m == -INFINITY ? 0.0f : r.m;
  const float zy = y < p.V ? to_f32(z[y]) : 0.0f;
  if (p.bonus != 0.0f || p.entropy) {
    float e = 0.0f;
    for (int j = tid; j < p.V; j += kThreads) {
      const float d = (to_f32(z[j]) - ref) * inv_tau;
      e += expf(d) * fmaxf(d, -1000.0f);
    }
    r.e = block_reduce(e, buf, Sum()) * kLog2e;
  }
  const PolicyRow k = policy_row(p, n, r, y, zy, w);
  if (tid == 0) write_policy(p, n, k);
  if (!grad) return;
  __syncthreads();   // (grad may be logits: all have read the token's)
  for (int j = tid; j < p.V; j += kThreads) {
    const float d = (to_f32(z[j]) - ref) * inv_tau;
    const float g = expf(d) * (k.k_one + k.k_log * (fmaxf(d, -1000.0f) * kLog2e));
    grad[j] = from_f32<E>(j == y ? g + k.k_token : g);
  }
}

template <typename E>
cudaError_t launch_policy(const PolicyArgs& p, int64_t N, cudaStream_t stream) {
  return launch_pdl(policy_stream_kernel<E>, dim3(unsigned(N)), dim3(kThreads), 0, stream, p);
}

}  // namespace
}  // namespace lm
}  // namespace gem

using namespace gem;
using namespace gem::lm;

extern "C" {

int gem_policy(int dtype, int64_t N, int64_t V, const void* logits, int64_t ld,
               const int32_t* tokens, const float* old_logp, const float* advantage,
               const float* ref_logp, const float* row_scale, float temperature, float clip_low,
               float clip_high, float kl, float bonus, float* loss, float* logp, float* entropy,
               void* grad, int64_t grad_ld, void* stream) {
  if (!rows_ok(dtype, N, V, logits, ld) || !temperature_ok(temperature)) return GEM_EINVAL;
  if (!(clip_low >= 0.0f && clip_low <= 1.0f) || !(clip_high >= 0.0f && clip_high < INFINITY)) return GEM_EINVAL;
  if (!(kl >= 0.0f && kl < INFINITY) || !(fabsf(bonus) < INFINITY)) return GEM_EINVAL;
  if (N == 0) return GEM_OK;
  if (!array_ok(tokens) || !array_ok(old_logp) || !array_ok(advantage) || !array_ok(loss)) return GEM_EINVAL;
  if ((kl > 0.0f && !array_ok(ref_logp)) || !optional_ok(ref_logp) || !optional_ok(row_scale)) return GEM_EINVAL;
  if (!optional_ok(logp) || !optional_ok(entropy)) return GEM_EINVAL;
  if (grad && (!grad_ok(dtype, V, grad, grad_ld) || (grad == logits && grad_ld != ld))) return GEM_EINVAL;
  const PolicyArgs p = {logits, grad, ld, grad_ld, int(V), tokens, old_logp, advantage, ref_logp, row_scale,
                        temperature, clip_low, clip_high, kl, bonus, loss, logp, entropy};
  return launch_status(BY_TYPE(launch_policy, p, N, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
