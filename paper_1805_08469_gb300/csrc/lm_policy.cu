// The clipped policy loss of sampled tokens with its gradient (include/gem_lm.h), over rows of logits.
//
// A row's statistics (maximum, sum and, for entropy and bonus, sum of p log p) give everything that its gradient needs beside
// the elements, so a row on chip is read from memory once and its gradient written once.  Clusters stay and take row after row:
// the gradient pass refills each slot with the next row's piece.  One cluster barrier a row.  4096 x 131072 bf16, all
// terms: 352 us (5.8 TB/s; a tenth of the rows is masked and not read), 16 instructions and 2 exponentials an element in 0.67 of the
// issue slots; one block a row that streams it took 3.1 ms.
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

// What a row is given beside its logits.
struct PolicyInput {
  int y;
  float w, old, A, far;
  bool live;   // it is read at all
};
__device__ __forceinline__ PolicyInput policy_input(const PolicyArgs& p, int64_t n, int64_t N) {
  PolicyInput r = {-1, 0.0f, 0.0f, 0.0f, 0.0f, false};
  if (n >= N) return r;
  r.y = p.tokens[n];
  r.w = p.row_scale ? p.row_scale[n] : 1.0f;
  r.old = p.old_logp[n];
  r.A = p.advantage[n];
  if (p.kl != 0.0f) r.far = p.ref_logp[n];
  r.live = r.y >= 0 && r.w != 0.0f;
  return r;
}

// A row's loss, and what its gradient needs: the element's is
//   e (k_one + k_log x), e = exp2(x), x = (z - ref) log2(e) / tau,
// and at the token k_token more.
struct PolicyRow {
  float ref, k_one, k_log, k_token;
  float loss, logp, entropy;
};

// From the statistics r of the row (e only where the bonus or the entropy is asked for), its token y and that one's
// logit zy; w is its scale.
__device__ __forceinline__ PolicyRow policy_row(const PolicyArgs& p, const PolicyInput& in, const Stats& r, float zy) {
  PolicyRow k;
  const float inv_tau = 1.0f / p.tau;
  k.ref = r.m == -INFINITY ? 0.0f : r.m;
  const float log_s = logf(r.s);   // (-inf for a row without mass, whose loss is NaN)
  k.entropy = log_s - r.e / r.s * (1.0f / kLog2e);
  k.logp = in.y < p.V ? (zy - k.ref) * inv_tau - log_s : NAN;
  const float ratio = expf(k.logp - in.old);
  const float plain = -ratio * in.A, clipped = -fminf(fmaxf(ratio, 1.0f - p.low), 1.0f + p.high) * in.A;
  // (written so that a NaN stays one)
  k.loss = plain >= clipped ? plain : isnan(plain) ? plain : clipped;
  float d = plain >= clipped ? plain : isnan(plain) ? plain : 0.0f;
  if (p.kl != 0.0f) {
    const float far = in.far - k.logp, more = expm1f(far);
    k.loss += p.kl * (more - far);
    d -= p.kl * more;
  }
  const float scale = in.w * inv_tau / r.s;
  k.k_one = -scale * d;
  k.k_log = 0.0f;
  if (p.bonus != 0.0f) {
    k.loss -= p.bonus * k.entropy;
    k.k_one += scale * p.bonus * (k.entropy - log_s);
    k.k_log = scale * p.bonus * (1.0f / kLog2e);
  }
  k.k_token = in.w * inv_tau * d;
  return k;
}

__device__ __forceinline__ void write_policy(const PolicyArgs& p, int64_t n, const PolicyRow& k) {
  p.loss[n] = k.loss;
  if (p.logp) p.logp[n] = k.logp;
  if (p.entropy) p.entropy[n] = k.entropy;
}

// The gradients of two elements but for the token's term.  LOG: with the bonus' term; FAR: where e is 0, x may be -inf or k_log x leave
// fp32, and e x is 0 all the same.  (Always taken it costs 4% at 4096 x 131072 bf16.)
template <typename E, bool LOG, bool FAR>
__device__ __forceinline__ Vec<2> policy_grad(Vec<2> v, const PolicyRow& k, float c) {
  Vec<2> x = (v + splat<2>(-k.ref)) * splat<2>(c);
  const Vec<2> e = {exp2_grad<E>(x.v[0]), exp2_grad<E>(x.v[1])};
  if constexpr (!LOG) return e * splat<2>(k.k_one);
  if constexpr (!FAR) return e * fma<2>(splat<2>(k.k_log), x, splat<2>(k.k_one));
  x = {fmaxf(x.v[0], -1000.0f), fmaxf(x.v[1], -1000.0f)};
  return fma<2>(splat<2>(k.k_log), e * x, e * splat<2>(k.k_one));
}

// Whether k_one + k_log x stays in fp32 for any finite x.
__device__ __forceinline__ bool factors_stay(const PolicyRow& k) { return fabsf(k.k_log) <= 0.25f && fabsf(k.k_one) <= 1e38f; }

// Writes the gradients of a piece to out, at any alignment; `token`: the token's element of it, or -1.
template <typename E, bool LOG, bool FAR>
__device__ __forceinline__ void write_policy_piece(const uint4& w, E* out, bool aligned, const PolicyRow& k, float c, int token) {
  Vec<2> v[kPairs<E>];
  unpack<E>(w, v);
#pragma unroll
  for (int m = 0; m < kPairs<E>; ++m) v[m] = policy_grad<E, LOG, FAR>(v[m], k, c);
  if (token >= 0) {
#pragma unroll
    for (int m = 0; m < kPer<E>; ++m)
      if (m == token) v[m / 2].v[m % 2] += k.k_token;
  }
  const uint4 g = pack<E>(v);
  if (aligned) {
    *reinterpret_cast<uint4*>(out) = g;
  } else {
    const E* e = reinterpret_cast<const E*>(&g);
#pragma unroll
    for (int m = 0; m < kPer<E>; ++m) out[m] = e[m];
  }
}
template <typename E>
__device__ __forceinline__ void write_zero_piece(E* out, bool aligned) {
  if (aligned) {
    *reinterpret_cast<uint4*>(out) = make_uint4(0, 0, 0, 0);
  } else {
#pragma unroll
    for (int m = 0; m < kPer<E>; ++m) out[m] = from_f32<E>(0.0f);
  }
}

// A thread's statistics of its pieces; far: the logarithm of some element's p is not finite (it counts as 0 times it).
template <typename E, bool LOG>
__device__ __forceinline__ Stats policy_stats(const uint4* data, int pieces, int t, int T, float c, bool& far) {
  Stats mine = no_stats();
  mine.m = thread_max<E>(data, pieces, t, T);
  thread_sums<E, LOG, kNoLabels, false>(data, pieces, t, T, c, mine, [](int) {});
  far = LOG && isnan(mine.e);
  if (far) thread_sums<E, LOG, kNoLabels, true>(data, pieces, t, T, c, mine, [](int) {});
  return mine;
}

template <typename E, bool LOG>
__global__ void __launch_bounds__(kRowThreads, 3) policy_kernel(const PolicyArgs p, int64_t N, int C) {
  extern __shared__ uint4 data[];
  __shared__ Stats all[2][kRowCluster * kRowParts];
  pdl_entry();
  const int rank = blockIdx.x % C, tid = threadIdx.x, T = kRowThreads, parts = kRowThreads / 32;
  const int64_t step = gridDim.x / C;
  const float c = kLog2e * (1.0f / p.tau);
  const E* const logits = static_cast<const E*>(p.logits);
  E* const grads = static_cast<E*>(p.grad);
  int64_t n = blockIdx.x / C;
  PolicyInput in = policy_input(p, n, N);
  cluster_started();
  Slice<E> s = slice_of(logits + n * p.ld, p.V, rank, C);
  if (in.live)
    for (int i = tid; i < s.pieces; i += T) load_piece(data + i, s.data() + i);
  load_commit();
  cluster_wait();
  for (int b = 0; n < N; n += step, b ^= 1) {
    // the next row, whose pieces follow this one's
    const PolicyInput next_in = policy_input(p, n + step, N);
    const Slice<E> next = slice_of(logits + (n + step) * p.ld, p.V, rank, C);
    const int next_pieces = next_in.live ? next.pieces : 0;
    // the first block's first warp has the elements before and after the whole pieces
    const int je = rank == 0 && tid < s.edges() ? s.edge(tid) : -1;
    float ze = 0.0f, zy = 0.0f;
    if (in.live) {
      if (in.y < p.V) zy = to_f32(s.row[in.y]);
      if (je >= 0) ze = to_f32(s.row[je]);
    }
    load_wait();
    bool far = false;   // some of the thread's elements are too far below its largest, or that one below the row's
    Stats mine = no_stats();
    if (in.live) {
      mine = policy_stats<E, LOG>(data, s.pieces, tid, T, c, far);
      if (je >= 0) join(mine, one_element(ze), c);
    }
    publish_stats(mine, all[b], rank, C, parts, c);
    cluster_arrive();
    cluster_wait();
    PolicyRow k = {};
    if (in.live) k = policy_row(p, in, collect_stats(all[b], C, parts, c), zy);
    far |= (mine.m - k.ref) * c < -1000.0f || !factors_stay(k);
    if (rank == 0 && tid == 0) write_policy(p, n, k);
    const int most = max(s.pieces, next_pieces);
    if (!grads) {
      for (int i = tid; i < next_pieces; i += T) load_piece(data + i, next.data() + i);
    } else {
      E* const row = grads + n * p.grad_ld;
      E* const out = row + s.index(0);
      const bool aligned = reinterpret_cast<uintptr_t>(out) % 16 == 0;
      const int at = in.y - s.index(0), token_piece = in.y < p.V && at >= 0 ? at / kPer<E> : -1, token = at % kPer<E>;
      auto write = [&](auto live, auto is_far) {
#pragma unroll 2
        for (int i = tid; i < most; i += T) {
          if (i < s.pieces) {
            if constexpr (decltype(live)::value)
              write_policy_piece<E, LOG, decltype(is_far)::value>(data[i], out + int64_t(i) * kPer<E>, aligned, k, c, i == token_piece ? token : -1);
            else
              write_zero_piece(out + int64_t(i) * kPer<E>, aligned);
          }
          if (i < next_pieces) load_piece(data + i, next.data() + i);
        }
      };
      if (!in.live)
        write(std::false_type(), std::false_type());
      else if (LOG && far)
        write(std::true_type(), std::true_type());
      else
        write(std::true_type(), std::false_type());
      if (je >= 0) {
        const float g = in.live ? policy_grad<E, LOG, true>(splat<2>(ze), k, c).v[0] + (je == in.y ? k.k_token : 0.0f) : 0.0f;
        row[je] = from_f32<E>(g);
      }
    }
    load_commit();
    s = next;
    in = next_in;
  }
  cluster_arrive();
  cluster_wait();
}

// Short rows: a warp for each.
template <typename E, bool LOG>
__global__ void __launch_bounds__(kShortWarps * 32, 8) policy_short_kernel(const PolicyArgs p, int64_t N, unsigned warp_bytes) {
  extern __shared__ uint4 shared[];
  pdl_entry();
  const int64_t n = int64_t(blockIdx.x) * kShortWarps + threadIdx.x / 32;
  if (n >= N) return;
  const int lane = threadIdx.x % 32;
  uint4* const data = warp_part<uint4>(shared, warp_bytes);
  const Slice<E> s = slice_of(static_cast<const E*>(p.logits) + n * p.ld, p.V, 0, 1);
  const PolicyInput in = policy_input(p, n, N);
  E* const grad = p.grad ? static_cast<E*>(p.grad) + n * p.grad_ld : nullptr;
  const float c = kLog2e * (1.0f / p.tau);
  const int je = lane < s.edges() ? s.edge(lane) : -1;
  PolicyRow k = {};
  float ze = 0.0f;
  if (in.live) {
    load_row(s, data);
    const float zy = in.y < p.V ? to_f32(s.row[in.y]) : 0.0f;
    if (je >= 0) ze = to_f32(s.row[je]);
    load_wait();
    bool far;
    Stats mine = policy_stats<E, LOG>(data, s.pieces, lane, 32, c, far);
    if (je >= 0) join(mine, one_element(ze), c);
    k = policy_row(p, in, warp_join(mine, c), zy);
  }
  if (lane == 0) write_policy(p, n, k);
  if (!grad) return;
  E* const out = grad + s.index(0);
  const bool aligned = reinterpret_cast<uintptr_t>(out) % 16 == 0;
  const int at = in.y - s.index(0), token_piece = in.y < p.V && at >= 0 ? at / kPer<E> : -1, token = at % kPer<E>;
  for (int i = lane; i < s.pieces; i += 32) {
    if (in.live)
      write_policy_piece<E, LOG, true>(data[i], out + i * kPer<E>, aligned, k, c, i == token_piece ? token : -1);
    else
      write_zero_piece(out + i * kPer<E>, aligned);
  }
  if (je >= 0) {
    const float g = in.live ? policy_grad<E, LOG, true>(splat<2>(ze), k, c).v[0] + (je == in.y ? k.k_token : 0.0f) : 0.0f;
    grad[je] = from_f32<E>(g);
  }
}

// A block streams the row: rows longer than a cluster's shared memory.
template <typename E>
__global__ void __launch_bounds__(kThreads) policy_stream_kernel(const PolicyArgs p, int64_t N) {
  pdl_entry();
  __shared__ float buf[kThreads / 32];
  const int64_t n = blockIdx.x;
  const E* z = static_cast<const E*>(p.logits) + n * p.ld;
  E* const grad = p.grad ? static_cast<E*>(p.grad) + n * p.grad_ld : nullptr;
  const int tid = threadIdx.x;
  const PolicyInput in = policy_input(p, n, N);
  if (!in.live) {
    if (grad)
      for (int j = tid; j < p.V; j += kThreads) grad[j] = from_f32<E>(0.0f);
    if (tid == 0) write_policy(p, n, PolicyRow{});
    return;
  }
  const float inv_tau = 1.0f / p.tau;
  Stats r = no_stats();
  row_stats(z, p.V, inv_tau, buf, r.m, r.s);
  const float ref = r.m == -INFINITY ? 0.0f : r.m;
  const float zy = in.y < p.V ? to_f32(z[in.y]) : 0.0f;
  if (p.bonus != 0.0f || p.entropy) {
    float e = 0.0f;
    for (int j = tid; j < p.V; j += kThreads) {
      const float d = (to_f32(z[j]) - ref) * inv_tau;
      e += expf(d) * fmaxf(d, -1000.0f);
    }
    r.e = block_reduce(e, buf, Sum()) * kLog2e;
  }
  const PolicyRow k = policy_row(p, in, r, zy);
  if (tid == 0) write_policy(p, n, k);
  if (!grad) return;
  __syncthreads();   // (grad may be logits: all have read the token's)
  for (int j = tid; j < p.V; j += kThreads) {
    const float d = (to_f32(z[j]) - ref) * inv_tau;
    const float e = expf(d);
    const float g = fmaf(k.k_log, e * (fmaxf(d, -1000.0f) * kLog2e), e * k.k_one);
    grad[j] = from_f32<E>(j == in.y ? g + k.k_token : g);
  }
}

template <typename E, bool LOG>
cudaError_t launch_policy_as(const PolicyArgs& p, int dtype, int64_t N, cudaStream_t stream) {
  if (row_is_short(dtype, p.V)) return launch_short<policy_short_kernel<E, LOG>>(p, dtype, N, 0, stream);
  const RowCut c = row_cut(dtype, N, p.V, 0);
  if (c.cluster == 0) return launch_pdl(policy_stream_kernel<E>, dim3(unsigned(N)), dim3(kThreads), 0, stream, p, N);
  return launch_rows<policy_kernel<E, LOG>>(c, N, stream, p, N, c.cluster);
}
// (the entropy's sum is taken where either the bonus or the entropy itself is asked for)
template <typename E>
cudaError_t launch_policy(const PolicyArgs& p, int dtype, int64_t N, cudaStream_t stream) {
  return p.bonus != 0.0f || p.entropy ? launch_policy_as<E, true>(p, dtype, N, stream) : launch_policy_as<E, false>(p, dtype, N, stream);
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
  return launch_status(BY_TYPE(launch_policy, p, dtype, N, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
