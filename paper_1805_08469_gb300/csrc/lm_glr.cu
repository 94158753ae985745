// Gated linear recurrence (include/gem_lm.h): h_t = a_t h_{t-1} + u_t with a = sigmoid(f) and
// u = (1 - a) x or x, and its backward pass.
#include "lm_internal.h"

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

// sigmoid(f) and 1 - sigmoid(f) = sigmoid(-f), each to its own relative precision.
__device__ __forceinline__ void gate(float f, float& a, float& b) {
  const float e = expf(-fabsf(f));
  const float r = 1.0f / (1.0f + e);
  a = f < 0.0f ? e * r : r;
  b = f < 0.0f ? r : e * r;
}

__device__ __forceinline__ int64_t steps_of(const GlrArgs& p, int64_t b) {
  if (!p.lengths) return p.T;
  const int64_t n = p.lengths[b];
  return n < 0 ? 0 : n > p.T ? p.T : n;
}

// One thread per channel, one step after the other.
template <typename E, bool LERP>
__global__ void glr_forward_kernel(const GlrArgs p) {
  pdl_entry();
  const int64_t i = int64_t(blockIdx.x) * blockDim.x + threadIdx.x;
  if (i >= p.B * p.D) return;
  const int64_t b = i / p.D, d = i % p.D;
  const int64_t n = steps_of(p, b);
  float h = p.h0 ? p.h0[i] : 0.0f;
  for (int64_t t = 0; t < p.T; ++t) {
    if (p.saved_out && t % kChunk == 0)
      p.saved_out[(b * ((p.T + kChunk - 1) / kChunk) + t / kChunk) * p.D + d] = h;
    float shown = 0.0f;
    if (t < n) {
      float a, c;
      gate(to_f32(*at<const E>(p.f, b, t, d)), a, c);
      const float x = to_f32(*at<const E>(p.x, b, t, d));
      const float u = LERP ? c * x : x;
      h = p.reset && p.reset[b * p.T + t] ? u : fmaf(a, h, u);
      shown = h;
    }
    *at<E>(p.h, b, t, d) = from_f32<E>(shown);
  }
  if (p.h_last) p.h_last[i] = h;
}

template <typename E, bool LERP>
__global__ void glr_backward_kernel(const GlrArgs p) {
  pdl_entry();
  const int64_t i = int64_t(blockIdx.x) * blockDim.x + threadIdx.x;
  if (i >= p.B * p.D) return;
  const int64_t b = i / p.D, d = i % p.D;
  const int64_t n = steps_of(p, b);
  const int64_t chunks = (p.T + kChunk - 1) / kChunk;
  float g = p.dh_last ? p.dh_last[i] : 0.0f;   // a_{t+1} g_{t+1}
  for (int64_t c = chunks - 1; c >= 0; --c) {
    float before[kChunk];
    float h = p.saved_in[(b * chunks + c) * p.D + d];
    for (int k = 0; k < kChunk; ++k) {
      const int64_t t = c * kChunk + k;
      if (t >= n) break;
      const bool fresh = p.reset && p.reset[b * p.T + t];
      float a, m;
      gate(to_f32(*at<const E>(p.f, b, t, d)), a, m);
      const float x = to_f32(*at<const E>(p.x, b, t, d));
      const float u = LERP ? m * x : x;
      before[k] = fresh ? 0.0f : h;
      h = fresh ? u : fmaf(a, h, u);
    }
    for (int k = kChunk - 1; k >= 0; --k) {
      const int64_t t = c * kChunk + k;
      if (t >= p.T) continue;
      float dx = 0.0f, df = 0.0f;
      if (t < n) {
        float a, m;
        gate(to_f32(*at<const E>(p.f, b, t, d)), a, m);
        g += to_f32(*at<const E>(p.dh, b, t, d));
        const float x = to_f32(*at<const E>(p.x, b, t, d));
        dx = LERP ? m * g : g;
        df = g * (LERP ? before[k] - x : before[k]) * (a * m);
        g = p.reset && p.reset[b * p.T + t] ? 0.0f : a * g;
      }
      *at<E>(p.dx, b, t, d) = from_f32<E>(dx);
      *at<E>(p.df, b, t, d) = from_f32<E>(df);
    }
  }
  if (p.dh0) p.dh0[i] = g;
}

template <typename E>
cudaError_t launch(const GlrArgs& p, int form, bool backward, cudaStream_t stream) {
  const int64_t blocks = (p.B * p.D + 127) / 128;
  auto* k = backward ? (form == GEM_GLR_LERP ? glr_backward_kernel<E, true> : glr_backward_kernel<E, false>)
                     : (form == GEM_GLR_LERP ? glr_forward_kernel<E, true> : glr_forward_kernel<E, false>);
  return launch_pdl(k, dim3(unsigned(blocks)), dim3(128), 0, stream, p);
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
  return B == 0 || D <= (int64_t(1) << 36) / B;   // B D channels: a grid of blocks of at least 32
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
