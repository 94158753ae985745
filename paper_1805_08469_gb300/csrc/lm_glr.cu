// Gated linear recurrence: the calls of include/gem_lm.h (argument checks and dispatch).
#include "lm_glr.h"

namespace gem {
namespace lm {
namespace glr {
namespace {

bool sizes_ok(int dtype, int form, int64_t B, int64_t T, int64_t D) {
  if (!dtype_ok(dtype) || (form != GEM_GLR_LERP && form != GEM_GLR_ADD)) return false;
  if (!extent_ok(B) || !extent_ok(T) || !extent_ok(D)) return false;
  return B == 0 || (D + 31) / 32 <= (int64_t(1) << 27) / B;   // a block at least for 32 channels of a sequence
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
  return launch_status(BY_TYPE(launch_forward, p, form, static_cast<cudaStream_t>(stream)));
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
  return launch_status(BY_TYPE(launch_backward, p, form, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
