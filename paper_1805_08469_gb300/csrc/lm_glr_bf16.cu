// Gated linear recurrence: the kernels for bf16.
#include "lm_glr_backward.h"
#include "lm_glr_forward.h"

namespace gem {
namespace lm {
namespace glr {

template cudaError_t launch_forward<__nv_bfloat16>(const GlrArgs&, int, cudaStream_t);
template cudaError_t launch_backward<__nv_bfloat16>(const GlrArgs&, int, cudaStream_t);

}  // namespace glr
}  // namespace lm
}  // namespace gem
