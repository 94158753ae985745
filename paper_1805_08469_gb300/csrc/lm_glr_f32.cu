// Gated linear recurrence: the kernels for fp32.
#include "lm_glr_backward.h"
#include "lm_glr_forward.h"

namespace gem {
namespace lm {
namespace glr {

template cudaError_t launch_forward<float>(const GlrArgs&, int, cudaStream_t);
template cudaError_t launch_backward<float>(const GlrArgs&, int, cudaStream_t);

}  // namespace glr
}  // namespace lm
}  // namespace gem
