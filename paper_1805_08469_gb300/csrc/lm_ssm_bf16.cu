// Selective state space scan: the kernels for bf16.
#include "lm_ssm_backward.h"
#include "lm_ssm_forward.h"

namespace gem {
namespace lm {
namespace ssm {

template cudaError_t launch_forward<__nv_bfloat16>(SsmArgs, cudaStream_t);
template cudaError_t launch_backward<__nv_bfloat16>(SsmArgs, cudaStream_t);

}  // namespace ssm
}  // namespace lm
}  // namespace gem
