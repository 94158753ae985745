// Selective state space scan: the kernels for fp16.
#include "lm_ssm_backward.h"
#include "lm_ssm_forward.h"

namespace gem {
namespace lm {
namespace ssm {

template cudaError_t launch_forward<__half>(SsmArgs, cudaStream_t);
template cudaError_t launch_backward<__half>(SsmArgs, cudaStream_t);

}  // namespace ssm
}  // namespace lm
}  // namespace gem
