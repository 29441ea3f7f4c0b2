// The kernels of norm_last.hpp for bfloat16.
#include "norm_last.hpp"

namespace oaa {

template hipError_t launch_last_forward<bf16>(const GroupNormParams&, const NormCut&, hipStream_t);
template hipError_t launch_last_backward<bf16>(const GroupNormParams&, const NormCut&, const NormSums&, hipStream_t);

}  // namespace oaa
