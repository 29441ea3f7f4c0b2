// The kernels of norm_planes.hpp for bfloat16.
#include "norm_planes.hpp"

namespace oaa {

template hipError_t launch_planes_forward<bf16>(const GroupNormParams&, const NormCut&, hipStream_t);
template hipError_t launch_planes_backward<bf16>(const GroupNormParams&, const NormCut&, const NormSums&, hipStream_t);

}  // namespace oaa
