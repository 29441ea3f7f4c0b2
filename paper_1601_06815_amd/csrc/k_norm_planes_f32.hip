// The kernels of norm_planes.hpp for float32.
#include "norm_planes.hpp"

namespace oaa {

template hipError_t launch_planes_forward<float>(const GroupNormParams&, const NormCut&, hipStream_t);
template hipError_t launch_planes_backward<float>(const GroupNormParams&, const NormCut&, const NormSums&, hipStream_t);

}  // namespace oaa
