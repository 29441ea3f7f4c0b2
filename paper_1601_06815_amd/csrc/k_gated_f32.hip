// The gated unit's products and passes, float.
#include "gated_few.hpp"
#include "gated_passes.hpp"
#include "product.hpp"

namespace oaa {
template hipError_t launch_product<float>(const ProductParams&, ProductKind, hipStream_t);
template hipError_t launch_few<float>(const FewParams&, hipStream_t);
template hipError_t launch_slope<float>(const SlopeParams&, hipStream_t);
template hipError_t launch_bias_join<float>(const float*, long, int, void*, void*, hipStream_t);
template hipError_t launch_join<float>(const JoinParams&, hipStream_t);
template hipError_t launch_pack<float>(const PackParams&, hipStream_t);
template hipError_t launch_zero<float>(void*, long, hipStream_t);
}  // namespace oaa
