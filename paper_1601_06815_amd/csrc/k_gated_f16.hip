// The gated unit's products and passes, f16.
#include "gated_few.hpp"
#include "gated_passes.hpp"
#include "product.hpp"

namespace oaa {
template hipError_t launch_product<f16>(const ProductParams&, ProductKind, hipStream_t);
template hipError_t launch_few<f16>(const FewParams&, hipStream_t);
template hipError_t launch_slope<f16>(const SlopeParams&, hipStream_t);
template hipError_t launch_bias_join<f16>(const float*, long, int, void*, void*, hipStream_t);
template hipError_t launch_join<f16>(const JoinParams&, hipStream_t);
template hipError_t launch_pack<f16>(const PackParams&, hipStream_t);
template hipError_t launch_zero<f16>(void*, long, hipStream_t);
}  // namespace oaa
