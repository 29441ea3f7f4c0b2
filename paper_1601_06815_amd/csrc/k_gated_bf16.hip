// The gated unit's products and passes, bf16.
#include "gated_few.hpp"
#include "gated_passes.hpp"
#include "product.hpp"

namespace oaa {
template hipError_t launch_product<bf16>(const ProductParams&, ProductKind, hipStream_t);
template hipError_t launch_few<bf16>(const FewParams&, hipStream_t);
template hipError_t launch_slope<bf16>(const SlopeParams&, hipStream_t);
template hipError_t launch_bias_join<bf16>(const float*, long, int, void*, void*, hipStream_t);
template hipError_t launch_join<bf16>(const JoinParams&, hipStream_t);
template hipError_t launch_pack<bf16>(const PackParams&, hipStream_t);
template hipError_t launch_zero<bf16>(void*, long, hipStream_t);
}  // namespace oaa
