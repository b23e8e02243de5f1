// The layer products' kernels for bfloat16.
#include "products_kernels.hpp"

namespace dpar {
namespace products {

hipError_t launch_bf16(Form f, const Args& a, hipStream_t stream) {
  return run_type<Type::BF16>(f, a, stream);
}
hipError_t launch_slope_bf16(const SlopeArgs& a, hipStream_t stream) {
  return run_slope<Type::BF16>(a, stream);
}
hipError_t launch_sums_bf16(const SumArgs& a, hipStream_t stream) {
  return run_sums<Type::BF16>(a, stream);
}

}  // namespace products
}  // namespace dpar
