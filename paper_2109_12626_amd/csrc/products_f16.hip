// The layer products' kernels for float16.
#include "products_kernels.hpp"

namespace dpar {
namespace products {

hipError_t launch_f16(Form f, const Args& a, hipStream_t stream) {
  return run_type<Type::F16>(f, a, stream);
}
hipError_t launch_slope_f16(const SlopeArgs& a, hipStream_t stream) {
  return run_slope<Type::F16>(a, stream);
}
hipError_t launch_sums_f16(const SumArgs& a, hipStream_t stream) {
  return run_sums<Type::F16>(a, stream);
}

}  // namespace products
}  // namespace dpar
