// The layer products' kernels for float32.
#include "products_kernels.hpp"

namespace dpar {
namespace products {

hipError_t launch_f32(Form f, const Args& a, hipStream_t stream) {
  return run_type<Type::F32>(f, a, stream);
}
hipError_t launch_slope_f32(const SlopeArgs& a, hipStream_t stream) {
  return run_slope<Type::F32>(a, stream);
}

}  // namespace products
}  // namespace dpar
