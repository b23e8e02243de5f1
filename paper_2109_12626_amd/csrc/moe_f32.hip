// The mixture-of-experts layer's kernels for float32 activations.
#include "moe_kernels.hpp"

namespace dpar {
namespace moe {

hipError_t launch_f32(const Args& a, hipStream_t stream) {
  return run_moe<Type::F32, Type::F32>(a, stream);
}

}  // namespace moe
}  // namespace dpar
