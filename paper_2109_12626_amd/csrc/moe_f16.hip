// The mixture-of-experts layer's kernels for float16 activations.
#include "moe_kernels.hpp"

namespace dpar {
namespace moe {

hipError_t launch_f16(bool eight, const Args& a, hipStream_t stream) {
  return eight ? run_moe<Type::I8, Type::F16>(a, stream)
               : run_moe<Type::F16, Type::F16>(a, stream);
}

}  // namespace moe
}  // namespace dpar
