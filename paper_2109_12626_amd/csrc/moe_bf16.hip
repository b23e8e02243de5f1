// The mixture-of-experts layer's kernels for bfloat16 activations.
#include "moe_kernels.hpp"

namespace dpar {
namespace moe {

hipError_t launch_bf16(bool eight, const Args& a, hipStream_t stream) {
  return eight ? run_moe<Type::I8, Type::BF16>(a, stream)
               : run_moe<Type::BF16, Type::BF16>(a, stream);
}

}  // namespace moe
}  // namespace dpar
