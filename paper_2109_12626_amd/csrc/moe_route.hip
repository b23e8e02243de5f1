// The mixture-of-experts layer: the choice of experts.
#include "moe_kernels.hpp"

namespace dpar {
namespace moe {
namespace {

constexpr int kRouteThreads = 1024;

// One workgroup per table.
__global__ __launch_bounds__(kRouteThreads) void k_moe_route(MoeArgs) {
  GivenMoe& a = *(GivenMoe*)__builtin_amdgcn_kernarg_segment_ptr();
  __shared__ int lds[Choice::bytes(kTokens * kTop, kExperts) / 4];
  const Choice c((LDS char*)lds, a.tokens * a.top,
                 a.experts * (a.tables == 1 ? a.ranks : 1));
  route<kRouteThreads>(a, blockIdx.x, c, -1, true);
}

}  // namespace

hipError_t launch_route(const Args& a, hipStream_t stream) {
  hipLaunchKernelGGL(k_moe_route, dim3(a.tables), dim3(kRouteThreads), 0,
                     stream, a);
  return hipGetLastError();
}

}  // namespace moe
}  // namespace dpar
