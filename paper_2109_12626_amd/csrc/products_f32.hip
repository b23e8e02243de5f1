// The layer products' kernels for float32.
#include "products_kernels.hpp"

namespace dpar {
namespace products {
namespace {

using GivenCopy = const __attribute__((address_space(4))) CopyArgs;

// One 16-byte piece of the copy per thread and turn, bound by memory (two
// 2001 x 2001 16-bit operands: 9.6 us).
__global__ __launch_bounds__(256) void k_copy(CopyArgs) {
  GivenCopy& a = *(GivenCopy*)__builtin_amdgcn_kernarg_segment_ptr();
  auto& job = a.job[blockIdx.z];
  const int mat = blockIdx.y;
  if (mat >= job.mats) return;
  const unsigned short* from = (const unsigned short*)job.from[mat];
  const size_t per = job.pitch / 16, all = per * job.rows;
  char* to = job.to + (size_t)mat * job.rows * job.pitch;
  for (size_t id = (size_t)blockIdx.x * 256 + threadIdx.x; id < all;
       id += (size_t)gridDim.x * 256) {
    const size_t row = id / per, piece = id % per;
    *(i32x4*)(to + id * 16) = load_piece<unsigned short>(
        from + row * job.ld + piece * 8, (long)job.cols - (long)piece * 8);
  }
}

}  // namespace

hipError_t launch_copy(const CopyArgs& a, hipStream_t stream) {
  size_t most = 0;
  int mats = 0;
  for (int k = 0; k < a.jobs; ++k) {
    most = std::max(most, a.job[k].pitch / 16 * a.job[k].rows);
    mats = std::max(mats, a.job[k].mats);
  }
  const size_t blocks = std::min<size_t>((most + 255) / 256, 2048);
  hipLaunchKernelGGL(k_copy, dim3((unsigned)blocks, mats, a.jobs), dim3(256),
                     0, stream, a);
  return hipGetLastError();
}

hipError_t launch_f32(Form f, const Args& a, hipStream_t stream) {
  return run_type<Type::F32>(f, a, stream);
}
hipError_t launch_slope_f32(const SlopeArgs& a, hipStream_t stream) {
  return run_slope<Type::F32>(a, stream);
}

}  // namespace products
}  // namespace dpar
