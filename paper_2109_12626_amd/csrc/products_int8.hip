// The layer products' kernels for 8-bit integers, and the rows' way there.
#include "products_kernels.hpp"

namespace dpar {
namespace products {
namespace {

using GivenCopy = const __attribute__((address_space(4))) CopyArgs;
using GivenQuantize = const __attribute__((address_space(4))) QuantizeArgs;

// One 16-byte piece per thread and turn, sizes in bytes.
__global__ __launch_bounds__(256) void k_int8_copy(CopyArgs) {
  GivenCopy& a = *(GivenCopy*)__builtin_amdgcn_kernarg_segment_ptr();
  auto& job = a.job[blockIdx.z];
  const int mat = blockIdx.y;
  if (mat >= job.mats) return;
  const signed char* from = (const signed char*)job.from[mat];
  const size_t per = job.pitch / 16, all = per * job.rows;
  char* to = job.to + (size_t)mat * job.rows * job.pitch;
  for (size_t id = (size_t)blockIdx.x * 256 + threadIdx.x; id < all;
       id += (size_t)gridDim.x * 256) {
    const size_t row = id / per, piece = id % per;
    *(i32x4*)(to + id * 16) = load_piece<signed char>(
        from + row * job.ld + piece * 16,
        (long)job.cols - (long)piece * 16);
  }
}

// x / scale to the nearest whole number, halves to the even one; inverse: 1 /
// scale.  x inverse is 2^-15 off at most (127 and three roundings of 2^-24
// each), so only a product that near to a half is looked at again: with q
// whole, x - q scale is a number of 24 bits and comes exactly from a fused
// multiplication and addition.
__device__ inline float nearest(float x, float scale, float inverse) {
  const float f = x * inverse;
  float q = rintf(f);
  if (fabsf(f - q) > 0.5f - 0x1p-14f) {
    const float e = fmaf(-q, scale, x), off = fabsf(e) * 2.f;
    const float toward = e > 0.f ? q + 1.f : q - 1.f;
    const bool odd = ((int)q & 1) != 0;
    if (off > scale || (off == scale && odd)) q = toward;
  }
  return fminf(fmaxf(q, -127.f), 127.f);
}

// N values as bytes.
template <int N>
__device__ inline void store_bytes(signed char* q, const float* v, long left) {
  signed char t[N];
#pragma unroll
  for (int k = 0; k < N; ++k) t[k] = (signed char)(int)v[k];
  if (left >= N) {
    __builtin_memcpy(q, t, N);
    return;
  }
#pragma unroll
  for (int k = 0; k < N; ++k)
    if (k < left) q[k] = t[k];
}

// W wavefronts take a row, P pieces of 16 bytes per lane in registers between
// the two passes; what a row has beyond that is read again.
template <typename V, int W, int P>
__device__ inline void quantize_row(GivenQuantize& a, int rank, size_t row,
                                    uint32_t (&met)[4]) {
  constexpr int E = 16 / sizeof(V), kLanes = W * 64;
  const int t = threadIdx.x, lane = t % kLanes;
  const V* x = (const V*)a.x[rank] + row * a.ldx;
  const long cols = (long)a.cols;

  i32x4 held[P];
  // as whole numbers: infinities and NaN come after everything finite
  uint32_t most = 0;
  auto largest = [&](i32x4 piece) {
    V v[E];
    __builtin_memcpy(v, &piece, 16);
#pragma unroll
    for (int k = 0; k < E; ++k) {
      const uint32_t b =
          __builtin_bit_cast(uint32_t, (float)v[k]) & 0x7fffffffu;
      most = b > most ? b : most;
    }
  };
#pragma unroll
  for (int n = 0; n < P; ++n) {
    const long j = (long)(n * kLanes + lane) * E;
    held[n] = j < cols ? load_piece<V>(x + j, cols - j) : i32x4{0, 0, 0, 0};
  }
#pragma unroll
  for (int n = 0; n < P; ++n) largest(held[n]);
  for (long j = (long)(P * kLanes + lane) * E; j < cols; j += kLanes * E)
    largest(load_piece<V>(x + j, cols - j));
#pragma unroll
  for (int far = 1; far < 64; far *= 2) {
    const uint32_t b = __shfl_xor(most, far);
    most = b > most ? b : most;
  }
  if constexpr (W > 1) {
    if ((t & 63) == 0) met[t / 64] = most;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < W; ++k) most = met[k] > most ? met[k] : most;
  }
  const bool fine = most < 0x7f800000u;
  const float scale = fine ? __builtin_bit_cast(float, most) / 127.f
                           : __builtin_bit_cast(float, 0x7fc00000u);
  if (lane == 0) a.scale[rank][row] = scale;
  // (a scale this small may have no inverse in 32 bits)
  const float lift = scale < 0x1p-100f ? 0x1p40f : 1.f;
  const float s = scale * lift, inverse = 1.f / s;
  signed char* q = a.q[rank] + row * a.ldq;
  auto give = [&](i32x4 piece, long j) {
    V v[E];
    float r[E];
    __builtin_memcpy(v, &piece, 16);
#pragma unroll
    for (int k = 0; k < E; ++k)
      r[k] = scale > 0.f ? nearest((float)v[k] * lift, s, inverse) : 0.f;
    store_bytes<E>(q + j, r, cols - j);
  };
#pragma unroll
  for (int n = 0; n < P; ++n) {
    const long j = (long)(n * kLanes + lane) * E;
    if (j < cols) give(held[n], j);
  }
  for (long j = (long)(P * kLanes + lane) * E; j < cols; j += kLanes * E)
    give(load_piece<V>(x + j, cols - j), j);
}

// A workgroup per row.
template <typename V>
__global__ __launch_bounds__(256) void k_quantize_few(QuantizeArgs) {
  GivenQuantize& a = *(GivenQuantize*)__builtin_amdgcn_kernarg_segment_ptr();
  __shared__ uint32_t met[4];
  quantize_row<V, 4, 4>(a, blockIdx.y, blockIdx.x, met);
}

// A wavefront per row.
template <typename V>
__global__ __launch_bounds__(256) void k_quantize(QuantizeArgs) {
  GivenQuantize& a = *(GivenQuantize*)__builtin_amdgcn_kernarg_segment_ptr();
  uint32_t none[4];
  for (size_t row = (size_t)blockIdx.x * 4 + uniform(threadIdx.x / 64);
       row < a.rows; row += (size_t)gridDim.x * 4)
    quantize_row<V, 1, 8>(a, blockIdx.y, row, none);
}

template <typename V>
hipError_t quantize(const QuantizeArgs& a, hipStream_t stream) {
  if (a.rows < 2048)
    hipLaunchKernelGGL(k_quantize_few<V>, dim3((unsigned)a.rows, a.ranks),
                       dim3(256), 0, stream, a);
  else
    hipLaunchKernelGGL(
        k_quantize<V>,
        dim3((unsigned)std::min<size_t>((a.rows + 3) / 4, 1 << 20), a.ranks),
        dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_copy_int8(const CopyArgs& a, hipStream_t stream) {
  size_t most = 0;
  int mats = 0;
  for (int k = 0; k < a.jobs; ++k) {
    most = std::max(most, a.job[k].pitch / 16 * a.job[k].rows);
    mats = std::max(mats, a.job[k].mats);
  }
  const size_t blocks = std::min<size_t>((most + 255) / 256, 2048);
  hipLaunchKernelGGL(k_int8_copy, dim3((unsigned)blocks, mats, a.jobs),
                     dim3(256), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_int8(Form f, const Args& a, hipStream_t stream) {
  return f == Form::GATED ? run_form<Type::I8, Form::GATED>(a, stream)
                          : run_form<Type::I8, Form::LINEAR>(a, stream);
}

hipError_t launch_quantize(const QuantizeArgs& a, hipStream_t stream) {
  switch ((Type)a.type) {
    case Type::BF16: return quantize<__bf16>(a, stream);
    case Type::F16: return quantize<_Float16>(a, stream);
    default: return quantize<float>(a, stream);
  }
}

}  // namespace products
}  // namespace dpar
