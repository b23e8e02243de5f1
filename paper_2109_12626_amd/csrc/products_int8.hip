// The layer products' kernels for 8-bit integers, and the rows' way there.
#include "products_kernels.hpp"

namespace dpar {
namespace products {
namespace {

using GivenCopy = const __attribute__((address_space(4))) CopyArgs;
using GivenQuantize = const __attribute__((address_space(4))) QuantizeArgs;

// A wavefront per row and turn, sizes in bytes.
__global__ __launch_bounds__(256) void k_int8_copy(CopyArgs) {
  GivenCopy& a = *(GivenCopy*)__builtin_amdgcn_kernarg_segment_ptr();
  auto& job = a.job[blockIdx.z];
  const int mat = blockIdx.y, lane = threadIdx.x % 64;
  if (mat >= job.mats) return;
  const signed char* from = (const signed char*)job.from[mat];
  char* to = job.to + (size_t)mat * job.rows * job.pitch;
  for (size_t row = (size_t)blockIdx.x * 4 + uniform(threadIdx.x / 64);
       row < job.rows; row += (size_t)gridDim.x * 4)
    for (size_t at = (size_t)lane * 16; at < job.pitch; at += 1024)
      *(i32x4*)(to + row * job.pitch + at) = load_piece<signed char>(
          from + row * job.ld + at, (long)job.cols - (long)at);
}

// What orders values by size, as whole numbers: infinities and NaN come after
// everything finite.  16-bit types: the larger of either half of the registers.
template <typename V>
__device__ inline uint32_t larger(uint32_t a, uint32_t b) {
  if constexpr (sizeof(V) == 4) return a > b ? a : b;
  typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(
      uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a),
                                          __builtin_bit_cast(u16x2, b)));
}
template <typename V>
__device__ inline uint32_t size_of_bits(int v) {
  return (uint32_t)v & (sizeof(V) == 4 ? 0x7fffffffu : 0x7fff7fffu);
}

// x / scale to the nearest whole number, halves to the even one; inverse: 1 /
// scale.  The sum of x * inverse and 1.5 * 2^23 rounds the exact product to a
// whole number, which its lower bits are.  The product is 2^-17 off at most (127
// times the inverse's rounding), so only one that near to a half is looked at
// again (*worst keeps the largest distance from a whole number).
constexpr float kWhole = 12582912.f;
__device__ inline float nearest(float x, float inverse, float* worst) {
  const float q = fmaf(x, inverse, kWhole);
  *worst = fmaxf(*worst, fabsf(fmaf(x, inverse, kWhole - q)));
  return q;
}
// With q whole and the product near to a half, x - q scale is a number of 24
// bits and comes exactly from a fused multiplication and addition.
__device__ inline float nearest_checked(float x, float scale, float inverse) {
  float q = rintf(x * inverse);
  const float e = fmaf(-q, scale, x), off = fabsf(e) * 2.f;
  if (off > scale || (off == scale && ((int)q & 1)))
    q += e > 0.f ? 1.f : -1.f;
  return kWhole + fminf(fmaxf(q, -127.f), 127.f);
}

// The lowest bytes of N values.
template <int N>
__device__ inline void store_bytes(signed char* q, const float* v, long left) {
  uint32_t w[N / 4];
#pragma unroll
  for (int k = 0; k < N / 4; ++k) {
    uint32_t b[4];
    __builtin_memcpy(b, v + k * 4, 16);
    w[k] = __builtin_amdgcn_perm(b[1], b[0], 0x0c0c0400u) |
           __builtin_amdgcn_perm(b[3], b[2], 0x04000c0cu);
  }
  if (left >= N) {
    __builtin_memcpy(q, w, N);
    return;
  }
#pragma unroll
  for (int k = 0; k < N; ++k)
    if (k < left) q[k] = (signed char)(w[k / 4] >> (k % 4 * 8));
}

// W wavefronts take a row, P pieces of 16 bytes per lane in registers between
// the two passes; what a row has beyond that is read again.
template <typename V, int W, int P>
__device__ inline void quantize_row(GivenQuantize& a, int rank, size_t row,
                                    LDS uint32_t* met) {
  constexpr int E = 16 / sizeof(V), kLanes = W * 64;
  const int t = threadIdx.x, lane = t % kLanes;
  const V* x = (const V*)a.x[rank] + row * a.ldx;
  const long cols = (long)a.cols, more = (long)(P * kLanes + lane) * E;
  i32x4 held[P];
#pragma unroll
  for (int n = 0; n < P; ++n) {
    const long j = (long)(n * kLanes + lane) * E;
    held[n] = j < cols ? load_piece<V>(x + j, cols - j) : i32x4{0, 0, 0, 0};
  }
  uint32_t most = 0;
  auto largest = [&](i32x4 piece) {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      most = larger<V>(most, size_of_bits<V>(piece[k]));
  };
#pragma unroll
  for (int n = 0; n < P; ++n) largest(held[n]);
  for (long j = more; j < cols; j += kLanes * E)
    largest(load_piece<V>(x + j, cols - j));
#pragma unroll
  for (int far = 1; far < 64; far *= 2)
    most = larger<V>(most, __shfl_xor(most, far));
  if constexpr (W > 1) {
    if ((t & 63) == 0) met[t / 64] = most;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < W; ++k) most = larger<V>(most, met[k]);
  }
  float big;
  if constexpr (sizeof(V) == 4) {
    big = __builtin_bit_cast(float, most);
  } else {
    const unsigned short hi = most >> 16, lo = (unsigned short)most;
    big = (float)__builtin_bit_cast(V, hi > lo ? hi : lo);
  }
  const bool fine = big < __builtin_inff();
  const float scale =
      fine ? big / 127.f : __builtin_bit_cast(float, 0x7fc00000u);
  if (lane == 0) a.scale[rank][row] = scale;
  // (a scale this small may have no inverse in 32 bits)
  const bool tiny = scale < 0x1p-100f, zero = !(scale > 0.f);
  const float s = tiny ? scale * 0x1p40f : scale, inverse = 1.f / s;
  signed char* q = a.q[rank] + row * a.ldq;
  auto give = [&](i32x4 piece, long j) {
    V v[E];
    float r[E], worst = 0.f;
    __builtin_memcpy(v, &piece, 16);
#pragma unroll
    for (int k = 0; k < E; ++k) r[k] = nearest((float)v[k], inverse, &worst);
    if (tiny || worst > 0.5f - 0x1p-14f) {
#pragma unroll
      for (int k = 0; k < E; ++k)
        r[k] = nearest_checked(tiny ? (float)v[k] * 0x1p40f : (float)v[k], s,
                               inverse);
    }
    if (zero) {
#pragma unroll
      for (int k = 0; k < E; ++k) r[k] = kWhole;
    }
    store_bytes<E>(q + j, r, cols - j);
  };
#pragma unroll
  for (int n = 0; n < P; ++n) {
    const long j = (long)(n * kLanes + lane) * E;
    if (j < cols) give(held[n], j);
  }
  for (long j = more; j < cols; j += kLanes * E)
    give(load_piece<V>(x + j, cols - j), j);
}

// 4 / W rows per workgroup.  Bound by memory: 8192 x 4096 bf16 23.8 us with four
// wavefronts to a row (4.2 TB/s; at the rate of a large copy 19.4), 30.9 with one,
// 34.5 with one that asks for the next row ahead in a quarter of the workgroups.
constexpr size_t kGroups = (size_t)1 << 22;      // along a launch's first axis
template <typename V, int W, int P>
__global__ __launch_bounds__(256) void k_quantize(QuantizeArgs) {
  GivenQuantize& a = *(GivenQuantize*)__builtin_amdgcn_kernarg_segment_ptr();
  __shared__ uint32_t met[4];
  const size_t row = ((size_t)blockIdx.z * kGroups + blockIdx.x) * (4 / W) +
                     uniform(threadIdx.x / (W * 64));
  if (row < a.rows)
    quantize_row<V, W, P>(a, blockIdx.y, row, (LDS uint32_t*)met);
}

// A wavefront takes rows of up to 128 pieces, a workgroup longer ones.
template <typename V>
hipError_t quantize(const QuantizeArgs& a, hipStream_t stream) {
  const size_t pieces = (a.cols + 16 / sizeof(V) - 1) / (16 / sizeof(V));
  const size_t n = pieces <= 128 ? (a.rows + 3) / 4 : a.rows;
  const dim3 grid((unsigned)std::min(n, kGroups), a.ranks,
                  (unsigned)((n + kGroups - 1) / kGroups)),
      threads(256);
  if (pieces <= 128)
    hipLaunchKernelGGL((k_quantize<V, 1, 2>), grid, threads, 0, stream, a);
  else if (pieces <= 512)
    hipLaunchKernelGGL((k_quantize<V, 4, 2>), grid, threads, 0, stream, a);
  else
    hipLaunchKernelGGL((k_quantize<V, 4, 4>), grid, threads, 0, stream, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_copy_int8(const CopyArgs& a, hipStream_t stream) {
  size_t most = 0;
  int mats = 0;
  for (int k = 0; k < a.jobs; ++k) {
    most = std::max(most, a.job[k].rows);
    mats = std::max(mats, a.job[k].mats);
  }
  const size_t blocks = std::min<size_t>((most + 3) / 4, 4096);
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
