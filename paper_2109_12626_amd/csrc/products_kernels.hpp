// Layer products on gfx950's matrix cores: types bf16, fp16 and fp32, every
// form of products.hpp, results accumulated in fp32.  Figures: one MI355X,
// sizes as rows x in x out.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>
#include <type_traits>

#include "products.hpp"

namespace dpar {
namespace products {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

#define LDS __attribute__((address_space(3)))

// The arguments as the kernel finds them: read in place with scalar loads
// (indexing a by-value copy by rank would put all of it in scratch memory).
using Given = const __attribute__((address_space(4))) Args;
using GivenSlope = const __attribute__((address_space(4))) SlopeArgs;
using GivenSums = const __attribute__((address_space(4))) SumArgs;

// A piece is 16 bytes; every tile holds 128 bytes of the contraction: 64
// 16-bit or 32 32-bit values, in two steps of 4 pieces (one per lane group
// of 16).
constexpr int kLine = 128;

template <Type T> struct Elem;
template <> struct Elem<Type::BF16> {
  using V = __bf16;
  static __device__ f32x4 mma(i32x4 a, i32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(
        __builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0,
        0);
  }
  static __device__ i32x4 ones() {
    const bf16x8 v = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
    return __builtin_bit_cast(i32x4, v);
  }
};
template <> struct Elem<Type::F16> {
  using V = _Float16;
  static __device__ f32x4 mma(i32x4 a, i32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(
        __builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0,
        0);
  }
  static __device__ i32x4 ones() {
    const f16x8 v = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
    return __builtin_bit_cast(i32x4, v);
  }
};
template <> struct Elem<Type::F32> {
  using V = float;
  // Component s of the four lane groups' pieces makes one product of depth 4;
  // both operands order the contraction alike.
  static __device__ f32x4 part(i32x4 a, i32x4 b, f32x4 c, int s) {
    return __builtin_amdgcn_mfma_f32_16x16x4f32(
        __builtin_bit_cast(f32x4, a)[s], __builtin_bit_cast(f32x4, b)[s], c, 0,
        0, 0);
  }
  static __device__ f32x4 mma(i32x4 a, i32x4 b, f32x4 c) {
    for (int s = 0; s < 4; ++s) c = part(a, b, c, s);
    return c;
  }
  static __device__ i32x4 ones() {
    const f32x4 v = {1.f, 1.f, 1.f, 1.f};
    return __builtin_bit_cast(i32x4, v);
  }
};

// c[n] += a[n] b for N independent sums, in an order that leaves time between
// two products into one sum.
template <Type T, int N>
__device__ inline void mma_row(const i32x4 (&a)[N], i32x4 b, f32x4 (&c)[N]) {
  if constexpr (T == Type::F32) {
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int n = 0; n < N; ++n) c[n] = Elem<T>::part(a[n], b, c[n], s);
  } else {
#pragma unroll
    for (int n = 0; n < N; ++n) c[n] = Elem<T>::mma(a[n], b, c[n]);
  }
}

// ---------------------------------------------------------------- activations

// EXACT: results stored in 32 bits, a few units in the last place off.  Else
// what is rounded to 16 bits: there exponentials and reciprocals of one
// instruction or two will do (a correctly rounded division alone takes ten).
template <bool EXACT>
__device__ inline float inverse(float x) {
  return EXACT ? 1.f / x : __builtin_amdgcn_rcpf(x);
}
template <bool EXACT>
__device__ inline float power(float x) {
  return EXACT ? expf(x) : __expf(x);
}

// 1 / (1 + exp(-z)); *both: its product with 1 minus it.  From exp(-|z|), so
// that neither end loses what 1 - (almost 1) would.
template <bool EXACT>
__device__ inline float sigmoid(float z, float* both) {
  const float e = power<EXACT>(-fabsf(z)), big = inverse<EXACT>(1.f + e),
              small = e * big;
  *both = big * small;
  return z < 0.f ? small : big;
}
template <bool EXACT>
__device__ inline float sigmoid(float z) {
  return inverse<EXACT>(1.f + power<EXACT>(-z));
}

// 0.5 (1 + tanh a) = sigmoid(2 a)
constexpr float kTanh2 = 1.5957691216057308f;   // 2 sqrt(2 / pi)
constexpr float kCubic = 0.044715f;
constexpr float kInvSqrt2 = 0.70710678118654752f;
constexpr float kInvSqrt2Pi = 0.39894228040143268f;

// (1 + erf(z / sqrt 2)) / 2 and exp(-z^2 / 2).  Not EXACT: Abramowitz and
// Stegun 7.1.26, whose truncation is 7.5e-8 at most; in 32 bits the whole is
// 2.8e-7 off at most, measured over -12 .. 12 (EXACT: 9.3e-8): a thousandth of
// what rounding a result of 1 to fp16 costs.
template <bool EXACT>
__device__ inline float normal_cdf(float z, float* density) {
  if (EXACT) {
    *density = expf(-0.5f * z * z);
    return 0.5f * erfcf(-z * kInvSqrt2);
  }
  const float x = fabsf(z) * kInvSqrt2;
  const float t = inverse<false>(fmaf(0.3275911f, x, 1.f));
  const float e = __expf(-x * x);
  float p = fmaf(1.061405429f, t, -1.453152027f);
  p = fmaf(p, t, 1.421413741f);
  p = fmaf(p, t, -0.284496736f);
  p = fmaf(p, t, 0.254829592f);
  const float tail = 0.5f * p * t * e;
  *density = e;
  return z < 0.f ? tail : 1.f - tail;
}

// The activations beyond +-128 are z or -0 and their slopes 1 or 0 in 32 bits;
// z is held there so that infinities give the limits.
__device__ inline float held(float z) { return z < -128.f ? -128.f : z; }

template <Act A, bool EXACT>
__device__ inline float act_of(float z) {
  if (A == Act::RELU) return z > 0.f ? z : (z != z ? z : 0.f);
  if (A == Act::NONE) return z;
  z = held(z);
  if (A == Act::GELU) {
    float e;
    return z * normal_cdf<EXACT>(z, &e);
  }
  if (A == Act::GELU_TANH)
    return z * sigmoid<EXACT>(kTanh2 * (z + kCubic * z * z * z));
  return z * sigmoid<EXACT>(z);
}

// act(z) and act'(z)
template <Act A, bool EXACT>
__device__ inline float slope_of(float z, float* value) {
  if (A == Act::NONE) {
    *value = z;
    return 1.f;
  }
  if (A == Act::RELU) {
    *value = act_of<A, EXACT>(z);
    return z > 0.f ? 1.f : (z != z ? z : 0.f);
  }
  z = held(z);
  const float y = z > 128.f ? 128.f : z;
  if (A == Act::GELU) {
    float e;
    const float c = normal_cdf<EXACT>(y, &e);
    *value = z * c;
    return c + y * kInvSqrt2Pi * e;
  }
  if (A == Act::GELU_TANH) {
    float both;
    const float s =
        sigmoid<EXACT>(kTanh2 * (y + kCubic * y * y * y), &both);
    *value = z * s;
    return s + y * both * kTanh2 * (1.f + 3.f * kCubic * y * y);
  }
  float both;
  const float s = sigmoid<EXACT>(y, &both);
  *value = z * s;
  return s + y * both;
}

// f(activation) with the activation as a type: one branch for many values.
template <typename Fn>
__device__ inline void with_act(int act, Fn f) {
  switch (act) {
    case (int)Act::RELU: f(std::integral_constant<Act, Act::RELU>()); break;
    case (int)Act::GELU: f(std::integral_constant<Act, Act::GELU>()); break;
    case (int)Act::GELU_TANH:
      f(std::integral_constant<Act, Act::GELU_TANH>());
      break;
    case (int)Act::SILU: f(std::integral_constant<Act, Act::SILU>()); break;
    default: f(std::integral_constant<Act, Act::NONE>());
  }
}
// f(EXACT), which holds for 32-bit values and for 32-bit results (out32) of
// 16-bit ones.  Around loops over results: inside, the longer code of the exact
// forms made 16-bit results slower (7 x 875 x 1001 x 1000 fp16 gelu 37.0
// against 35.8 us).
template <Type T, bool ACTS = true, typename Fn>
__device__ inline void with_exact(bool out32, Fn f) {
  if constexpr (T == Type::F32) {
    f(std::integral_constant<bool, true>());
  } else {
    if (ACTS && out32)
      f(std::integral_constant<bool, true>());
    else
      f(std::integral_constant<bool, false>());
  }
}

// ---------------------------------------------------------------- tiles

__device__ const i32x4 g_zero = {0, 0, 0, 0};

// Where a piece lies in its LDS row: pieces are exchanged by a key of the row
// so that the 16 lanes that read together touch all banks.
//   CC (row of the operand, 8 pieces): lanes read one piece of 16 rows.
//   RC (one step of the contraction, W values): lanes read 4 contraction
//      rows x 16 values (16-bit, transposing reads), or one value each (32).
// G: distance of the 4-value groups that one matrix row index takes.
template <Type T, bool CC, int W, int G>
__device__ inline int key_of(int row) {
  if (CC) {
    if (G == 4) return row & 7;
    return (row & 3) | ((row / G & 1) << 2);
  }
  if (T == Type::F32) {
    const int q = (row >> 2) & 3;
    return G == 4 ? q * 4 : q;
  }
  // 64 values: two rows share the banks' 256 bytes
  const int r = W == 64 ? (row >> 1) & 1 : row & 3;
  const int hi = W == 64 ? (row >> 3) & 1 : 0;
  if (G == 4) return (r | hi << 1 | (W == 64 ? 0 : ((row >> 3) & 1) << 2)) * 2;
  if (G == 8) return r * 4;
  return r | ((row >> 3) & 1) << 3;
}

template <typename V>
__device__ inline i32x4 load_piece(const V* p, long n) {
  constexpr int E = 16 / sizeof(V);
  i32x4 v = {0, 0, 0, 0};
  if (n >= E) {
    __builtin_memcpy(&v, p, 16);       // any alignment
  } else if (n > 0) {
    V t[E];
    for (int k = 0; k < E; ++k) t[k] = k < n ? p[k] : (V)0.f;
    __builtin_memcpy(&v, t, 16);
  }
  return v;
}

// A whole piece.
template <bool ALIGNED, typename V>
__device__ inline i32x4 load_whole(const V* p) {
  if constexpr (ALIGNED) return *(const i32x4*)p;
  i32x4 v;
  __builtin_memcpy(&v, p, 16);
  return v;
}

// Sixteen bytes per lane straight from memory to LDS, lane after lane from
// `lds` on (the same address in the whole wavefront).  Written as assembly so
// that the compiler does not wait for them before every LDS read: the kernel
// waits itself (landed()) before the barrier that publishes a tile.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"   // m0: set before every use
__device__ inline void dma16(uint32_t lds, const void* base, uint32_t off) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\t"
               "global_load_lds_dwordx4 %1, %2"
               :: "s"(lds), "v"(off), "s"(base) : "memory", "m0");
}
// The same for data that is read once.
__device__ inline void dma16_once(uint32_t lds, const void* base,
                                  uint32_t off) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\t"
               "global_load_lds_dwordx4 %1, %2 nt"
               :: "s"(lds), "v"(off), "s"(base) : "memory", "m0");
}
__device__ inline void dma16_at(uint32_t lds, const void* p) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\t"
               "global_load_lds_dwordx4 %1, off"
               :: "s"(lds), "v"(p) : "memory", "m0");
}
#pragma clang diagnostic pop
template <int LEFT>
__device__ inline void landed() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" :: "n"(LEFT) : "memory");
}

// The workgroup's wavefronts meet.  The barrier alone orders nothing that the
// compiler moves; no access to memory or LDS crosses this.
__device__ inline void meet() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}
// The same for lanes of one wavefront that exchange values through LDS, which
// serves a wavefront's accesses in their order.
__device__ inline void in_order() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_wave_barrier();
  asm volatile("" ::: "memory");
}

// A value that is the same in every lane, in scalar registers.
__device__ inline uint32_t uniform(uint32_t v) {
  return __builtin_amdgcn_readfirstlane(v);
}
__device__ inline const char* uniform(const char* p) {
  const uint64_t v = (uint64_t)p;
  return (const char*)((uint64_t)uniform((uint32_t)(v >> 32)) << 32 |
                       uniform((uint32_t)v));
}

using Yes = std::integral_constant<bool, true>;
using No = std::integral_constant<bool, false>;

// One operand's tile: W rows (CC) or W values of every contraction step (RC).
template <Type T, bool CC, int W, int G, int THREADS>
struct Operand {
  using V = typename Elem<T>::V;
  static constexpr int E = 16 / sizeof(V);       // values per piece
  static constexpr int KT = kLine / sizeof(V);   // contraction per tile
  static constexpr int N = W * 8 / THREADS;      // pieces per thread
  static constexpr int P = CC ? 8 : W / E;       // pieces per LDS row

  // row, first value of thread t's n-th piece (LDS order is linear in t)
  static __device__ void at(int n, int t, int* row, int* val) {
    const int o = n * THREADS + t;
    *row = o / P;
    *val = ((o % P) ^ key_of<T, CC, W, G>(*row)) * E;
  }

  // Byte offset of a piece from the tile's first value at contraction 0.
  // Rows and values past the operand's end give the last ones (their results
  // are not stored).  Whole pieces only (fast operands).
  static __device__ uint32_t offset(size_t ld, size_t i0, size_t ni, int n,
                                    int t) {
    int row, val;
    at(n, t, &row, &val);
    const size_t most = ni - i0;        // i0 < ni
    if (CC) {
      if ((size_t)row >= most) row = (int)most - 1;
      return (uint32_t)(((size_t)row * ld + val) * sizeof(V));
    }
    if ((size_t)val >= most) val = (int)most - E;
    return (uint32_t)(((size_t)row * ld + val) * sizeof(V));
  }
  // Bytes from one contraction tile to the next, and to the tile's first
  // value.
  static __device__ size_t step(size_t ld) {
    return CC ? (size_t)kLine : (size_t)KT * ld * sizeof(V);
  }
  static __device__ size_t origin(size_t ld, size_t i0) {
    return (CC ? i0 * ld : i0) * sizeof(V);
  }
  // Whether a piece lies past the contraction's end (the last tile only).
  // Such pieces are read from somewhere inside the operand, and zeros take
  // their place once they have landed.
  static __device__ bool past(size_t c0, size_t nc, int n, int t) {
    int row, val;
    at(n, t, &row, &val);
    return c0 + (CC ? val : row) >= nc;
  }
  // What keeps a tile's offsets inside the operand: CC, the bytes to go back
  // for this lane's even or odd pieces (each at one place in their rows);
  // RC, the largest offset, that of the last piece of the last row.
  static __device__ uint32_t guard(size_t ld, size_t i0, size_t ni, size_t c0,
                                   size_t nc, int n, int t) {
    if constexpr (CC) {
      // (a lane's rows have one key, or one for even and one for odd n)
      static_assert(THREADS / P % G == 0 || G == 4);
      int row, val;
      at(n & 1, t, &row, &val);
      return c0 + val >= nc ? (uint32_t)(val * sizeof(V)) : 0;
    } else {
      const size_t last = nc - c0 < (size_t)KT ? nc - c0 - 1 : KT - 1;
      const size_t w = ni - i0 < (size_t)W ? ni - i0 : W;
      return (uint32_t)((last * ld + w - E) * sizeof(V));
    }
  }
  static __device__ uint32_t guarded(uint32_t off, uint32_t g) {
    return CC ? off - g : off < g ? off : g;
  }

  // The same for any alignment and length, into registers.
  static __device__ i32x4 fetch(const V* base, size_t ld, size_t i0, size_t ni,
                                size_t c0, size_t nc, int n, int t) {
    int row, val;
    at(n, t, &row, &val);
    if (CC) {
      size_t i = i0 + row;
      const size_t c = c0 + val;
      if (i >= ni) i = ni - 1;
      return load_piece<V>(base + i * ld + c, (long)nc - (long)c);
    }
    const size_t c = c0 + row, i = i0 + val;
    return load_piece<V>(base + c * ld + i,
                         c < nc ? (long)ni - (long)i : 0);
  }

  // The piece of the contraction that lane group q feeds the matrix cores
  // with in step ks, for 16 rows: group g of 4 of them starts at `first` +
  // g * G (+ group_of(g, n), so that in the end a lane holds G consecutive
  // results).  Where two groups share a bank's 16 bytes they take their
  // halves in opposite order.
  static __device__ int group_of(int g, int n) {
    return (G >= 16 ? n ^ (g & 1) : n) * 4;
  }
  static __device__ i32x4 frag(LDS char* s, int ks, int first, int n,
                               int lane) {
    const int r = lane & 15, q = lane >> 4;
    if constexpr (CC) {
      const int row = first + (r >> 2) * G + group_of(r >> 2, n) + (r & 3);
      const int piece = (ks * 4 + q) ^ key_of<T, CC, W, G>(row);
      return *(LDS i32x4*)(s + row * kLine + piece * 16);
    } else if constexpr (T == Type::F32) {
      i32x4 v;
      const int col = first + (r >> 2) * G + group_of(r >> 2, n) + (r & 3);
      for (int k = 0; k < 4; ++k) {
        const int c = ks * 16 + q * 4 + k;
        v[k] = *(LDS int*)(s + c * (W * 4) +
                           ((col >> 2) ^ key_of<T, CC, W, G>(c)) * 16 +
                           (col & 3) * 4);
      }
      return v;
    } else {
      // transposing read: within 16 lanes, lane 4 k + g gives the address of
      // 4 values of group g in contraction row k; lane r receives value
      // r % 4 of group r / 4 from the four rows
      i16x4 h[2];
      const int col = first + (r & 3) * G + group_of(r & 3, n);
      for (int k = 0; k < 2; ++k) {
        const int c = ks * 32 + q * 8 + k * 4 + (r >> 2);
        h[k] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (LDS i16x4*)(s + c * (W * 2) +
                         ((col >> 3) ^ key_of<T, CC, W, G>(c)) * 16 +
                         ((col >> 2) & 1) * 8));
      }
      i32x4 v;
      __builtin_memcpy(&v, h, 16);
      return v;
    }
  }
};

// ---------------------------------------------------------------- results

template <int BYTES> struct Piece;
template <> struct Piece<16> { using I = i32x4; };
template <> struct Piece<8> { using I = long; };
template <> struct Piece<4> { using I = int; };
template <> struct Piece<2> { using I = short; };

// N consecutive results of a row: in pieces of up to 16 bytes where they are
// aligned to that and all there (`left` are), else one by one.
template <typename V, int N>
__device__ inline void store_vals(V* p, const float* v, long left, bool wide) {
  constexpr int B = N * sizeof(V) < 16 ? N * sizeof(V) : 16, E = B / sizeof(V);
  using I = typename Piece<B>::I;
  if (wide && left >= N) {
#pragma unroll
    for (int k = 0; k < N; k += E) {
      V t[E];
#pragma unroll
      for (int e = 0; e < E; ++e) t[e] = (V)v[k + e];
      I w;
      __builtin_memcpy(&w, t, B);
      *(I*)(p + k) = w;
    }
    return;
  }
  if (left >= N) {
    V t[N];
#pragma unroll
    for (int k = 0; k < N; ++k) t[k] = (V)v[k];
    __builtin_memcpy(p, t, N * sizeof(V));
    return;
  }
#pragma unroll
  for (int k = 0; k < N; ++k)
    if (k < left) p[k] = (V)v[k];
}

template <typename V, int N>
__device__ inline void fetch_vals(const V* p, float* v, long left, bool wide) {
  constexpr int B = N * sizeof(V) < 16 ? N * sizeof(V) : 16, E = B / sizeof(V);
  using I = typename Piece<B>::I;
  if (wide && left >= N) {
#pragma unroll
    for (int k = 0; k < N; k += E) {
      const I w = *(const I*)(p + k);
      V t[E];
      __builtin_memcpy(t, &w, B);
#pragma unroll
      for (int e = 0; e < E; ++e) v[k + e] = (float)t[e];
    }
    return;
  }
  if (left >= N) {
    V t[N];
    __builtin_memcpy(t, p, N * sizeof(V));
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = (float)t[k];
    return;
  }
#pragma unroll
  for (int k = 0; k < N; ++k) v[k] = k < left ? (float)p[k] : 0.f;
}

template <int N>
__device__ inline void store_out(void* o, size_t at, const float* v, long left,
                                 int out32, bool wide, float) {
  store_vals<float, N>((float*)o + at, v, left, wide);
}
template <int N, typename V>
__device__ inline void store_out(void* o, size_t at, const float* v, long left,
                                 int out32, bool wide, V) {
  if (out32)
    store_vals<float, N>((float*)o + at, v, left, wide);
  else
    store_vals<V, N>((V*)o + at, v, left, wide);
}

// The biases of N consecutive results from j on: b[0] (GATED: of g), b[1] of u.
template <Type T, Form F, int N>
__device__ inline void fetch_bias(Given& a, int rank, size_t j,
                                  float (&b)[2][N]) {
  using V = typename Elem<T>::V;
  if constexpr (F == Form::LINEAR || F == Form::GATED) {
    const long left = (long)a.nj - (long)j;
#pragma unroll
    for (int p = 0; p < (F == Form::GATED ? 2 : 1); ++p) {
      if (const V* e = (const V*)a.e[p][rank]) {
        fetch_vals<V, N>(e + j, b[p], left, a.wide_out);
      } else {
#pragma unroll
        for (int k = 0; k < N; ++k) b[p][k] = 0.f;
      }
    }
  }
}

// Forms whose results have an activation.
constexpr bool acts(Form f) { return f == Form::LINEAR || f == Form::GATED; }

// N consecutive values j .. of row i: bias, activation, residual, rounding,
// stores.  v: the product's sums (GATED: v of g, u2 of u).
template <Type T, Form F, bool EXACT, int N>
__device__ inline void finish(Given& a, int rank, int pair, size_t i,
                              size_t j, float* v, float* u2,
                              const float (&b)[2][N]) {
  using V = typename Elem<T>::V;
  const long left = (long)a.nj - (long)j;
  const bool wide = a.wide_out;
  if constexpr (F == Form::LINEAR) {
    const void* r = a.e[1][rank];
    float t[N];
    if (r) {
      if (a.out32)
        fetch_vals<float, N>((const float*)r + i * a.lde + j, t, left, wide);
      else
        fetch_vals<V, N>((const V*)r + i * a.lde + j, t, left, wide);
    }
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] += b[0][k];
    if (V* z = (V*)a.o[1][rank])
      store_vals<V, N>(z + i * a.ldk + j, v, left, wide);
    with_act(a.act, [&](auto act) {
#pragma unroll
      for (int k = 0; k < N; ++k) v[k] = act_of<act.value, EXACT>(v[k]);
    });
    if (r) {
#pragma unroll
      for (int k = 0; k < N; ++k) v[k] += t[k];
    }
    store_out<N>(a.o[0][rank], i * a.ldo + j, v, left, a.out32, wide, V());
  } else if constexpr (F == Form::GATED) {
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] += b[0][k];
#pragma unroll
    for (int k = 0; k < N; ++k) u2[k] += b[1][k];
    if (V* g = (V*)a.o[1][rank])
      store_vals<V, N>(g + i * a.ldk + j, v, left, wide);
    if (V* u = (V*)a.u[0][rank])
      store_vals<V, N>(u + i * a.ldk + j, u2, left, wide);
    with_act(a.act, [&](auto act) {
#pragma unroll
      for (int k = 0; k < N; ++k)
        v[k] = act_of<act.value, EXACT>(v[k]) * u2[k];
    });
    store_out<N>(a.o[0][rank], i * a.ldo + j, v, left, a.out32, wide, V());
  } else {
    store_out<N>(a.o[F == Form::DW ? pair : 0][rank], i * a.ldo + j, v, left,
                 a.out32, wide, V());
  }
}

// One operand's addresses along the contraction: the tile to ask for next, kept
// in scalar registers so that the loop neither loads nor multiplies for them.
// DX: the second pair follows the first.
struct Walk {
  const char *p, *u;          // the tile's first value (u: GATED, of u)
  const char *o, *ou;         // the operands themselves
  const char *p2, *o2;        // DX: the second pair's
  size_t step;
  unsigned c, n;              // the tile, and the tiles of a pair

  __device__ void next() {
    p = uniform(p + step);
    u = uniform(u + step);
    if (++c == n && p2) {
      p = p2;
      o = o2;
      c = 0;
    }
  }
};

// OP's addresses from tile `first` on; b, b2: the (first) pair's and the second
// pair's operand, u: GATED, the second weights.
template <Form F, typename OP>
__device__ inline Walk walk_from(const void* b, const void* u, const void* b2,
                                 size_t ld, size_t i0, unsigned first,
                                 unsigned tiles) {
  Walk x;
  x.step = OP::step(ld);
  x.n = tiles;
  const size_t o = OP::origin(ld, i0);
  const bool second = F == Form::DX && first >= tiles;
  x.p2 = F == Form::DX && b2 && !second ? (const char*)b2 + o : nullptr;
  x.o2 = (const char*)b2;
  x.o = (const char*)(second ? b2 : b);
  x.ou = (const char*)u;
  x.c = second ? first - tiles : first;
  x.p = uniform((const char*)(second ? b2 : b) + o + x.c * x.step);
  x.u = u ? uniform((const char*)u + o + x.c * x.step) : x.p;
  return x;
}

// Which results a workgroup computes.
template <int BM, int BJ>
struct Place {
  size_t i0, j0;        // first row and column
  unsigned split;       // part of the contraction
  int rank, pair;

  __device__ Place(Given& a, Form form) {
    // (weights' gradients without columns still have bias sums)
    const size_t mt = (a.ni + BM - 1) / BM,
                 nt = a.nj ? (a.nj + BJ - 1) / BJ : 1;
    // consecutive workgroups go to the 8 XCDs in turn: give each XCD a run of
    // neighbouring tiles so that they share operands in its L2
    unsigned id = blockIdx.x;
    {
      const unsigned n = gridDim.x, per = n / 8, more = n % 8;
      const unsigned x = id % 8, k = id / 8;
      id = x * per + (x < more ? x : more) + k;
    }
    // (the host keeps the number of workgroups below 2^31)
    const unsigned tiles = (unsigned)mt * (unsigned)nt;
    split = uniform(id % a.splits);
    unsigned rest = id / a.splits;
    const unsigned tile = rest % tiles;
    rest = uniform(rest / tiles);
    pair = form == Form::DW ? rest % a.pairs : 0;
    rank = form == Form::DW ? rest / a.pairs : rest;
    // groups of 8 tile rows, columns inside
    const unsigned eight = 8 * (unsigned)nt;
    const unsigned row8 = tile / eight, in = tile % eight;
    const unsigned left = (unsigned)mt - row8 * 8, high = left < 8 ? left : 8;
    i0 = (size_t)uniform(row8 * 8 + in % high) * BM;
    j0 = (size_t)uniform(in / high) * BJ;
  }
};

// The sums of A over the contraction (bias gradients) that a wavefront holds:
// of its rows m * 16 .. with m % SHARES == its share, each 16 in a product of
// their own with ones, so that a value that is not finite stays in its row.
template <int MI, int SHARES>
struct Sums {
  static constexpr int N = MI / SHARES;
  static_assert(MI % SHARES == 0);
  f32x4 v[N] = {};

  template <Type T>
  __device__ void add(int m, int share, i32x4 a) {
    if (m % SHARES == share)
      v[m / SHARES] = Elem<T>::mma(Elem<T>::ones(), a, v[m / SHARES]);
  }
};

// Joins the parts of bias gradients that SumArgs left, in their order: those of
// the tile's rows, by the workgroup of its first columns (a launch of its own
// took 5 us).
template <Type T, int BM>
__device__ inline void join_sums(Given& a, int rank, int pair, unsigned split,
                                 size_t i0, size_t j0) {
  const size_t i = i0 + threadIdx.x;
  if (!a.sum || split != 0 || j0 != 0 || threadIdx.x >= BM || i >= a.ni)
    return;
  const float* w = a.sum + ((size_t)(a.first + rank) * a.pairs + pair) * a.ni +
                   i;
  const size_t step = (size_t)a.all * a.pairs * a.ni;
  float v = 0.f;
#pragma unroll 16
  for (int k = 0; k < a.parts; ++k) v += w[k * step];
  store_out<1>(a.u[pair][rank], i, &v, 1, a.out32, false,
               typename Elem<T>::V());
}

// Stores a wavefront's WM x WN results (GATED: g's and u's halves) from row iw
// and column jw on, and the sums of A that it holds.
template <Type T, Form F, bool SUMS, int WM, int WN, int SHARES, typename OB>
struct Results {
  using V = typename Elem<T>::V;
  static constexpr bool kGated = F == Form::GATED;
  static constexpr int MI = WM / 16, NJ = WN / 16, NT = kGated ? NJ / 2 : NJ;

  static __device__ void store(Given& a, int rank, int pair, unsigned split,
                               size_t iw, size_t jw, bool sums, int share,
                               const Sums<MI, SHARES>& sum,
                               f32x4 (&acc)[MI][NJ], LDS char* lds, int wave,
                               int lane) {
    if constexpr (SUMS)
      if (sums && lane < 16) {
        // (every lane group holds the same sums, of row `lane`)
#pragma unroll
        for (int n = 0; n < Sums<MI, SHARES>::N; ++n) {
          const size_t i = iw + (n * SHARES + share) * 16 + lane;
          if (i >= a.ni) continue;
          float v = sum.v[n][0];
          if (a.splits == 1)
            store_out<1>(a.u[pair][rank], i, &v, 1, a.out32, false, V());
          else    // after all partial results: [split][rank][pair][row]
            a.part[(size_t)a.splits * a.ranks * a.pairs * a.ni * a.nj +
                   (((size_t)split * a.ranks + rank) * a.pairs + pair) * a.ni +
                   i] = v;
        }
      }

    // Results by way of LDS (each wavefront its own part, MH of its tile rows
    // at a time), so that 8 consecutive ones are in one lane, whole rows side
    // by side in a store, and the code that finishes them stays short.
    constexpr int MH = MI < 4 ? MI : 4, CH = WN / 4,
                  PER = (kGated ? WN / 2 : WN) / 8;
    constexpr int kTurn = CH < 16 ? CH - 1 : 15;   // pieces exchanged by row
    LDS char* mine = lds + wave * (MH * 16 * WN * 4);
    // a lane's results are all in the same 8 columns
    static_assert(64 % PER == 0);
    const int c = lane % PER * 2;
    const size_t j = jw + c * 4;
    float bias[2][8];
    if (a.splits == 1 && j < a.nj) fetch_bias<T, F, 8>(a, rank, j, bias);
    landed<0>();
    meet();
#pragma unroll
    for (int mh = 0; mh < MI; mh += MH) {
      const int r = lane & 15, q = lane >> 4;
#pragma unroll
      for (int m = 0; m < MH; ++m)
#pragma unroll
        for (int n = 0; n < NJ; ++n) {
          // lane (r, q): row r, columns q * G + n * 4 ..; u's after g's
          const int c = n < NT ? q * NT + OB::group_of(q, n) / 4
                               : CH / 2 + q * NT + OB::group_of(q, n - NT) / 4;
          *(LDS f32x4*)(mine + (m * 16 + r) * (WN * 4) +
                        (c ^ (r & kTurn)) * 16) = acc[mh + m][n];
        }
      in_order();
      with_exact<T, acts(F)>(a.out32, [&](auto exact) {
#pragma unroll 1
        for (int row = lane / PER; row < MH * 16; row += 64 / PER) {
          const size_t i = iw + mh * 16 + row;
          if (i >= a.ni || j >= a.nj) continue;
          float v[8], u2[8];
          LDS char* at = mine + row * (WN * 4);
          const int x = row & kTurn;
          *(f32x4*)v = *(LDS f32x4*)(at + (c ^ x) * 16);
          *(f32x4*)(v + 4) = *(LDS f32x4*)(at + ((c + 1) ^ x) * 16);
          if constexpr (kGated) {
            *(f32x4*)u2 = *(LDS f32x4*)(at + ((CH / 2 + c) ^ x) * 16);
            *(f32x4*)(u2 + 4) = *(LDS f32x4*)(at + ((CH / 2 + c + 1) ^ x) * 16);
          }
          if (a.splits == 1) {
            finish<T, F, exact.value, 8>(a, rank, pair, i, j, v, u2, bias);
          } else {
            // [split][rank][pair or projection][row][column]
            const int np = F == Form::DW ? a.pairs : kGated ? 2 : 1;
            const size_t sz = a.ni * a.nj;
            float* p = a.part + (((size_t)split * a.ranks + rank) * np + pair)
                       * sz + i * a.nj + j;
            const long left = (long)a.nj - (long)j;
            const bool wide = a.nj % 4 == 0;
            store_vals<float, 8>(p, v, left, wide);
            if constexpr (kGated) store_vals<float, 8>(p + sz, u2, left, wide);
          }
        }
      });
      in_order();
    }
  }
};

// ---------------------------------------------------------------- the kernels

// C = A B over BM x BN results per workgroup (GATED: BN / 2 of g and of u), a
// tile of 128 bytes of the contraction at a time from one of R buffers in LDS.
// A result costs 2 / BN + 2 / BM values read from L2 per product, so large
// sizes are bound by the matrix cores with large tiles (PingPong below) and
// small ones by how many workgroups there are: 64 x 64 with two buffers (5
// workgroups per CU) or four (2 per CU, three tiles on their way: 128 x 4096 x
// 4096 26.6 against 37.0 us), 128 x 128 with two (2 per CU).  fp32 always runs
// here, bound by its matrix products (76% busy, 124 TFLOP/s at 8 x 256 x 1024
// x 4096).
//
// FAST: operands of whole aligned pieces, straight to LDS.  Else by way of
// registers, half a tile ahead (asking a whole tile ahead was no faster: 36 and
// 38 us at 7 x 875 x 1001 x 1000; loads off 16 bytes take two to three times
// as long).
//
// SUMS: DW with the sums of A.
template <Type T, Form F, bool SUMS, bool FAST, int BM, int BN, int WM, int WN,
          int R>
struct Tiled {
  using V = typename Elem<T>::V;
  static constexpr bool kGated = F == Form::GATED;
  static constexpr bool kACC = F != Form::DW;
  static constexpr bool kBCC = F == Form::LINEAR || F == Form::GATED;
  static constexpr int kThreads = BM / WM * (BN / WN) * 64;
  static constexpr int MI = WM / 16, NJ = WN / 16;
  // a lane's consecutive results: 4 per tile of 16, over all tiles of the
  // wave (GATED: half are g's, half u's)
  static constexpr int NT = kGated ? NJ / 2 : NJ;
  static constexpr int G = 4 * NT;
  static constexpr int BJ = kGated ? BN / 2 : BN;   // result columns
  using OA = Operand<T, kACC, BM, 4, kThreads>;
  using OB = Operand<T, kBCC, BN, G, kThreads>;
  static constexpr int KT = OA::KT;
  static constexpr int kBytesA = BM * kLine, kBytes = (BM + BN) * kLine;

  static __device__ void run(Given& a, LDS char* lds) {
    const int t = threadIdx.x, lane = t & 63, wave = uniform(t >> 6);
    const int wm = wave / (BN / WN), wn = wave % (BN / WN);
    const Place<BM, BJ> at(a, F);
    const int rank = at.rank, pair = at.pair;
    const unsigned split = at.split;
    const size_t i0 = at.i0, j0 = at.j0;

    const unsigned nk1 = (unsigned)((a.nc + KT - 1) / KT);
    const unsigned nk = F == Form::DX ? nk1 * a.pairs : nk1;
    const unsigned k0 = uniform((unsigned)((uint64_t)nk * split / a.splits)),
                   k1 = uniform((unsigned)((uint64_t)nk * (split + 1) /
                                           a.splits));
    const unsigned whole = uniform((unsigned)(a.nc / KT));  // tiles

    f32x4 acc[MI][NJ] = {};
    Sums<MI, BN / WN> sum;
    const bool sums = SUMS && a.u[pair][rank] && j0 == 0;

    // addresses: a 64-bit base per operand and contraction tile (scalar), a
    // 32-bit offset per piece
    uint32_t va[FAST ? OA::N : 1], vb[FAST ? OB::N : 1];
    i32x4 ra[FAST ? 1 : OA::N], rb[FAST ? 1 : OB::N];
    if constexpr (FAST) {
#pragma unroll
      for (int n = 0; n < OA::N; ++n)
        va[n] = OA::offset(a.lda, i0, a.na, n, t);
      // (GATED: the tile's second half holds u's rows, from j0 again)
#pragma unroll
      for (int n = 0; n < OB::N; ++n)
        vb[n] = kGated ? OB::offset(a.ldb, j0, a.nb, n % (OB::N / 2), t)
                       : OB::offset(a.ldb, j0, a.nb, n, t);
    }
    const uint32_t lds0 = (uint32_t)(uintptr_t)lds +
                          uniform(wave) * 1024;

    Walk xa = walk_from<F, OA>(a.a[pair][rank], nullptr, a.a[1][rank], a.lda,
                               i0, k0, nk1),
         xb = walk_from<F, OB>(a.b[0][rank], kGated ? a.b[1][rank] : nullptr,
                               a.b[1][rank], a.ldb, j0, k0, nk1);
    constexpr int kPieces = OA::N + OB::N;
    // Pieces n0 .. n1 - 1 of the next tile (A's, then B's) into a buffer.
    auto dma = [&](int buf, int n0, int n1) {
      const uint32_t d = lds0 + buf * kBytes;
      const size_t c0 = (size_t)xa.c * KT;
      const bool all = xa.c < whole;
      const uint32_t ga =
          all ? 0 : OA::guard(a.lda, i0, a.na, c0, a.nc, 0, t);
#pragma unroll
      for (int n = n0; n < n1; ++n) {
        const int m = n - OA::N;
        if (n < OA::N)
          dma16(d + n * kThreads * 16, xa.p,
                all ? va[n] : OA::guarded(va[n], ga));
        else
          dma16(d + n * kThreads * 16, kGated && m >= OB::N / 2 ? xb.u : xb.p,
                all ? vb[m]
                    : OB::guarded(vb[m], OB::guard(a.ldb, j0, a.nb, c0, a.nc,
                                                   m, t)));
      }
    };
    auto walk = [&] {
      xa.next();
      xb.next();
    };
    // Loads the next contraction tile: FAST into LDS, else into registers.
    auto issue = [&](int buf) {
      if constexpr (FAST) {
        dma(buf, 0, kPieces);
      } else {
        const size_t c0 = (size_t)xa.c * KT;
#pragma unroll
        for (int n = 0; n < OA::N; ++n)
          ra[n] = OA::fetch((const V*)xa.o, a.lda, i0, a.ni, c0, a.nc, n, t);
#pragma unroll
        for (int n = 0; n < OB::N; ++n) {
          const bool up = kGated && n >= OB::N / 2;
          rb[n] = OB::fetch((const V*)(up ? xb.ou : xb.o), a.ldb,
                            up ? j0 - BJ : j0, a.nj, c0, a.nc, n, t);
        }
      }
      walk();
    };
    // Zeros in the place of this thread's pieces past the contraction's end,
    // after they have landed.
    auto clear = [&](unsigned kt, int buf) {
      const unsigned c = F == Form::DX && kt >= nk1 ? kt - nk1 : kt;
      if (!FAST || c < whole) return;
      LDS char* d = lds + buf * kBytes + t * 16;
      int o = t;
      asm volatile("" : "+v"(o));    // (nothing kept for it in the loop)
#pragma unroll 1
      for (int n = 0; n < kPieces; ++n)
        if (n < OA::N ? OA::past((size_t)c * KT, a.nc, n, o)
                      : OB::past((size_t)c * KT, a.nc, n - OA::N, o))
          *(LDS i32x4*)(d + n * kThreads * 16) = i32x4{0, 0, 0, 0};
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    };
    auto land = [&](int buf) {
      if constexpr (!FAST) {
        LDS char* d = lds + buf * kBytes + t * 16;
#pragma unroll
        for (int n = 0; n < OA::N; ++n)
          *(LDS i32x4*)(d + n * kThreads * 16) = ra[n];
        d += kBytesA;
#pragma unroll
        for (int n = 0; n < OB::N; ++n)
          *(LDS i32x4*)(d + n * kThreads * 16) = rb[n];
      }
    };

    // Two steps per tile.  While the matrix cores work on one step, the next
    // one's fragments are read: B's into registers of their own, A's row by
    // row into those the products have just used.  One barrier per tile, in
    // the middle of the second step: by then every wavefront has read all of
    // this tile, so its buffer takes the tile after next, and the next tile,
    // asked for one tile ago, has landed.  The order is the program's
    // (sched_barrier): left alone the compiler reads each fragment just before
    // its use.
    i32x4 fa[MI], fb[2][NJ];
    auto read_b = [&](int ks, int buf) {
      LDS char* sb = lds + buf * kBytes + kBytesA;
#pragma unroll
      for (int n = 0; n < NJ; ++n) {
        const int first = kGated ? (n < NT ? 0 : BJ) + wn * (WN / 2)
                                 : wn * WN;
        fb[ks][n] = OB::frag(sb, ks, first, n % NT, lane);
      }
    };
    auto read_a = [&](int m, int ks, int buf) {
      fa[m] = OA::frag(lds + buf * kBytes, ks, wm * WM + m * 16, 0, lane);
    };
    auto multiply = [&](int m, int ks, auto with_sums) {
      mma_row<T>(fb[ks], fa[m], acc[m]);
      if constexpr (with_sums) sum.template add<T>(m, wn, fa[m]);
    };
    static_assert(kPieces % (MI / 2) == 0);
    auto loop = [&](auto with_sums) {
      int buf = 0;
#pragma unroll 1
      for (unsigned kt = k0; kt < k1; ++kt) {
        const int then = buf + 1 == R ? 0 : buf + 1;
        const bool ahead = kt + R < k1;
        if (!FAST && ahead) issue(buf);
        read_b(1, buf);
#pragma unroll
        for (int m = 0; m < MI; ++m) {
          multiply(m, 0, with_sums);
          read_a(m, 1, buf);
          __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int m = 0; m < MI / 2; ++m) multiply(m, 1, with_sums);
        __builtin_amdgcn_sched_barrier(0);
        if (FAST && kt + R - 1 < k1)
          landed<(R - 2) * kPieces>();
        else
          landed<0>();
        if (kt + 1 < k1) clear(kt + 1, then);
        meet();
        __builtin_amdgcn_sched_barrier(0);
        if (!FAST && ahead) land(buf);
        // (after the last tile this reads a buffer that nothing uses any
        // more)
        read_b(0, then);
#pragma unroll
        for (int m = MI / 2; m < MI; ++m) {
          read_a(m - MI / 2, 0, then);
          multiply(m, 1, with_sums);
          read_a(m, 0, then);
          if (FAST && ahead) {
            constexpr int kEach = kPieces / (MI / 2);
            dma(buf, (m - MI / 2) * kEach, (m - MI / 2 + 1) * kEach);
            if (m == MI - 1) walk();
          }
          __builtin_amdgcn_sched_barrier(0);
        }
        buf = then;
      }
    };

    if (k0 < k1) {
#pragma unroll
      for (int n = 0; n < R; ++n)
        if (k0 + n < k1) {
          issue(n);
          land(n);
        }
      if (FAST && k0 + R - 1 < k1)
        landed<(R - 1) * kPieces>();
      else
        landed<0>();
      clear(k0, 0);
      meet();
      read_b(0, 0);
#pragma unroll
      for (int m = 0; m < MI; ++m) read_a(m, 0, 0);
      // (kept apart from the loop's reads: merged with them they would move
      // into the loop, in front of their use)
#pragma unroll
      for (int m = 0; m < MI; ++m) asm volatile("" : "+v"(fa[m]));
#pragma unroll
      for (int n = 0; n < NJ; ++n) asm volatile("" : "+v"(fb[0][n]));
      if constexpr (SUMS) {
        if (sums)
          loop(Yes{});
        else
          loop(No{});
      } else {
        loop(No{});
      }
    }

    Results<T, F, SUMS, WM, WN, BN / WN, OB>::store(
        a, rank, pair, split, i0 + wm * WM,
        j0 + wn * (kGated ? WN / 2 : WN), sums, wn, sum, acc, lds, wave, lane);
    if constexpr (F == Form::DW && !SUMS)
      join_sums<T, BM>(a, rank, pair, split, i0, j0);
  }
};

// 256 x BN results (GATED: 256 x BN / 2 of each), 8 wavefronts of 128 x 64 (BN
// = 256) or 64 x 64 (BN = 128).  A tile of the contraction is 128 bytes of 256
// rows of A and of BN rows of B; the LDS holds three tiles of A and two (BN =
// 256: 160 KB in all) or three of B, so that loads have one and a half or two
// tiles of time to arrive.  (Stages of 64 bytes a row would leave more, but
// loads of 64 bytes of 16 rows reach half the rate of 128 bytes of 8: 67
// against 123 GB/s per CU from L2.)
//
// Each SIMD has two wavefronts, one of either half of the workgroup, and the
// halves run one phase apart: while one half reads the fragments of a step
// and asks for a later operand, the other has the matrix cores to itself (32
// or 16 products of 16 x 16 x 32, 512 or 256 cycles); then a barrier, and they
// change places.
//
// 256 x 256 (two operands of 64 KB per 2 x 256 x 256 x 64 products) reaches
// 1200 to 1290 TFLOP/s, by card, at 8192 x 4096 x 16384 with both results
// stored, 1470 without the stores: power bound, the matrix cores 63% busy at
// 1.7 to 1.9 GHz.  256 x 128
// fills the card with half the results (1 x 2048 x 4096 x 4096: 69 us, 80 with
// 256 x 256, 76 with 128 x 128).
//
// Operands of whole aligned pieces only (FAST in Tiled); SUMS as there.
template <Type T, Form F, bool SUMS, int BN>
struct PingPong {
  using V = typename Elem<T>::V;
  static constexpr bool kGated = F == Form::GATED;
  static constexpr bool kACC = F != Form::DW;
  static constexpr bool kBCC = F == Form::LINEAR || F == Form::GATED;
  static constexpr int BM = 256, WM = BN == 256 ? 128 : 64, WN = 64;
  static constexpr int kThreads = 512, kAcross = BN / WN;
  static constexpr int MI = WM / 16, NJ = WN / 16, NT = kGated ? NJ / 2 : NJ;
  static constexpr int G = 4 * NT, BJ = kGated ? BN / 2 : BN;
  using OA = Operand<T, kACC, BM, 4, kThreads>;
  using OB = Operand<T, kBCC, BN, G, kThreads>;
  static constexpr int KT = OA::KT, NA = OA::N, NB = OB::N;
  // tiles of A and of B in LDS
  static constexpr int kRingA = 3, kRingB = BN == 256 ? 2 : 3;
  static constexpr int kSlotA = BM * kLine, kSlotB = BN * kLine;
  static constexpr int kLds = kRingA * kSlotA + kRingB * kSlotB;
  static_assert(kLds <= 160 * 1024);

  static __device__ void run(Given& a, LDS char* lds) {
    const int t = threadIdx.x, lane = t & 63, wave = uniform(t >> 6);
    const int wm = wave / kAcross, wn = wave % kAcross;
    const bool late = wave >= 4;             // the half that runs behind
    const Place<BM, BJ> at(a, F);
    const int rank = at.rank, pair = at.pair;
    const unsigned split = at.split;
    const size_t i0 = at.i0, j0 = at.j0;

    const unsigned nk1 = (unsigned)((a.nc + KT - 1) / KT);
    const unsigned nk = F == Form::DX ? nk1 * a.pairs : nk1;
    const unsigned k0 = uniform((unsigned)((uint64_t)nk * split / a.splits)),
                   k1 = uniform((unsigned)((uint64_t)nk * (split + 1) /
                                           a.splits));
    const unsigned whole = uniform((unsigned)(a.nc / KT));

    f32x4 acc[MI][NJ] = {};
    Sums<MI, kAcross> sum;
    const bool sums = SUMS && a.u[pair][rank] && j0 == 0;

    uint32_t va[NA], vb[NB];
#pragma unroll
    for (int n = 0; n < NA; ++n) va[n] = OA::offset(a.lda, i0, a.na, n, t);
#pragma unroll
    for (int n = 0; n < NB; ++n)
      vb[n] = OB::offset(a.ldb, j0, a.nb, kGated ? n % (NB / 2) : n, t);
    LDS char* const ringb = lds + kRingA * kSlotA;
    const uint32_t lds0 = (uint32_t)(uintptr_t)lds + wave * 1024;

    Walk xa = walk_from<F, OA>(a.a[pair][rank], nullptr, a.a[1][rank], a.lda,
                               i0, k0, nk1),
         xb = walk_from<F, OB>(a.b[0][rank], kGated ? a.b[1][rank] : nullptr,
                               a.b[1][rank], a.ldb, j0, k0, nk1);

    // A's or B's part of the next tile into a slot.
    auto ask_a = [&](int slot) {
      const uint32_t d = lds0 + slot * kSlotA;
      if (xa.c < whole) {
#pragma unroll
        for (int n = 0; n < NA; ++n) dma16(d + n * kThreads * 16, xa.p, va[n]);
      } else {
        const uint32_t g = OA::guard(a.lda, i0, a.na, (size_t)xa.c * KT, a.nc,
                                     0, t);
#pragma unroll
        for (int n = 0; n < NA; ++n)
          dma16(d + n * kThreads * 16, xa.p, OA::guarded(va[n], g));
      }
      xa.next();
    };
    auto ask_b = [&](int slot) {
      const uint32_t d = lds0 + kRingA * kSlotA + slot * kSlotB;
      if (xb.c < whole) {
#pragma unroll
        for (int n = 0; n < NB; ++n)
          dma16(d + n * kThreads * 16, kGated && n >= NB / 2 ? xb.u : xb.p,
                vb[n]);
      } else {
#pragma unroll
        for (int n = 0; n < NB; ++n)
          dma16(d + n * kThreads * 16, kGated && n >= NB / 2 ? xb.u : xb.p,
                OB::guarded(vb[n], OB::guard(a.ldb, j0, a.nb,
                                             (size_t)xb.c * KT, a.nc, n, t)));
      }
      xb.next();
    };
    // As in Tiled: zeros past the contraction's end.
    auto clear = [&](unsigned kt) {
      const unsigned c = F == Form::DX && kt >= nk1 ? kt - nk1 : kt;
      if (c < whole) return;
      const size_t c0 = (size_t)c * KT;
      LDS char* da = lds + (kt - k0) % kRingA * kSlotA + t * 16;
      LDS char* db = ringb + (kt - k0) % kRingB * kSlotB + t * 16;
      int o = t;
      asm volatile("" : "+v"(o));
#pragma unroll 1
      for (int n = 0; n < NA; ++n)
        if (OA::past(c0, a.nc, n, o))
          *(LDS i32x4*)(da + n * kThreads * 16) = i32x4{0, 0, 0, 0};
#pragma unroll 1
      for (int n = 0; n < NB; ++n)
        if (OB::past(c0, a.nc, n, o))
          *(LDS i32x4*)(db + n * kThreads * 16) = i32x4{0, 0, 0, 0};
    };
    // Waits until this wavefront's pieces of tile kt have landed; `newer`: the
    // tile after it is there, and A's part of it (kRingB > 2: and B's) has
    // been asked for since.
    auto ready = [&](unsigned kt, bool newer) {
      if (kt >= k1) return;
      if (newer)
        asm volatile("s_waitcnt vmcnt(%0)"
                     :: "n"(kRingB > 2 ? NA + NB : NA) : "memory");
      else
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      clear(kt);
    };
    auto change = [] {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      meet();
      __builtin_amdgcn_sched_barrier(0);
    };

    auto loop = [&](auto with_sums) {
      int sa = 0, sb = 0;
#pragma unroll 1
      for (unsigned kt = k0; kt < k1; ++kt) {
        LDS char* la = lds + sa * kSlotA;
        LDS char* lb = ringb + sb * kSlotB;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
          i32x4 fa[MI], fb[NJ];
#pragma unroll
          for (int n = 0; n < NJ; ++n)
            fb[n] = OB::frag(lb, ks, kGated ? (n < NT ? 0 : BJ) + wn * (WN / 2)
                                            : wn * WN, n % NT, lane);
#pragma unroll
          for (int m = 0; m < MI; ++m)
            fa[m] = OA::frag(la, ks, wm * WM + m * 16, 0, lane);
          if (ks == 0) {
            // the slot of tile kt - 1, which both halves have read
            constexpr int on = kRingB - 1;
            if (kt + on < k1) ask_b(sb == 0 ? on : sb - 1);
          } else {
            if (kt + 2 < k1) ask_a(sa == 0 ? 2 : sa - 1);
            if (late) ready(kt + 1, kt + 2 < k1);
          }
          __builtin_amdgcn_sched_barrier(0);
          change();
          __builtin_amdgcn_s_setprio(1);
#pragma unroll
          for (int m = 0; m < MI; ++m) {
            mma_row<T>(fb, fa[m], acc[m]);
            if constexpr (with_sums) sum.template add<T>(m, wn, fa[m]);
          }
          __builtin_amdgcn_s_setprio(0);
          __builtin_amdgcn_sched_barrier(0);
          if (ks == 1 && !late) ready(kt + 1, kt + 2 < k1);
          change();
        }
        sa = sa + 1 == kRingA ? 0 : sa + 1;
        sb = sb + 1 == kRingB ? 0 : sb + 1;
      }
    };

    if (k0 < k1) {
      ask_a(0);
      ask_b(0);
      if (k0 + 1 < k1) {
        if (kRingB > 2) ask_b(1);
        ask_a(1);
      }
      ready(k0, k0 + 1 < k1);
      change();
      if (late) meet();   // one phase behind
      if constexpr (SUMS) {
        if (sums)
          loop(Yes{});
        else
          loop(No{});
      } else {
        loop(No{});
      }
      if (!late) meet();
    }
    Results<T, F, SUMS, WM, WN, kAcross, OB>::store(
        a, rank, pair, split, i0 + wm * WM,
        j0 + wn * (kGated ? WN / 2 : WN), sums, wn, sum, acc, lds, wave, lane);
    if constexpr (F == Form::DW && !SUMS)
      join_sums<T, BM>(a, rank, pair, split, i0, j0);
  }
};

template <Type T, Form F, bool SUMS, int BN>
__global__ __launch_bounds__(512) void k_pingpong(Args) {
  Given& a = *(Given*)__builtin_amdgcn_kernarg_segment_ptr();
  extern __shared__ char lds[];
  PingPong<T, F, SUMS, BN>::run(a, (LDS char*)lds);
}

template <Type T, Form F, bool SUMS, bool FAST, int BM, int BN, int WM, int WN,
          int R>
__global__ __launch_bounds__((BM / WM) * (BN / WN) * 64) void k_tiled(Args) {
  Given& a = *(Given*)__builtin_amdgcn_kernarg_segment_ptr();
  extern __shared__ char lds[];
  Tiled<T, F, SUMS, FAST, BM, BN, WM, WN, R>::run(a, (LDS char*)lds);
}

// ---------------------------------------------------------------- few rows

// Few rows of x (MT tiles of 16), bound by one read of the weights: a wavefront
// takes NW x 16 rows of w (GATED: half of them of each) and one of S parts of
// the contraction, straight from memory to the matrix cores' registers, U steps
// of loads at a time; the workgroup's S wavefronts join their sums in LDS, in
// order.  Every weight is read once, by all lanes of a wavefront side by side
// (64 bytes of 16 rows a load); x is small and comes from the caches.  Runs
// what FewFast cannot: operands off 16 bytes.
template <Type T, Form F, bool FAST, int MT, int NW, int S>
struct Few {
  using V = typename Elem<T>::V;
  static constexpr int E = 16 / sizeof(V), K = 4 * E;   // per piece, per step
  static constexpr bool kGated = F == Form::GATED;
  static constexpr int BJ = kGated ? 8 * NW : 16 * NW;
  static constexpr int U = MT * NW <= 2 ? 8 : 4;

  static __device__ void run(Given& a, LDS char* lds) {
    const int t = threadIdx.x, lane = t & 63, wave = uniform(t >> 6);
    const int r = lane & 15, q = lane >> 4;
    const unsigned nt = (unsigned)((a.nj + BJ - 1) / BJ);
    const unsigned rank = uniform(blockIdx.x / nt);
    const size_t j0 = (size_t)uniform(blockIdx.x % nt) * BJ;
    const unsigned steps = (unsigned)((a.nc + K - 1) / K);
    const unsigned s0 = (unsigned)((uint64_t)steps * wave / S),
                   s1 = (unsigned)((uint64_t)steps * (wave + 1) / S);
    const V* w[NW];
    const V* x[MT];
#pragma unroll
    for (int n = 0; n < NW; ++n) {
      size_t j = j0 + (kGated ? n / 2 : n) * 16 + r;
      if (j >= a.nj) j = a.nj - 1;
      w[n] = (const V*)a.b[kGated ? n % 2 : 0][rank] + j * a.ldb + q * E;
    }
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      size_t i = m * 16 + r;
      if (i >= a.ni) i = a.ni - 1;
      x[m] = (const V*)a.a[0][rank] + i * a.lda + q * E;
    }
    f32x4 acc[MT][NW] = {};
    unsigned s = s0;
    const unsigned full = (unsigned)(a.nc / K) < s1 ? (unsigned)(a.nc / K) : s1;
#pragma unroll 1
    for (; s + U <= full; s += U) {
      i32x4 fw[U][NW], fx[U][MT];
#pragma unroll
      for (int k = 0; k < U; ++k) {
#pragma unroll
        for (int n = 0; n < NW; ++n)
          fw[k][n] = load_whole<FAST>(w[n] + (size_t)(s + k) * K);
#pragma unroll
        for (int m = 0; m < MT; ++m)
          fx[k][m] = load_whole<FAST>(x[m] + (size_t)(s + k) * K);
      }
#pragma unroll
      for (int k = 0; k < U; ++k)
#pragma unroll
        for (int n = 0; n < NW; ++n)
#pragma unroll
          for (int m = 0; m < MT; ++m)
            acc[m][n] = Elem<T>::mma(fw[k][n], fx[k][m], acc[m][n]);
    }
#pragma unroll 1
    for (; s < s1; ++s) {
      const long left = (long)a.nc - (long)s * K - q * E;
      i32x4 fw[NW], fx[MT];
#pragma unroll
      for (int n = 0; n < NW; ++n)
        fw[n] = load_piece<V>(w[n] + (size_t)s * K, left);
#pragma unroll
      for (int m = 0; m < MT; ++m)
        fx[m] = load_piece<V>(x[m] + (size_t)s * K, left);
#pragma unroll
      for (int n = 0; n < NW; ++n)
#pragma unroll
        for (int m = 0; m < MT; ++m)
          acc[m][n] = Elem<T>::mma(fw[n], fx[m], acc[m][n]);
    }
    finish_all(a, (f32x4(LDS*)[MT * NW][64])lds, acc, rank, j0, wave, lane);
  }

  // Adds the S wavefronts' sums in their order and finishes the results, by way
  // of LDS, so that the code that finishes a tile of results is there once.
  static __device__ void finish_all(Given& a, f32x4 (LDS* part)[MT * NW][64],
                                    f32x4 (&acc)[MT][NW], unsigned rank,
                                    size_t j0, int wave, int lane) {
    const int r = lane & 15, q = lane >> 4;
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int n = 0; n < NW; ++n) part[wave][m * NW + n][lane] = acc[m][n];
    if (S > 1)
      __syncthreads();
    else
      in_order();
    // result tile (m, n): wavefront tile % S
    constexpr int NO = kGated ? NW / 2 : NW, NS = kGated ? 2 : 1;
    with_exact<T>(a.out32, [&](auto exact) {
#pragma unroll 1
      for (int t = wave; t < MT * NO; t += S) {
        const int m = t / NO, n = t % NO, w = m * NW + n * NS;
        f32x4 v = part[0][w][lane], u = part[0][w + NS - 1][lane];
#pragma unroll
        for (int k = 1; k < S; ++k) {
          v += part[k][w][lane];
          if (kGated) u += part[k][w + 1][lane];
        }
        const size_t i = m * 16 + r, j = j0 + n * 16 + q * 4;
        if (i >= a.ni || j >= a.nj) continue;
        float va[4], ua[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) va[e] = v[e], ua[e] = u[e];
        float bias[2][4];
        fetch_bias<T, F, 4>(a, rank, j, bias);
        finish<T, F, exact.value, 4>(a, rank, 0, i, j, va, ua, bias);
      }
    });
  }
};

// The same with whole 16-byte pieces: the weights go to LDS in chunks of 16
// rows x 512 bytes, two rows of 512 bytes per load, which memory serves faster
// than 64 bytes of 16 rows (a copy of the loads alone: 6.5 against 5.9 TB/s
// at 268 MB); x goes to registers.  Each wavefront has two chunks of LDS of
// its own and needs no barrier: while it multiplies one chunk the next is on
// its way.  The NW sets of weight rows take turns and share x.  8 x 1 x 4096 x
// 2048 gated: 40.9 us, 6.6 TB/s (53.8 by way of registers); 48 x 4096 x 8192
// gated 28.9, of which x's loads are a third.
template <Type T, Form F, int MT, int NW, int S>
struct FewFast {
  using V = typename Elem<T>::V;
  using Old = Few<T, F, true, MT, NW, S>;
  static constexpr bool kGated = F == Form::GATED;
  static constexpr int BJ = Old::BJ, E = Old::E;
  static constexpr int kRow = 512, kChunk = 16 * kRow;
  static constexpr int KC = kRow / (int)sizeof(V);   // contraction per chunk
  static constexpr int U = kRow / 64;                // steps per chunk

  static __device__ void run(Given& a, LDS char* lds) {
    const int t = threadIdx.x, lane = t & 63, wave = uniform(t >> 6);
    const int r = lane & 15, q = lane >> 4;
    const unsigned nt = (unsigned)((a.nj + BJ - 1) / BJ);
    const unsigned rank = uniform(blockIdx.x / nt);
    const size_t j0 = (size_t)uniform(blockIdx.x % nt) * BJ;
    const unsigned chunks = (unsigned)((a.nc + KC - 1) / KC);
    const unsigned c0 = uniform((unsigned)((uint64_t)chunks * wave / S)),
                   c1 = uniform((unsigned)((uint64_t)chunks * (wave + 1) / S));
    // load h: rows 2 h, 2 h + 1; pieces exchanged by the row.  Rows past the
    // last give its last piece.
    const char* base[NW];
    uint32_t cap[NW], off[8];
    const int slot = lane & 31;
    auto set_row = [&](int n) {
      return j0 + (kGated ? n / 2 : n) * 16;
    };
#pragma unroll
    for (int n = 0; n < NW; ++n) {
      const size_t jn = set_row(n), first = jn < a.nj ? jn : a.nj - 1;
      const size_t most = a.nj - first - 1;
      base[n] = uniform((const char*)a.b[kGated ? n % 2 : 0][rank] +
                        first * a.ldb * sizeof(V));
      cap[n] = uniform((uint32_t)((most < 15 ? most : 15) * a.ldb *
                                  sizeof(V)) + kRow - 16);
    }
#pragma unroll
    for (int h = 0; h < 8; ++h) {
      const int row = h * 2 + (lane >> 5);
      off[h] = (uint32_t)(row * a.ldb * sizeof(V)) + (slot ^ (row & 7)) * 16;
    }
    const uint32_t mine = (uint32_t)(uintptr_t)lds + wave * (2 * kChunk);
    LDS char* const src = lds + wave * (2 * kChunk);
    const V* x[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      size_t i = m * 16 + r;
      if (i >= a.ni) i = a.ni - 1;
      x[m] = (const V*)a.a[0][rank] + i * a.lda + q * E;
    }
    auto issue = [&](unsigned c, int n, int buf) {
      const char* b = uniform(base[n] + (size_t)c * kRow);
      const uint32_t d = uniform(mine + buf * kChunk);
      if ((size_t)(c + 1) * KC <= a.nc) {
#pragma unroll
        for (int h = 0; h < 8; ++h)
          dma16_once(d + h * 1024, b, off[h] < cap[n] ? off[h] : cap[n]);
      } else {
        // the contraction's last chunk: zeros past its end
        const size_t left = a.nj - 1;
        int o = lane;
        asm volatile("" : "+v"(o));
#pragma unroll 1
        for (int h = 0; h < 8; ++h) {
          const int row = h * 2 + (o >> 5);
          size_t at = set_row(n) + row;
          if (at > left) at = left;
          const size_t k = (size_t)c * KC + (size_t)((o & 31) ^ (row & 7)) * E;
          dma16_at(uniform(d + h * 1024),
                   k < a.nc ? (const char*)((const V*)
                                  a.b[kGated ? n % 2 : 0][rank] + at * a.ldb +
                                  k)
                            : (const char*)&g_zero);
        }
      }
    };
    i32x4 fx[U][MT];
    auto load_x = [&](unsigned c) {
      if ((size_t)(c + 1) * KC <= a.nc) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int m = 0; m < MT; ++m)
            fx[u][m] = *(const i32x4*)(x[m] + (size_t)c * KC + u * 4 * E);
      } else {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int m = 0; m < MT; ++m) {
            const size_t k = (size_t)c * KC + u * 4 * E;
            fx[u][m] = k + q * E < a.nc ? *(const i32x4*)(x[m] + k)
                                        : i32x4{0, 0, 0, 0};
          }
      }
    };
    f32x4 acc[MT][NW] = {};
    if (c0 < c1) issue(c0, 0, 0);
    int buf = 0;
#pragma unroll 1
    for (unsigned c = c0; c < c1; ++c) {
      load_x(c);
#pragma unroll
      for (int n = 0; n < NW; ++n) {
        // (the wait also covers x)
        landed<0>();
        if (n + 1 < NW)
          issue(c, n + 1, buf ^ 1);
        else if (c + 1 < c1)
          issue(c + 1, 0, buf ^ 1);
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const i32x4 fw = *(LDS i32x4*)(src + buf * kChunk + r * kRow +
                                         (((u * 4 + q) ^ (r & 7)) * 16));
#pragma unroll
          for (int m = 0; m < MT; ++m)
            acc[m][n] = Elem<T>::mma(fw, fx[u][m], acc[m][n]);
        }
        buf ^= 1;
      }
    }
    // the parts meet in LDS where the chunks were
    if (S > 1) __syncthreads();
    Old::finish_all(a, (f32x4(LDS*)[MT * NW][64])lds, acc, rank, j0, wave,
                    lane);
  }
};

template <Type T, Form F, bool FAST, int MT, int NW, int S>
__global__ __launch_bounds__(S * 64) void k_few(Args) {
  Given& a = *(Given*)__builtin_amdgcn_kernarg_segment_ptr();
  extern __shared__ char lds[];
  if constexpr (FAST)
    FewFast<T, F, MT, NW, S>::run(a, (LDS char*)lds);
  else
    Few<T, F, FAST, MT, NW, S>::run(a, (LDS char*)lds);
}

// Joins the parts of a split contraction in their order and finishes: 4
// results per thread, bound by reading the parts (about 4 us more than their
// bytes at 2.3 TB/s, the writing of them included).
template <Type T, Form F>
__global__ __launch_bounds__(256) void k_join(Args) {
  Given& a = *(Given*)__builtin_amdgcn_kernarg_segment_ptr();
  using V = typename Elem<T>::V;
  const size_t per = (a.nj + 3) / 4;
  const size_t id = (size_t)blockIdx.x * 256 + threadIdx.x;
  const int np = F == Form::DW ? a.pairs : 1;
  const size_t all = per * a.ni * a.ranks * np;
  const size_t sz = a.ni * a.nj;
  constexpr int NP = F == Form::GATED ? 2 : 1;
  if (id < all) {
    const size_t j = id % per * 4, x = id / per;
    const size_t i = x % a.ni;
    const int pair = x / a.ni % np, rank = x / a.ni / np;
    const long left = (long)a.nj - (long)j;
    float v[4] = {}, u2[4] = {}, t[4];
    const size_t step = (size_t)a.ranks * np * NP * sz;
    const float* w = a.part + ((size_t)rank * np + pair) * NP * sz + i * a.nj
                     + j;
    for (int s = 0; s < a.splits; ++s, w += step) {
      fetch_vals<float, 4>(w, t, left, a.nj % 4 == 0);
      for (int k = 0; k < 4; ++k) v[k] += t[k];
      if (F == Form::GATED) {
        fetch_vals<float, 4>(w + sz, t, left, a.nj % 4 == 0);
        for (int k = 0; k < 4; ++k) u2[k] += t[k];
      }
    }
    float bias[2][4];
    fetch_bias<T, F, 4>(a, rank, j, bias);
    with_exact<T, acts(F)>(a.out32, [&](auto exact) {
      finish<T, F, exact.value, 4>(a, rank, pair, i, j, v, u2, bias);
    });
  }
  if (F == Form::DW) {
    const size_t n = (size_t)a.ranks * a.pairs * a.ni;
    if (a.sums && id < n &&
        a.u[id / a.ni % a.pairs][id / a.ni / a.pairs]) {
      const float* w = a.part +
                       (size_t)a.splits * a.ranks * a.pairs * sz + id;
      float s = 0.f;
      for (int k = 0; k < a.splits; ++k) s += w[k * n];
      store_out<1>(a.u[id / a.ni % a.pairs][id / a.ni / a.pairs], id % a.ni,
                   &s, 1, a.out32, false, V());
    }
  }
}

// One piece's gradients before the activation: d (dy) becomes dz or dg, and o
// du; z and u: their places in the kept values.
template <bool GATED, bool EXACT, int E, typename V>
__device__ inline void slopes(int act, const V* z, const V* u, long left,
                              bool wide, float (&d)[E], float (&o)[E]) {
  float s[E], g[E];
  fetch_vals<V, E>(z, g, left, wide);
  if (GATED) fetch_vals<V, E>(u, s, left, wide);
  with_act(act, [&](auto a) {
#pragma unroll
    for (int k = 0; k < E; ++k) {
      float v;
      const float c = slope_of<a.value, EXACT>(g[k], &v);
      if (GATED) {
        o[k] = d[k] * v;
        d[k] = d[k] * s[k] * c;
      } else {
        d[k] *= c;
      }
    }
  });
}

// The gradients before the activation: 16 bytes of a row per thread and turn,
// bound by memory (5 x 8 x 2048 x 2048 bf16: 70 us, 4.8 TB/s, the rate of a
// copy).  Kept apart from the products that read them, each value several
// times: there the slope would be computed as often.  Rounded to the operands'
// type, which the matrix cores take: 16-bit gradients are 2.4e-3 (bf16) off for
// it, 1.7e-3 with the results' rounding alone.  As two 16-bit halves nothing
// would be lost, at twice the operations (4096 x 4096 x 4096: dx 118 -> 188 us,
// dw 107 -> 207).
template <Type T, bool GATED>
__global__ __launch_bounds__(256) void k_slope(SlopeArgs) {
  GivenSlope& a = *(GivenSlope*)__builtin_amdgcn_kernarg_segment_ptr();
  using V = typename Elem<T>::V;
  constexpr int E = 16 / sizeof(V);
  const int rank = blockIdx.y;
  const size_t per = (a.cols + E - 1) / E, all = per * a.rows;
  const V* dy = (const V*)a.dy[rank];
  const V* z = (const V*)a.z[rank];
  const V* u = GATED ? (const V*)a.u[rank] : nullptr;
  V* dz = (V*)a.dz[rank];
  V* du = GATED ? (V*)a.du[rank] : nullptr;
  for (size_t id = (size_t)blockIdx.x * 256 + threadIdx.x; id < all;
       id += (size_t)gridDim.x * 256) {
    const size_t i = id / per, j = id % per * E;
    const long left = (long)a.cols - (long)j;
    float d[E], o[E];
    fetch_vals<V, E>(dy + i * a.ldy + j, d, left, a.wide);
    slopes<GATED, T == Type::F32, E, V>(
        a.act, z + i * a.ldz + j, GATED ? u + i * a.ldz + j : nullptr, left,
        a.wide, d, o);
    store_vals<V, E>(dz + i * a.ldz + j, d, left, a.wide);
    if (GATED) store_vals<V, E>(du + i * a.ldz + j, o, left, a.wide);
  }
}

// The same with the bias gradients of 16-bit types, the sums over the rows of
// the values before they are rounded to 16 bits.  (The products read the
// rounded ones, and so would sums made beside them on the matrix cores, as DW
// does for 32-bit values and for dy itself: 16-bit bias gradients would be
// sqrt 2 times as far off, 32-bit ones 2^-9.)  A workgroup takes 128 bytes of
// the columns of a part of the rows, 64 rows at a time; a column's values meet
// in an order that its place alone fixes, and columns never meet.  4096 x 4096
// bf16, 8 parts: 25 us (k_slope 20); bound by memory.
template <Type T, bool GATED>
__global__ __launch_bounds__(kSumThreads) void k_sums(SumArgs) {
  GivenSums& a = *(GivenSums*)__builtin_amdgcn_kernarg_segment_ptr();
  using V = typename Elem<T>::V;
  constexpr int E = 16 / sizeof(V), kLanes = kSumLine / 16, kCols = E * kLanes,
                NP = GATED ? 2 : 1, kWaves = kSumThreads / 64;
  __shared__ float lds[kWaves][NP][kCols];
  const int t = threadIdx.x, lane = t & 63, rank = blockIdx.y;
  const bool wide = a.s.wide;
  const size_t strips = (a.s.cols + kCols - 1) / kCols;
  for (size_t id = blockIdx.x; id < strips * a.parts; id += gridDim.x) {
    const size_t strip = id % strips, part = id / strips;
    const size_t i1 = a.s.rows * (part + 1) / a.parts;
    const size_t j = strip * kCols + t % kLanes * E;
    const long left = (long)a.s.cols - (long)j;
    const V* dy = (const V*)a.s.dy[rank] + j;
    const V* z = (const V*)a.s.z[rank] + j;
    const V* u = GATED ? (const V*)a.s.u[rank] + j : nullptr;
    V* dz = (V*)a.s.dz[rank] + j;
    V* du = GATED ? (V*)a.s.du[rank] + j : nullptr;
    float sum[NP][E] = {};
    with_exact<T>(a.out32, [&](auto exact) {
      if (left <= 0) return;
      for (size_t i = a.s.rows * part / a.parts + t / kLanes; i < i1;
           i += kSumThreads / kLanes) {
        float d[E], o[E];
        fetch_vals<V, E>(dy + i * a.s.ldy, d, left, wide);
        slopes<GATED, exact.value, E, V>(a.s.act, z + i * a.s.ldz,
                                         GATED ? u + i * a.s.ldz : nullptr,
                                         left, wide, d, o);
        store_vals<V, E>(dz + i * a.s.ldz, d, left, wide);
        if (GATED) store_vals<V, E>(du + i * a.s.ldz, o, left, wide);
#pragma unroll
        for (int k = 0; k < E; ++k) {
          sum[0][k] += d[k];
          if (GATED) sum[NP - 1][k] += o[k];
        }
      }
    });
#pragma unroll
    for (int p = 0; p < NP; ++p)
#pragma unroll
      for (int k = 0; k < E; ++k) {
        float v = sum[p][k];
#pragma unroll
        for (int far = kLanes; far < 64; far *= 2) v += __shfl_xor(v, far);
        if (lane < kLanes) lds[t / 64][p][lane * E + k] = v;
      }
    __syncthreads();
    const int p = t / kCols;
    const size_t col = strip * kCols + t % kCols;
    if (p < NP && col < a.s.cols) {
      float v = 0.f;
      for (int w = 0; w < kWaves; ++w) v += lds[w][p][t % kCols];
      if (a.parts == 1)
        store_out<1>(a.db[p][rank], col, &v, 1, a.out32, false, V());
      else
        a.part[((part * a.all + a.first + rank) * NP + p) * a.s.cols + col] =
            v;
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------- launches

// Launches K; more than 64 KB of LDS is asked for once per device.
template <void (*K)(Args)>
hipError_t launch_kernel(const Args& a, size_t groups, int threads,
                         size_t bytes, hipStream_t stream) {
  if (groups > 0x7fffffffu) return hipErrorInvalidConfiguration;
  if (bytes > 65536) {
    static std::atomic<uint64_t> asked{0};     // one bit per device
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    const uint64_t bit = dev < 64 ? (uint64_t)1 << dev : 0;
    if (!(asked.load(std::memory_order_relaxed) & bit)) {
      e = hipFuncSetAttribute((const void*)K,
                              hipFuncAttributeMaxDynamicSharedMemorySize,
                              (int)bytes);
      if (e != hipSuccess) return e;
      asked.fetch_or(bit, std::memory_order_relaxed);
    }
  }
  hipLaunchKernelGGL(K, dim3((unsigned)groups), dim3(threads), bytes, stream,
                     a);
  return hipGetLastError();
}

template <void (*K)(Args)>
hipError_t launch_tiles(Form f, const Args& a, int bm, int bj, int threads,
                        size_t bytes, hipStream_t stream) {
  const size_t tiles = (a.ni + bm - 1) / bm *
                       (a.nj ? (a.nj + bj - 1) / bj : 1);
  const size_t n = tiles * a.ranks * (f == Form::DW ? a.pairs : 1) * a.splits;
  if (n == 0) return hipSuccess;
  return launch_kernel<K>(a, n, threads, bytes, stream);
}

template <Type T, Form F, bool SUMS, bool FAST, int BM, int BN, int WM, int WN,
          int R>
hipError_t go(const Args& a, hipStream_t stream) {
  using K = Tiled<T, F, SUMS, FAST, BM, BN, WM, WN, R>;
  return launch_tiles<k_tiled<T, F, SUMS, FAST, BM, BN, WM, WN, R>>(
      F, a, BM, K::BJ, K::kThreads, R * K::kBytes, stream);
}

template <Type T, Form F, bool SUMS, int BN>
hipError_t go_pingpong(const Args& a, hipStream_t stream) {
  using K = PingPong<T, F, SUMS, BN>;
  return launch_tiles<k_pingpong<T, F, SUMS, BN>>(
      F, a, K::BM, K::BJ, K::kThreads, K::kLds, stream);
}

template <Type T, Form F, bool FAST, int MT, int NW, int S>
hipError_t go_few(const Args& a, hipStream_t stream) {
  using K = Few<T, F, FAST, MT, NW, S>;
  const size_t n = (a.nj + K::BJ - 1) / K::BJ * a.ranks;
  const size_t parts = (size_t)S * MT * NW * 1024;
  const size_t bytes =
      FAST ? std::max(parts, (size_t)S * 2 * FewFast<T, F, MT, NW, S>::kChunk)
           : parts;
  return launch_kernel<k_few<T, F, FAST, MT, NW, S>>(a, n, S * 64, bytes,
                                                     stream);
}

// Wavefronts: 8 only with the fewest sets of weight rows that a row count
// takes (more sets are for a workgroup per CU at least, and those get 4).
template <Type T, Form F, bool FAST, int MT, int NW>
hipError_t pick_waves(const Args& a, hipStream_t stream) {
  constexpr int kFewest = MT == 1 && F == Form::LINEAR ? 1 : 2;
  switch (a.waves) {
    case 1: return go_few<T, F, FAST, MT, NW, 1>(a, stream);
    case 2: return go_few<T, F, FAST, MT, NW, 2>(a, stream);
    case 4: return go_few<T, F, FAST, MT, NW, 4>(a, stream);
    case 8:
      if constexpr (NW == kFewest)
        return go_few<T, F, FAST, MT, NW, 8>(a, stream);
  }
  return hipErrorInvalidConfiguration;
}

// The kernels that the host's rule asks for: up to 16 rows one or two sets
// (GATED: of either weights), up to 32 two or four, beyond (16 bits) four.
template <Type T, Form F, bool FAST>
hipError_t pick_few(const Args& a, hipStream_t stream) {
  constexpr int kOne = F == Form::GATED ? 2 : 1;
  if (a.ni <= 16) {
    if (a.sets == kOne) return pick_waves<T, F, FAST, 1, kOne>(a, stream);
    if (a.sets == 2 * kOne)
      return pick_waves<T, F, FAST, 1, 2 * kOne>(a, stream);
  } else if (a.ni <= 32) {
    if (a.sets == 2) return pick_waves<T, F, FAST, 2, 2>(a, stream);
    if (a.sets == 4) return pick_waves<T, F, FAST, 2, 4>(a, stream);
  } else if constexpr (T != Type::F32) {
    if (a.sets == 4 && a.ni <= 48)
      return pick_waves<T, F, FAST, 3, 4>(a, stream);
    if (a.sets == 4 && a.ni <= 64)
      return pick_waves<T, F, FAST, 4, 4>(a, stream);
  }
  return hipErrorInvalidConfiguration;
}

template <Type T, Form F, bool SUMS, bool FAST>
hipError_t pick_tile(const Args& a, hipStream_t stream) {
  if constexpr (T != Type::F32 && FAST) {
    if (a.tile == 4) return go_pingpong<T, F, SUMS, 256>(a, stream);
    if (a.tile == 3) return go_pingpong<T, F, SUMS, 128>(a, stream);
  }
  if (a.tile == 2) return go<T, F, SUMS, FAST, 128, 128, 64, 64, 2>(a, stream);
  if constexpr (FAST)
    if (a.tile == 1) return go<T, F, SUMS, FAST, 64, 64, 32, 32, 4>(a, stream);
  return go<T, F, SUMS, FAST, 64, 64, 32, 32, 2>(a, stream);
}

template <Type T, Form F, bool FAST>
hipError_t pick(const Args& a, hipStream_t stream) {
  if constexpr (F == Form::LINEAR || F == Form::GATED)
    if (a.waves) return pick_few<T, F, FAST>(a, stream);
  // (the sums cost registers: without them 128 x 128 tiles of operands off 16
  // bytes run two to a CU)
  if constexpr (F == Form::DW)
    if (a.sums) return pick_tile<T, F, true, FAST>(a, stream);
  return pick_tile<T, F, false, FAST>(a, stream);
}

template <Type T, Form F>
hipError_t run_form(const Args& a, hipStream_t stream) {
  const hipError_t e = a.fast ? pick<T, F, true>(a, stream)
                              : pick<T, F, false>(a, stream);
  if (e != hipSuccess || a.splits == 1) return e;
  const size_t n = (a.nj + 3) / 4 * a.ni * a.ranks *
                   (F == Form::DW ? a.pairs : 1);
  hipLaunchKernelGGL((k_join<T, F>), dim3((unsigned)((n + 255) / 256)),
                     dim3(256), 0, stream, a);
  return hipGetLastError();
}

template <Type T>
hipError_t run_type(Form f, const Args& a, hipStream_t stream) {
  switch (f) {
    case Form::LINEAR: return run_form<T, Form::LINEAR>(a, stream);
    case Form::GATED: return run_form<T, Form::GATED>(a, stream);
    case Form::DX: return run_form<T, Form::DX>(a, stream);
    default: return run_form<T, Form::DW>(a, stream);
  }
}

template <Type T>
hipError_t run_slope(const SlopeArgs& a, hipStream_t stream) {
  constexpr int E = 16 / sizeof(typename Elem<T>::V);
  const size_t n = (a.cols + E - 1) / E * a.rows;
  const size_t blocks = (n + 255) / 256;
  const dim3 grid((unsigned)(blocks < 4096 ? blocks : 4096), a.ranks);
  if (a.gated)
    hipLaunchKernelGGL((k_slope<T, true>), grid, dim3(256), 0, stream, a);
  else
    hipLaunchKernelGGL((k_slope<T, false>), grid, dim3(256), 0, stream, a);
  return hipGetLastError();
}

template <Type T>
hipError_t run_sums(const SumArgs& a, hipStream_t stream) {
  constexpr size_t kCols = kSumLine / sizeof(typename Elem<T>::V);
  const size_t strips = (a.s.cols + kCols - 1) / kCols;
  const dim3 grid((unsigned)std::min<size_t>(strips * a.parts, 1 << 20),
                  a.s.ranks), threads(kSumThreads);
  if (a.s.gated)
    hipLaunchKernelGGL((k_sums<T, true>), grid, threads, 0, stream, a);
  else
    hipLaunchKernelGGL((k_sums<T, false>), grid, threads, 0, stream, a);
  return hipGetLastError();
}

}  // namespace
}  // namespace products
}  // namespace dpar
