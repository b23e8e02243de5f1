// Interface between the C entry points of the layer products and their
// kernels.
#pragma once

#include <hip/hip_runtime_api.h>

#include <cstddef>
#include <cstdint>

namespace dpar {
namespace products {

// Element types (values of dpar_dtype_t).
enum class Type : int { F32 = 1, BF16 = 3, F16 = 4, I8 = 5 };
// Activations (values of dpar_act_t).
enum class Act : int { NONE = 0, RELU = 1, GELU = 2, GELU_TANH = 3, SILU = 4 };

// One launch covers up to this many ranks: their addresses travel in the
// kernel arguments (10 arrays of 48 addresses, 3.8 KB of the 4 KB a launch
// takes), so a call stages nothing, allocates nothing and can be captured.
constexpr int kRanks = 48;

// C[i][j] = sum over c of A(i, c) B(j, c), for every rank of a launch.
//   LINEAR  A = x[i][c],  B = w[j][c];        C = act(.. + bias) + residual
//   GATED   A = x[i][c],  B = wg, wu[j][c];   C = act(g) * u
//   DX      A = dz[i][c], B = w[c][j], one or two pairs summed
//   DW      A = dz[c][i], B = x[c][j]; with two pairs two results, and the
//           sums of A over c (bias gradients, unless SumArgs has them)
enum class Form : int { LINEAR = 0, GATED = 1, DX = 2, DW = 3 };

struct Args {
  const void* a[2][kRanks];
  const void* b[2][kRanks];
  // LINEAR: bias, residual; GATED: bias of g, of u
  const void* e[2][kRanks];
  // LINEAR: y, z; GATED: h, g (u is in `u`); DX: dx; DW: dw, dw of u
  void* o[2][kRanks];
  // GATED: u; DW: bias gradients (sums)
  void* u[2][kRanks];
  // I8: the scales of A's rows are in a[1], of B's in u[0] (GATED: wg's) and
  // u[1] (wu's); nothing is kept
  size_t ni, nj, nc;         // rows and columns of C, contraction
  size_t na, nb;             // rows (columns, where stored so) of A and B
                             // that loads may touch: ni, nj or more
  size_t lda, ldb, ldo, ldk, lde;  // row distances (elements): A, B, result,
                                   // kept values, residual
  float* part;               // partial results of a split contraction
  const float* sum;          // DW: parts of the bias gradients (SumArgs)
  int parts, all, first;     // as there
  int ranks, pairs;
  int act;
  int out32;                 // result in 32 bits
  int out_type;              // I8: type of result, bias and residual
  int sums;                  // DW: with the sums of A
  int splits;                // parts of the contraction
  int waves;                 // few rows: parts of the contraction per
                             // workgroup (0: tiles)
  int sets;                  // few rows: sets of 16 weight rows per wavefront
  int tile;                  // results per workgroup: 64 x 64 with two (0)
                             // or four (1) tiles in LDS, 128 x 128, 256 x
                             // 128, 256 x 256
  int fast;                  // A, B: 16-byte rows and whole 16-byte pieces
  int wide_out;              // results, kept values, residual, bias: 16-byte
                             // pieces
};

static_assert(sizeof(Args) <= 4096, "kernel arguments");

// dz = dy act'(z) (gated == 0), or dg = dy u act'(g), du = dy act(g).
struct SlopeArgs {
  const void* dy[kRanks];
  const void* z[kRanks];
  const void* u[kRanks];
  void* dz[kRanks];
  void* du[kRanks];
  size_t rows, cols, ldy, ldz;
  int ranks, act, gated, wide;
};

// The same with the bias gradients, sums over the rows (16-bit types).
struct SumArgs {
  SlopeArgs s;
  void* db[2][kRanks];
  float* part;               // parts of the sums, [part][rank][pair][column]
  int parts, all, first;     // parts of the rows; ranks of the call, and the
                             // launch's first
  int out32;
};
constexpr int kSumThreads = 512, kSumLine = 128;   // bytes of a row per
                                                   // workgroup

// Copies matrices to 16-byte rows `pitch` bytes apart, zeros after the values;
// sizes in 2-byte units (launch_copy_int8: in bytes).  Up to two matrices of either operand.
struct CopyArgs {
  struct Job {
    const void* from[kRanks];
    char* to;
    size_t rows, cols, ld, pitch;
    int mats;
  } job[4];
  int jobs;
};
hipError_t launch_copy(const CopyArgs& a, hipStream_t stream);

// One source file per type.
hipError_t launch_bf16(Form f, const Args& a, hipStream_t stream);
hipError_t launch_f16(Form f, const Args& a, hipStream_t stream);
hipError_t launch_f32(Form f, const Args& a, hipStream_t stream);
hipError_t launch_int8(Form f, const Args& a, hipStream_t stream);
hipError_t launch_copy_int8(const CopyArgs& a, hipStream_t stream);
hipError_t launch_slope_bf16(const SlopeArgs& a, hipStream_t stream);
hipError_t launch_slope_f16(const SlopeArgs& a, hipStream_t stream);
hipError_t launch_slope_f32(const SlopeArgs& a, hipStream_t stream);
hipError_t launch_sums_bf16(const SumArgs& a, hipStream_t stream);
hipError_t launch_sums_f16(const SumArgs& a, hipStream_t stream);

// Rows to 8 bits with a scale each.
struct QuantizeArgs {
  const void* x[kRanks];
  signed char* q[kRanks];
  float* scale[kRanks];
  size_t rows, cols, ldx, ldq;
  int ranks, type;
};
hipError_t launch_quantize(const QuantizeArgs& a, hipStream_t stream);

}  // namespace products
}  // namespace dpar
