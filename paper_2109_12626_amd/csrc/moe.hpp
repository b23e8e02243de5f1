// Interface between the C entry point of the mixture-of-experts layer and its
// kernels.
#pragma once

#include "products.hpp"

namespace dpar {
namespace moe {

using products::Act;
using products::Type;

enum class Route : int { SOFTMAX = 0, SIGMOID = 1 };
// How the projections' launch knows who chose what: from a launch of the choice;
// every workgroup by itself; every workgroup for its own expert.
enum class Mode : int { TABLE = 0, FUSED = 1, DIRECT = 2 };

// Hidden values between the products: 32-bit ones as the second product takes
// them (fp32), 32-bit ones that its kernels split into three 16-bit parts, or
// these parts.
enum class Hidden : int { WHOLE = 1, VALUES = 2, PARTS = 3 };

// Ranks of a launch, as in products.hpp: 12 arrays of 32 addresses.
constexpr int kRanks = 32;
constexpr int kTokens = 128, kTop = 16, kExperts = 1024;
constexpr int kDirect = 256;   // experts of Mode::DIRECT
constexpr int kSmall = 8;      // tokens of the kernels for the fewest
// Sets of 16 columns of a workgroup of up, which share the activations: as many
// as let those be half of the loads (8-bit weights are half the bytes), and as
// the registers have sums for (shift: rows off 16 bytes, which need some too; with
// 8-bit weights and two tiles 192 bytes per lane are in scratch memory all the same:
// 64 tokens, 2 of 8 experts 4097 x 8191 395 us, 4096 x 8192 177).
constexpr int columns_up(Type w, bool fused, bool shift, int tiles) {
  if (fused) return 1;
  const int n = w != Type::I8 ? tiles : tiles < 4 ? 2 * tiles : 2;
  return shift && n > 2 ? 2 : n;
}

// An expert that some token chose: its rank of the launch, its number there, and
// its list of pairs (token, place among the token's choices).
struct Record {
  int rank, expert, first, count;
};

// A table of the workspace: how many records there are and which is each rank's
// first (`kStarts` numbers; not with Mode::DIRECT), the records in the experts'
// order, the pairs by expert, every pair's weight and owner (expert of the rank *
// kRanks + rank; -1: none of the launch), and its hidden values and result.  Ranks that choose from the same logits
// (or by the same index and weight) share one table, others have one each.
constexpr int kStarts = kRanks + 2;
struct Layout {
  size_t records, pairs, weights, owner, hidden, parts, bytes;
};

struct Args {
  const void* x[kRanks];
  const float* logits[kRanks];
  const void* w[3][kRanks];      // gate, up, down
  const float* s[3][kRanks];     // 8-bit weights: their scales
  const void* r[kRanks];         // residual
  void* y[kRanks];
  int* index[kRanks];
  float* weight[kRanks];
  size_t in, hidden;
  size_t ldx, ldl, ldw, ldd, xw, xd, ldy, ldr;   // as in dpar_moe_t
  size_t pitch;                  // of the pairs' results
  char* work;
  Layout at;
  float scale;
  int tokens, experts, top;
  int ranks, first, all;         // of the launch, its first, of the call
  int tables;                    // 1, or one for each rank
  int act, route, normalize;
  int given;                     // index and weight are inputs
  int out32;
  int planes;                    // how hidden values are held (Hidden)
  int most;                      // records of a table at most
  int waves[2];                  // wavefronts per workgroup: up, down
  int fast[2];                   // up, down: weights of whole 16-byte pieces
  int tiles[2];                  // up, down: pairs at a time / 16
  int sets;                      // of 16 columns, of a workgroup of down
  int mode;                      // how up knows the choice (Mode)
  int small;                     // down sums by token itself
};
static_assert(sizeof(Args) <= 4096, "kernel arguments");

// The choice of experts (Mode::TABLE), then the products (eight: 8-bit
// weights).
hipError_t launch_route(const Args& a, hipStream_t stream);
hipError_t launch_bf16(bool eight, const Args& a, hipStream_t stream);
hipError_t launch_f16(bool eight, const Args& a, hipStream_t stream);
hipError_t launch_f32(const Args& a, hipStream_t stream);

}  // namespace moe
}  // namespace dpar
