// Interface between the C entry point of the mixture-of-experts layer and its
// kernels.
#pragma once

#include "products.hpp"

namespace dpar {
namespace moe {

using products::Act;
using products::Type;

enum class Route : int { SOFTMAX = 0, SIGMOID = 1 };

// Ranks of a launch, as in products.hpp: 12 arrays of 32 addresses.
constexpr int kRanks = 32;
constexpr int kTokens = 128, kTop = 16, kExperts = 1024;

// An expert that some token chose: its list of pairs (token, place among the
// token's choices) starts at `first`.
struct Record {
  int expert, first, count, pad;
};

// A rank's part of the workspace: the number of records, the records, the pairs
// by expert and their weights, whether a pair is the rank's, and the hidden
// values and the result of every pair.
struct Layout {
  size_t records, pairs, weights, owned, hidden, parts, bytes;
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
  int act, route, normalize;
  int given;                     // index and weight are inputs
  int out32;
  int planes;                    // 16-bit parts of a hidden value
  int most;                      // experts of a rank that can be chosen
  int waves[2];                  // wavefronts per workgroup: up, down
  int fast[2];                   // up, down: weights of whole 16-byte pieces
};
static_assert(sizeof(Args) <= 4096, "kernel arguments");

// The choice of experts, then the products (eight: 8-bit weights).
hipError_t launch_route(const Args& a, hipStream_t stream);
hipError_t launch_bf16(bool eight, const Args& a, hipStream_t stream);
hipError_t launch_f16(bool eight, const Args& a, hipStream_t stream);
hipError_t launch_f32(const Args& a, hipStream_t stream);

}  // namespace moe
}  // namespace dpar
