// The mixture-of-experts layer: the choice of experts.
#include "moe_kernels.hpp"

namespace dpar {
namespace moe {
namespace {

constexpr int kRouteThreads = 1024;

// Floats in their order as unsigned numbers: -0 equals 0, NaN comes last.
__device__ inline uint32_t ordered(float v) {
  if (v != v) return 0xffffffffu;
  const uint32_t b = __builtin_bit_cast(uint32_t, v + 0.f);
  return b ^ (b >> 31 ? 0xffffffffu : 0x80000000u);
}
constexpr uint32_t kNever = 0x007fffffu;    // -inf

// Exchanges within a wavefront: `v` of the lane that CTRL names, 0 where there is
// none.
template <int CTRL>
__device__ inline uint32_t from_lane(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf,
                                               false);
}
// Four steps within 16 lanes, two across: the last lane has met all.
template <typename Fn>
__device__ inline uint32_t gather(uint32_t v, Fn join) {
  v = join(v, from_lane<0x111>(v));        // one lane up the row of 16
  v = join(v, from_lane<0x112>(v));
  v = join(v, from_lane<0x114>(v));
  v = join(v, from_lane<0x118>(v));
  v = join(v, from_lane<0x142>(v));        // a row's last to the next row
  v = join(v, from_lane<0x143>(v));        // the lower half's to the upper
  return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}
__device__ inline uint32_t wave_max(uint32_t v) {
  return gather(v, [](uint32_t x, uint32_t y) { return x > y ? x : y; });
}
__device__ inline float wave_sum(float v) {
  return __builtin_bit_cast(
      float, gather(__builtin_bit_cast(uint32_t, v), [](uint32_t x, uint32_t y) {
        return __builtin_bit_cast(uint32_t, __builtin_bit_cast(float, x) +
                                                __builtin_bit_cast(float, y));
      }));
}

// One token's choice by a wavefront: lane i < top ends with its i-th expert
// (-1: none) and weight.
__device__ inline void choose(GivenMoe& a, const float* logits, int experts,
                              int lane, int* index, float* weight) {
  constexpr int N = kExperts / 64;
  uint32_t key[N];
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int e = n * 64 + lane;
    key[n] = 0;
    if (n * 64 < experts && e < experts) key[n] = ordered(logits[e]);
  }
  int mine = -1;
  for (int i = 0; i < a.top; ++i) {
    uint32_t best = 0;
#pragma unroll
    for (int n = 0; n < N; ++n)
      if (n * 64 < experts) best = key[n] > best ? key[n] : best;
    best = wave_max(best);
    if (best <= kNever) break;
    // the lowest expert that has it
    int found = -1;
#pragma unroll
    for (int n = 0; n < N; ++n)
      if (n * 64 < experts && found < 0) {
        const uint64_t has = __ballot(key[n] == best);
        if (has) {
          const int at = __builtin_ctzll(has);
          found = n * 64 + at;
          if (lane == at) key[n] = 0;
        }
      }
    if (lane == i) mine = found;
  }
  const float v = mine >= 0 ? logits[mine] : 0.f;
  float w = 0.f;
  if (a.route == (int)Route::SOFTMAX) {
    const float most = __shfl(v, 0);
    if (mine >= 0) w = expf(v - most);
    float sum;
    if (a.normalize) {
      sum = wave_sum(w);
    } else {
      sum = 0.f;
      for (int e = lane; e < experts; e += 64) sum += expf(logits[e] - most);
      sum = wave_sum(sum);
    }
    if (mine >= 0) w = w / sum;
  } else {
    if (mine >= 0) w = 1.f / (1.f + expf(-v));
    if (a.normalize) {
      const float sum = wave_sum(w);
      if (mine >= 0 && sum != 0.f) w = w / sum;
    }
  }
  *index = mine;
  *weight = w * a.scale;
}

// Every token's choice, and by expert the pairs of a rank's own ones: one
// workgroup per rank.  The order of an expert's pairs is not fixed and no result
// depends on it.
__global__ __launch_bounds__(kRouteThreads) void k_moe_route(MoeArgs) {
  GivenMoe& a = *(GivenMoe*)__builtin_amdgcn_kernarg_segment_ptr();
  __shared__ int expert[kTokens * kTop];
  __shared__ float share[kTokens * kTop];
  __shared__ unsigned short place[kTokens * kTop];
  __shared__ int count[kExperts], start[kExperts];
  const int t = threadIdx.x, lane = t & 63, wave = uniform(t >> 6);
  const int rank = blockIdx.x, top = a.top, pairs = a.tokens * top;
  const int all = a.experts * a.all, mine = a.experts * (a.first + rank);
  char* const work = work_of(a, rank);

  for (int e = t; e < a.experts; e += kRouteThreads) count[e] = 0;
  if (a.given) {
    for (int i = t; i < pairs; i += kRouteThreads) {
      const int e = a.index[rank][i];
      expert[i] = e >= 0 && e < all ? e : -1;
      share[i] = a.weight[rank][i];
    }
  } else {
    for (int k = wave; k < a.tokens; k += kRouteThreads / 64) {
      int e;
      float w;
      choose(a, a.logits[rank] + (size_t)k * a.ldl, all, lane, &e, &w);
      if (lane < top) {
        expert[k * top + lane] = e;
        share[k * top + lane] = w;
        if (a.index[rank]) a.index[rank][k * top + lane] = e;
        if (a.weight[rank]) a.weight[rank][k * top + lane] = w;
      }
    }
  }
  __syncthreads();
  if (a.given) {
    // an expert that a token names twice has one pair, with both weights
    for (int k = t; k < a.tokens; k += kRouteThreads)
      for (int i = 1; i < top; ++i)
        for (int j = 0; j < i; ++j)
          if (expert[k * top + i] >= 0 &&
              expert[k * top + i] == expert[k * top + j]) {
            share[k * top + j] += share[k * top + i];
            expert[k * top + i] = -1;
          }
    __syncthreads();
  }
  for (int i = t; i < pairs; i += kRouteThreads) {
    const int e = expert[i] - mine;
    if (expert[i] >= 0 && e >= 0 && e < a.experts)
      place[i] = (unsigned short)atomicAdd(&count[e], 1);
  }
  __syncthreads();
  if (wave == 0) {
    Record* const records = (Record*)(work + a.at.records);
    int before = 0, chosen = 0;
    for (int e0 = 0; e0 < a.experts; e0 += 64) {
      const int e = e0 + lane, n = e < a.experts ? count[e] : 0;
      int sum = n;
#pragma unroll
      for (int far = 1; far < 64; far *= 2) {
        const int o = __shfl_up(sum, far);
        if (lane >= far) sum += o;
      }
      const uint64_t some = __ballot(n > 0);
      const int first = before + sum - n;
      if (n > 0) {
        start[e] = first;
        const int at =
            chosen + __popcll(some & ((1ull << lane) - 1));
        records[at] = Record{e, first, n, 0};
      }
      before += __shfl(sum, 63);
      chosen += __popcll(some);
    }
    if (lane == 0) *(int*)work = chosen;
  }
  __syncthreads();
  int* const list = (int*)(work + a.at.pairs);
  float* const weights = (float*)(work + a.at.weights);
  int* const owned = (int*)(work + a.at.owned);
  for (int i = t; i < pairs; i += kRouteThreads) {
    const int e = expert[i] - mine;
    const bool own = expert[i] >= 0 && e >= 0 && e < a.experts;
    owned[i] = own;
    if (own) {
      const int at = start[e] + place[i];
      list[at] = i;
      weights[at] = share[i];
    }
  }
}

}  // namespace

hipError_t launch_route(const Args& a, hipStream_t stream) {
  hipLaunchKernelGGL(k_moe_route, dim3(a.ranks), dim3(kRouteThreads), 0,
                     stream, a);
  return hipGetLastError();
}

}  // namespace moe
}  // namespace dpar
