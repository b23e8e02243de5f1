// The mixture-of-experts layer for a few tokens on gfx950: the choice of
// experts, both gated projections of the chosen ones (up), and their second
// products (down) summed by token.  Reading the matrices of the chosen experts is
// what bounds the layer: 16 rows of a matrix at a time go to the matrix cores, the
// tokens that chose it are the columns, 16 to 64 at a time by an expert's mean share;
// an expert that has more takes further turns over its matrices.  Figures: one MI355X;
// every launch costs about 4 us beside it (its start and one wait for memory), so
// there are two for the fewest tokens and three or four else.
#pragma once

#include "moe.hpp"
#include "products_kernels.hpp"

namespace dpar {
namespace moe {
namespace {

using namespace products;
using MoeArgs = moe::Args;
using GivenMoe = const __attribute__((address_space(4))) MoeArgs;

__device__ inline char* table_of(GivenMoe& a, int table) {
  return a.work + (size_t)(a.first + table) * a.at.bytes;
}

// Who has a pair: a rank of the launch and its expert in one number.
__device__ inline int owner_of(int rank, int expert) {
  return expert * kRanks + rank;
}

// ---------------------------------------------------------------- the choice

// Floats in their order as unsigned numbers: -0 equals 0, NaN comes last.
__device__ inline uint32_t ordered(float v) {
  if (v != v) return 0xffffffffu;
  const uint32_t b = __builtin_bit_cast(uint32_t, v + 0.f);
  return b ^ (b >> 31 ? 0xffffffffu : 0x80000000u);
}
constexpr uint32_t kNever = 0x007fffffu;    // -inf
__device__ inline float as_value(uint32_t key) {
  return __builtin_bit_cast(float, key >> 31 ? key ^ 0x80000000u : ~key);
}

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

// Sums of the lanes up to each.
__device__ inline int wave_scan(int v) {
  v += (int)from_lane<0x111>((uint32_t)v);
  v += (int)from_lane<0x112>((uint32_t)v);
  v += (int)from_lane<0x114>((uint32_t)v);
  v += (int)from_lane<0x118>((uint32_t)v);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);
  return v;
}

// One token's choice by a wavefront, of at most 64 * N experts (value[n]: the
// lane's n-th logit): lane i < top ends with its i-th expert (-1: none) and
// weight.
template <int N>
__device__ inline void choose(GivenMoe& a, const float (&value)[N], int lane,
                              int* index, float* weight) {
  uint32_t key[N];
#pragma unroll
  for (int n = 0; n < N; ++n) key[n] = ordered(value[n]);
  int mine = -1;
  float v = 0.f, most = 0.f;
  for (int i = 0; i < a.top; ++i) {
    uint32_t best = key[0];
#pragma unroll
    for (int n = 1; n < N; ++n) best = key[n] > best ? key[n] : best;
    best = wave_max(best);
    if (best <= kNever) break;
    // the lowest expert that has it
    int found = -1;
#pragma unroll
    for (int n = 0; n < N; ++n)
      if (found < 0) {
        const uint64_t has = __ballot(key[n] == best);
        if (has) {
          const int at = __builtin_ctzll(has);
          found = n * 64 + at;
          if (lane == at) key[n] = 0;
        }
      }
    const float of = as_value(best);
    if (i == 0) most = of;
    if (lane == i) {
      mine = found;
      v = of;
    }
  }
  float w = 0.f;
  if (a.route == (int)Route::SOFTMAX) {
    if (mine >= 0) w = expf(v - most);
    float sum = w;
    if (!a.normalize) {
      sum = 0.f;
#pragma unroll
      for (int n = 0; n < N; ++n) sum += expf(value[n] - most);
    }
    sum = wave_sum(sum);
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

// The choice of every tokens-th one, f(token, index, weight) for each: the
// logits of B of them are on their way at a time.
template <int N, int B, typename Fn>
__device__ inline void choose_each(GivenMoe& a, const float* logits, int all,
                                   int first, int step, int lane, Fn f) {
  for (int k0 = first; k0 < a.tokens; k0 += B * step) {
    float value[B][N];
#pragma unroll
    for (int b = 0; b < B; ++b)
#pragma unroll
      for (int n = 0; n < N; ++n) {
        const int k = k0 + b * step, e = n * 64 + lane;
        value[b][n] = k < a.tokens && e < all
                          ? logits[(size_t)k * a.ldl + e]
                          : -__builtin_inff();
      }
#pragma unroll
    for (int b = 0; b < B; ++b)
      if (k0 + b * step < a.tokens) {
        int e;
        float w;
        choose<N>(a, value[b], lane, &e, &w);
        f(k0 + b * step, e, w);
      }
  }
}

// LDS of a workgroup that makes the choice.
struct Choice {
  LDS int* expert;           // of a pair
  LDS float* share;
  LDS int* place;            // among its expert's pairs
  LDS int* list;             // pairs by expert
  LDS int* count;            // of an expert's pairs, and the first of them
  LDS int* start;
  LDS Record* record;        // the one asked for
  LDS int* starts;           // as in the table

  static __host__ __device__ constexpr int bytes(int pairs, int experts) {
    return pairs * 16 + experts * 8 + (int)sizeof(Record) + kStarts * 4 + 8;
  }
  __device__ Choice(LDS char* lds, int pairs, int experts) {
    record = (LDS Record*)lds;
    expert = (LDS int*)(record + 1);
    share = (LDS float*)(expert + pairs);
    place = (LDS int*)(share + pairs);
    list = place + pairs;
    count = list + pairs;
    start = count + experts;
    starts = start + experts;
  }
};

// Every token's choice and, by expert, the pairs of a table's own ones, by a
// workgroup: into LDS, with the record `at`, and where asked to into the
// workspace and the index and weight arrays.  False if there are not so many
// records.  The order of an expert's pairs is not fixed, and no result depends
// on it.
template <int THREADS>
__device__ inline bool route(GivenMoe& a, int table, const Choice& c, int at,
                             bool write) {
  const int t = threadIdx.x, lane = t & 63, wave = uniform(t >> 6);
  const int top = a.top, pairs = a.tokens * top, all = a.experts * a.all;
  const bool one = a.tables == 1;
  // (the table's experts)
  const int low = a.experts * (a.first + (one ? 0 : table)),
            own = a.experts * (one ? a.ranks : 1);

  for (int e = t; e < own; e += THREADS) c.count[e] = 0;
  if (a.given) {
    for (int i = t; i < pairs; i += THREADS) {
      const int e = a.index[table][i];
      c.expert[i] = e >= 0 && e < all ? e : -1;
      c.share[i] = a.weight[table][i];
    }
  } else {
    auto keep = [&](int token, int e, float w) {
      if (lane >= top) return;
      const int i = token * top + lane;
      c.expert[i] = e;
      c.share[i] = w;
      if (write)
        for (int n = one ? 0 : table; n < (one ? a.ranks : table + 1); ++n) {
          if (a.index[n]) a.index[n][i] = e;
          if (a.weight[n]) a.weight[n][i] = w;
        }
    };
    const float* l = a.logits[table];
    constexpr int kStep = THREADS / 64;
    if (all <= 64)
      choose_each<1, 8>(a, l, all, wave, kStep, lane, keep);
    else if (all <= 256)
      choose_each<4, 4>(a, l, all, wave, kStep, lane, keep);
    else
      choose_each<kExperts / 64, 1>(a, l, all, wave, kStep, lane, keep);
  }
  __syncthreads();
  if (a.given) {
    // an expert that a token names twice has one pair, with both weights
    for (int k = t; k < a.tokens; k += THREADS)
      for (int i = 1; i < top; ++i)
        for (int j = 0; j < i; ++j)
          if (c.expert[k * top + i] >= 0 &&
              c.expert[k * top + i] == c.expert[k * top + j]) {
            c.share[k * top + j] += c.share[k * top + i];
            c.expert[k * top + i] = -1;
          }
    __syncthreads();
  }
  for (int i = t; i < pairs; i += THREADS) {
    const int e = c.expert[i] - low;
    if (c.expert[i] >= 0 && e >= 0 && e < own)
      c.place[i] = __hip_atomic_fetch_add(&c.count[e], 1, __ATOMIC_RELAXED,
                                          __HIP_MEMORY_SCOPE_WORKGROUP);
  }
  __syncthreads();
  char* const work = table_of(a, table);
  if (wave == 0) {
    Record* const records = (Record*)(work + a.at.records);
    int before = 0, chosen = 0;
    for (int e0 = 0; e0 < own; e0 += 64) {
      const int e = e0 + lane, n = e < own ? c.count[e] : 0;
      const int sum = wave_scan(n);
      const uint64_t some = __ballot(n > 0);
      const int first = before + sum - n;
      const int place = chosen + __popcll(some & ((1ull << lane) - 1));
      const int rank = (one ? 0 : table) + e / a.experts;
      if (e < own) {
        c.start[e] = first;
        if (e % a.experts == 0) c.starts[1 + rank] = place;
      }
      if (n > 0) {
        const Record r = {rank, e % a.experts, first, n};
        if (place == at) {
          c.record->rank = r.rank;
          c.record->expert = r.expert;
          c.record->first = r.first;
          c.record->count = r.count;
        }
        if (write) records[place] = r;
      }
      before += __builtin_amdgcn_readlane(sum, 63);
      chosen += __popcll(some);
    }
    if (lane == 0) {
      c.starts[0] = chosen;
      c.starts[1 + (one ? a.ranks : table + 1)] = chosen;
    }
  }
  __syncthreads();
  for (int i = t; i < pairs; i += THREADS) {
    const int e = c.expert[i] - low;
    const bool mine = c.expert[i] >= 0 && e >= 0 && e < own;
    if (mine) c.list[c.start[e] + c.place[i]] = i;
    if (!write) continue;
    ((int*)(work + a.at.owner))[i] =
        mine ? owner_of((one ? 0 : table) + e / a.experts, e % a.experts) : -1;
    if (mine) {
      ((int*)(work + a.at.pairs))[c.start[e] + c.place[i]] = i;
      ((float*)(work + a.at.weights))[i] = c.share[i];
    }
  }
  if (write)
    for (int i = t; i < kStarts; i += THREADS)
      if (i == 0 || (one ? i <= 1 + a.ranks
                         : i == 1 + table || i == 2 + table))
        ((int*)work)[i] = c.starts[i];
  __syncthreads();
  return at < c.starts[0];
}

// ---------------------------------------------------------------- types

typedef int i32x2 __attribute__((ext_vector_type(2)));

// Values as the upper halves of 32-bit floats, two of them in a register.
__device__ inline int upper_halves(float even, float odd) {
  return (int)__builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, odd),
                                    __builtin_bit_cast(uint32_t, even),
                                    0x07060302u);
}
__device__ inline float from_byte(int word, int k) {
  return (float)(signed char)(word >> (8 * k));
}

// Weights of type W beside activations of type X.  A step of the contraction is
// 16 bytes of weights per lane group, VB values, beside NX 16-byte pieces of
// activations: lane group q has E values of each run of 4 E, so that the four
// read 64 bytes of a row side by side.  (8 bits: two runs of 32 values.)
template <Type W, Type X> struct Mix {
  using V = typename Elem<W>::V;
  using XV = typename Elem<X>::V;
  static constexpr int VB = 16 / (int)sizeof(V), E = 16 / (int)sizeof(XV);
  static constexpr int NX = VB / E;
  // Bytes of a row in a chunk: 512, or 256 where the activations of that many,
  // `pieces` of each step, and `sums` take more than 160 registers, and for
  // SHIFT, which needs some for itself.
  static constexpr int row(int pieces, int sums, bool shift) {
    return shift || (pieces * 8 + sums) * 4 > 160 ? 256 : 512;
  }
  // Hidden values: 32-bit ones as they are, else three parts of 16 bits; their
  // pieces of a step, and those that come from memory (FORM: Hidden).
  static constexpr bool kWhole = X == Type::F32;
  static constexpr int kParts = kWhole ? 1 : 3 * VB / 8;
  static constexpr int pieces(int FORM) {
    return FORM == (int)Hidden::PARTS ? kParts : VB / 4;
  }

  static __device__ f32x4 up(i32x4 w, const i32x4 (&x)[NX], f32x4 c) {
    if constexpr (W != Type::I8) {
      return Elem<X>::mma(w, x[0], c);
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        i32x4 v;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int word = h * 2 + k / 2;
          const int bytes = w[word];
          const float even = from_byte(bytes, k % 2 * 2),
                      odd = from_byte(bytes, k % 2 * 2 + 1);
          if constexpr (X == Type::BF16) {
            v[k] = upper_halves(even, odd);
          } else {
            const auto two = __builtin_amdgcn_cvt_pkrtz(even, odd);
            v[k] = __builtin_bit_cast(int, two);
          }
        }
        c = Elem<X>::mma(v, x[h], c);
      }
      return c;
    }
  }

  // c += weights by hidden values, three parts of 8 values each: every weight as
  // one or two bfloat16 parts, which hold it exactly.
  static __device__ f32x4 down(i32x4 w, const i32x4 (&h)[kParts], f32x4 c) {
    constexpr int P = 3;
    if constexpr (kWhole) {
      return Elem<Type::F32>::mma(w, h[0], c);
    } else if constexpr (W == Type::BF16) {
#pragma unroll
      for (int p = 0; p < P; ++p) c = Elem<Type::BF16>::mma(w, h[p], c);
      return c;
    } else if constexpr (W == Type::F16) {
      const f16x8 f = __builtin_bit_cast(f16x8, w);
      i32x4 hi, lo;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float a = (float)f[2 * k], b = (float)f[2 * k + 1];
        const int both = upper_halves(a, b);
        hi[k] = both;
        const float ah = __builtin_bit_cast(float, both << 16),
                    bh = __builtin_bit_cast(float, both & (int)0xffff0000);
        lo[k] = upper_halves(a - ah, b - bh);
      }
#pragma unroll
      for (int p = 0; p < P; ++p) {
        c = Elem<Type::BF16>::mma(hi, h[p], c);
        c = Elem<Type::BF16>::mma(lo, h[p], c);
      }
      return c;
    } else {
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        i32x4 v;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int bytes = w[g * 2 + k / 2];
          v[k] = upper_halves(from_byte(bytes, k % 2 * 2),
                              from_byte(bytes, k % 2 * 2 + 1));
        }
#pragma unroll
        for (int p = 0; p < P; ++p)
          c = Elem<Type::BF16>::mma(v, h[g * P + p], c);
      }
      return c;
    }
  }
};

// Two 32-bit hidden values as three bfloat16 parts each: the upper half, the
// rest's upper half, and what is left, which together are the value.  (What an
// infinity leaves is NaN: whole_result().)
__device__ inline void split(float even, float odd, int (&part)[3]) {
  auto rest = [](float x) {
    return x - __builtin_bit_cast(
                   float, __builtin_bit_cast(uint32_t, x) & 0xffff0000u);
  };
  const float e1 = rest(even), o1 = rest(odd);
  part[0] = upper_halves(even, odd);
  part[1] = upper_halves(e1, o1);
  part[2] = upper_halves(rest(e1), rest(o1));
}

// ---------------------------------------------------------------- streams

// 16 rows of a matrix, `left` of them there, from memory to a wavefront's LDS in
// chunks of ROW bytes a row, pieces exchanged by the row (as FewFast does).
//
// SHIFT: rows that start anywhere and hold any number of values.  The pieces are
// those that lie on 16 bytes in memory, one more of a row than its chunk fills,
// and LDS is read from the row's own first byte on (33 tokens, 20 experts 1001 x
// 501 fp16, with a launch for the choice: 36 us; by way of registers 41).  A piece
// that holds a byte of the row is read whole; it lies in one page with that byte.
template <typename T, bool SHIFT> struct At { typedef T Type; };
template <typename T> struct At<T, true> {
  typedef T Type __attribute__((aligned(1)));
};
template <typename T, bool SHIFT>
using Anywhere = typename At<T, SHIFT>::Type;

template <typename V, int ROW, bool SHIFT>
struct Stream {
  static constexpr int VB = 16 / (int)sizeof(V), KC = ROW / (int)sizeof(V);
  static constexpr int kSteps = ROW / 64;
  static constexpr int kLanes = ROW / 16 + (SHIFT ? 1 : 0);    // of a row
  static constexpr int kPitch = kLanes * 16;
  static constexpr int kLoads = (16 * kLanes + 63) / 64;
  static constexpr int kChunk = kLoads * 1024, kRows = 64 / kLanes;
  // By what pieces are exchanged: the 16 rows' pieces read together lie in as many
  // banks (of rows of 128 bytes, two lie side by side across them).
  static __device__ int key(int row) {
    return kLanes < 16 ? row >> 1 & (kLanes - 1) : row & 15;
  }

  // Chunk c (of a contraction of nc values) of the rows from `base` on, as rows
  // FROM .. FROM + ROWS - 1 of the chunk.
  template <int FROM = 0, int ROWS = 16>
  static __device__ void ask(const char* base, size_t ld, int left, size_t nc,
                             unsigned c, uint32_t lds, int lane) {
    if constexpr (SHIFT) {
      constexpr int kPieces = ROWS * kLanes;
      const uint32_t low = (uint32_t)(uintptr_t)base & 15,
                     far = (uint32_t)(ld * sizeof(V)),
                     bytes = (uint32_t)(nc * sizeof(V));
      const char* b = uniform(base - low);
#pragma unroll
      for (int h = 0; h < (kPieces + 63) / 64; ++h) {
        const int n = h * 64 + lane, row = n / kLanes, piece = n % kLanes;
        // the row's first byte and its last piece; pieces past that are not
        // used, and it stands for them
        const uint32_t first = low + (row < left ? row : left - 1) * far,
                       last = (first + bytes - 1) & ~15u;
        const uint32_t at = (first & ~15u) + c * ROW + piece * 16;
        if (n < kPieces)
          dma16_once(uniform(lds + FROM * kPitch + h * 1024), b,
                     at < last ? at : last);
      }
    } else if ((size_t)(c + 1) * KC <= nc) {
      const int slot = lane % kLanes;
      const char* b = uniform(base + (size_t)c * ROW);
#pragma unroll
      for (int h = FROM / kRows; h < (FROM + ROWS) / kRows; ++h) {
        const int row = h * kRows + lane / kLanes;
        const int at = row - FROM < left ? row - FROM : left - 1;
        dma16_once(uniform(lds + h * 1024), b,
                   (uint32_t)(at * ld * sizeof(V)) + (slot ^ key(row)) * 16);
      }
    } else {
      // the last chunk: zeros past the contraction's end
      const int slot = lane % kLanes;
#pragma unroll 1
      for (int h = FROM / kRows; h < (FROM + ROWS) / kRows; ++h) {
        const int row = h * kRows + lane / kLanes;
        const int at = row - FROM < left ? row - FROM : left - 1;
        const size_t k = (size_t)c * KC + (size_t)(slot ^ key(row)) * VB;
        dma16_at(uniform(lds + h * 1024),
                 k < nc ? base + (at * ld + k) * sizeof(V)
                        : (const char*)&g_zero);
      }
    }
  }
  // Where row r of the rows from `base` on starts in its first piece.
  static __device__ int offset(const char* base, size_t ld, int left, int r) {
    if constexpr (!SHIFT) return 0;
    return (int)((uintptr_t)(base + (size_t)(r < left ? r : left - 1) * ld *
                                        sizeof(V)) &
                 15);
  }
  // Step u's values of row r for lane group q (Mix); off: offset(r); rest:
  // values from the chunk's first to the contraction's end (SHIFT: what lies
  // past it are another row's).
  static __device__ i32x4 take(LDS char* src, int u, int r, int q, int off,
                               int rest) {
    constexpr int kRuns = sizeof(V) == 1 ? 2 : 1, kBytes = 16 / kRuns;
    i32x4 v;
#pragma unroll
    for (int n = 0; n < kRuns; ++n) {
      const int at = u * 64 + n * 4 * kBytes + q * kBytes;
      LDS char* from =
          SHIFT ? src + r * kPitch + off + at
                : src + r * ROW + ((at / 16) ^ key(r)) * 16 + at % 16;
      if constexpr (kRuns == 1) {
        v = *(LDS Anywhere<i32x4, SHIFT>*)from;
      } else {
        const i32x2 half = *(LDS Anywhere<i32x2, SHIFT>*)from;
        v[n * 2] = half[0];
        v[n * 2 + 1] = half[1];
      }
      if (SHIFT && rest < KC) {
        const int bytes = rest * (int)sizeof(V) - at;
#pragma unroll
        for (int k = n * kBytes / 4; k < (n + 1) * kBytes / 4; ++k) {
          const int b = bytes - (k - n * kBytes / 4) * 4;
          v[k] = b >= 4 ? v[k] : b <= 0 ? 0 : v[k] & ((1 << (b * 8)) - 1);
        }
      }
    }
    return v;
  }
};

// After landed(): values that ordinary loads brought are taken as read here.
// Else the compiler, which does not know of that wait, waits for them at their
// first use, and there for everything asked for since.
template <int U, int N>
__device__ inline void arrived(i32x4 (&v)[U][N]) {
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int n = 0; n < N; ++n) asm volatile("" : "+v"(v[u][n]));
}

// Values from chunk c on, as far as the chunk.
template <typename St>
__device__ inline int rest_of(size_t nc, unsigned c) {
  const size_t left = nc - (size_t)c * St::KC;
  return left < (size_t)St::KC ? (int)left : St::KC;
}

// Waits until all but the last LEFT of this wavefront's loads have landed, and
// its LDS reads.
template <int LEFT>
__device__ inline void landed_but(bool all) {
  if (all)
    landed<0>();
  else
    landed<LEFT>();
}

// A wavefront's way through the chunks c0 .. c1 - 1 of NS sets of rows that share
// activations, with two buffers: load(c) loads a chunk's activations, ask(n, c,
// buffer) asks for set n's part, use(n, c, buffer) multiplies it.  Two parts are
// on their way whenever the wavefront waits: 16 KB, with 8 wavefronts 128 KB
// per CU.
template <int NS, int LOADS, typename Load, typename Pin, typename Ask,
          typename Use>
__device__ inline void sweep(unsigned c0, unsigned c1, Load load, Pin pin,
                             Ask ask, Use use) {
  static_assert(NS % 2 == 0);
#pragma unroll 1
  for (unsigned c = c0; c < c1; ++c) {
    load(c);
#pragma unroll
    for (int n = 0; n < NS; ++n) {
      if (n == 0) {
        landed<0>();                 // the activations, sets 0 and 1
        pin();
      } else if (n > 1) {
        landed_but<LOADS>(n + 1 == NS && c + 1 == c1);
      }
      use(n, c, n & 1);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if (n + 2 < NS)
        ask(n + 2, c, n & 1);
      else if (c + 1 < c1)
        ask(n + 2 - NS, c + 1, n & 1);
    }
  }
}

// The first `left` values at x, zeros behind them; 16 bytes before x + left are
// the row's too.
template <typename XV>
__device__ inline i32x4 load_tail(const XV* x, int left) {
  constexpr int E = 16 / (int)sizeof(XV);
  const int back = left < E ? left > 0 ? E - left : E : 0;
  uint64_t v[2];
  __builtin_memcpy(v, x + (left < E ? left - E : 0), 16);
  const int bits = back * (int)sizeof(XV) * 8;
  const uint64_t low =
      bits >= 64 ? v[1] >> (bits & 63)
                 : v[0] >> bits | (bits ? v[1] << (64 - bits) : 0);
  v[1] = bits >= 64 ? 0 : v[1] >> bits;
  v[0] = bits >= 128 ? 0 : low;
  i32x4 r;
  __builtin_memcpy(&r, v, 16);
  return r;
}

// NX pieces of a row of activations, of which `left` values are left (WHOLE: a
// multiple of a piece's; else the row has a piece at least), one of each run;
// rows may start anywhere.
template <bool WHOLE, typename XV, int NX>
__device__ inline void fetch_row(const XV* x, int left, i32x4 (&v)[NX]) {
  constexpr int E = 16 / (int)sizeof(XV);
#pragma unroll
  for (int n = 0; n < NX; ++n) {
    if constexpr (WHOLE)
      v[n] = n * 4 * E < left ? load_whole<false>(x + n * 4 * E)
                              : i32x4{0, 0, 0, 0};
    else
      v[n] = load_tail(x + n * 4 * E, left - n * 4 * E);
  }
}

// ---------------------------------------------------------------- gate and up

// What a workgroup of up or down works at: a chosen expert and its pairs.
struct Task {
  int rank, expert, count;
  const int* list;
  const float* weights;
  char* work;

  // The record `at` of a table; false if there are not so many.
  __device__ bool find(GivenMoe& a, int table, int at) {
    work = table_of(a, table);
    // (at < a.most: there is room for the record, whether it is one or not)
    const Record r = ((const Record*)(work + a.at.records))[at];
    if (at >= *(const int*)work) return false;
    rank = uniform(r.rank);
    expert = uniform(r.expert);
    count = uniform(r.count);
    list = (const int*)(work + a.at.pairs) + uniform(r.first);
    weights = (const float*)(work + a.at.weights);
    return count > 0;
  }
};

// A token's choice by a wavefront into a table's weights and owners, and where
// the choice is not an input into the index and weight arrays.
__device__ inline void keep_choice(GivenMoe& a, int table, int token,
                                   int lane) {
  const bool one = a.tables == 1;
  const int top = a.top, all = a.experts * a.all, i = token * top + lane;
  int e = -1;
  float w = 0.f;
  if (a.given) {
    if (lane < top) {
      e = a.index[table][i];
      w = a.weight[table][i];
      if (e < 0 || e >= all) e = -1;
    }
    // an expert named twice has one pair, the first, with both weights
    const int named = e;
    const float each = w;
    for (int k = 0; k < top; ++k) {
      const int other = __shfl(named, k);
      const float more = __shfl(each, k);
      if (named >= 0 && other == named) {
        if (k < lane) e = -1;
        if (k > lane) w += more;
      }
    }
  } else {
    const float* l = a.logits[table] + (size_t)token * a.ldl;
    float value[kDirect / 64];
#pragma unroll
    for (int n = 0; n < kDirect / 64; ++n)
      value[n] = n * 64 + lane < all ? l[n * 64 + lane] : -__builtin_inff();
    choose<kDirect / 64>(a, value, lane, &e, &w);
    if (lane < top)
      for (int n = one ? 0 : table; n < (one ? a.ranks : table + 1); ++n) {
        if (a.index[n]) a.index[n][i] = e;
        if (a.weight[n]) a.weight[n][i] = w;
      }
  }
  if (lane >= top) return;
  char* const work = table_of(a, table);
  const int low = a.experts * (a.first + (one ? 0 : table)),
            own = a.experts * (one ? a.ranks : 1);
  ((int*)(work + a.at.owner))[i] =
      e >= low && e < low + own
          ? owner_of((one ? 0 : table) + (e - low) / a.experts,
                     (e - low) % a.experts)
          : -1;
  ((float*)(work + a.at.weights))[i] = w;
}

// The pairs of one expert, in the order of the tokens, by a workgroup of S
// wavefronts into LDS (kDirectList numbers); how many.  A token's threads, as
// many as there are for each, count the experts that come before this one.
constexpr int kDirectList = 2 * kTokens + 4;
template <int S>
__device__ inline int chosen_by(GivenMoe& a, const Task& task, LDS int* list) {
  constexpr int kThreads = S * 64, kTurns = (kTokens + kThreads - 1) / kThreads;
  const int t = threadIdx.x, lane = t & 63, wave = uniform(t >> 6);
  const int all = a.experts * a.all,
            e = (a.first + task.rank) * a.experts + task.expert;
  LDS int* const before = list + kTokens;
  LDS int* const counts = before + kTokens;
  if (!a.given) {
    for (int i = t; i < kTokens; i += kThreads) before[i] = 0;
    __syncthreads();
    int places = 1;                    // (uniform)
    while (places < a.tokens) places *= 2;
    const int parts = places < kThreads ? kThreads / places : 1;
    for (int k0 = 0; k0 < a.tokens; k0 += kThreads) {
      const int token = k0 + t % places % kThreads, part = t / places;
      if (token < a.tokens) {
        const float* l = a.logits[task.rank] + (size_t)token * a.ldl;
        const uint32_t own = ordered(l[e]);
        int n = own <= kNever ? a.top : 0;
#pragma unroll 8
        for (int k = part; k < all; k += parts) {
          const uint32_t key = ordered(l[k]);
          n += key > own || (key == own && k < e);
        }
        if (n)
          __hip_atomic_fetch_add(&before[token], n, __ATOMIC_RELAXED,
                                 __HIP_MEMORY_SCOPE_WORKGROUP);
      }
    }
    __syncthreads();
  }
  int total = 0;
#pragma unroll
  for (int k = 0; k < kTurns; ++k) {
    const int token = k * kThreads + t;
    int place = -1;
    if (token < a.tokens) {
      if (a.given) {
        const int* index = a.index[task.rank] + (size_t)token * a.top;
        for (int i = a.top - 1; i >= 0; --i)
          if (index[i] == e) place = i;
      } else if (before[token] < a.top) {
        place = before[token];
      }
    }
    const uint64_t some = __ballot(place >= 0);
    if (lane == 0) counts[wave] = __popcll(some);
    __syncthreads();
    int from = total;
#pragma unroll
    for (int w = 0; w < S; ++w) {
      from += w < wave ? counts[w] : 0;
      total += counts[w];
    }
    if (place >= 0)
      list[from + __popcll(some & ((1ull << lane) - 1))] =
          token * a.top + place;
    __syncthreads();
  }
  return uniform(total);
}

// Distance of the hidden values' rows, in runs of 32, and the values that are
// written: whole tiles of 16 columns, zeros past the last one.
__device__ inline size_t runs_of(GivenMoe& a) { return (a.hidden + 31) / 32; }
__device__ inline size_t held_of(GivenMoe& a) {
  return (a.hidden + 15) / 16 * 16;
}

// h = act(g) * u of the pairs that chose an expert: a workgroup takes 16 * C
// columns (as many rows of either matrix) of one chosen expert, its S wavefronts
// a part of the contraction each; MT tiles of 16 pairs at a time.  Bound by the
// weights: 64 experts 2048 x 1024 bf16, 100 tokens 84 to 88 us for 537 MB (6.1 to
// 6.4 TB/s); 8-bit ones are as many loads of activations as of weights (8 experts
// 4096 x 8192, 64 tokens: 114 us with 16 columns, 101 with 32, 93 with 64).  Where
// the pairs come from (MODE):
//   TABLE   the choice's launch.
//   FUSED   every workgroup makes the choice for itself (few tokens), the first
//           one of a table keeps it.
//   DIRECT  (most experts are chosen) a workgroup belongs to an expert, asks for
//           its weights and, while they come, finds the tokens that chose it; for
//           the launches that follow the first workgroups make a token's choice
//           each, and those of the first columns keep their experts' pairs.
template <Type W, Type X, bool SHIFT, Mode MODE, int MT, int C, int S>
struct Up {
  using M = Mix<W, X>;
  using V = typename M::V;
  using XV = typename M::XV;
  using St = Stream<V, M::row(MT * M::NX, MT * C * 2, SHIFT), SHIFT>;
  static constexpr int VB = M::VB, NX = M::NX, K = 4 * VB;   // per step
  static constexpr int U = St::kSteps, KC = U * K, kChunk = St::kChunk;
  static constexpr int NS = 2 * C, BJ = 16 * C;
  static constexpr int kParts = S * MT * NS * 1024;
  static constexpr int kLds = std::max(S * 2 * kChunk, kParts);

  static __device__ void run(GivenMoe& a, LDS char* lds) {
    const int t = threadIdx.x, lane = t & 63, wave = uniform(t >> 6);
    const int r = lane & 15, q = lane >> 4;
    const unsigned tiles = (unsigned)((a.hidden + BJ - 1) / BJ);
    const unsigned id = uniform(blockIdx.x / tiles);
    const size_t j0 = (size_t)uniform(blockIdx.x % tiles) * BJ;
    const Choice choice(lds + kLds, a.tokens * a.top,
                        a.experts * (a.tables == 1 ? a.ranks : 1));
    // Asks for what follows the choice from the arguments, of rank 0 (and below
    // in down_small; one token 27.2 -> 26.6 us).
    if constexpr (MODE == Mode::FUSED)
      asm volatile("" ::"s"(a.w[0][0]), "s"(a.w[1][0]), "s"(a.x[0]),
                   "s"(a.ldx), "s"(a.xw), "s"(a.work), "s"(a.act),
                   "s"(a.at.hidden), "s"(a.s[0][0]), "s"(a.s[1][0]));
    Task task;
    if constexpr (MODE == Mode::DIRECT) {
      task.rank = uniform(id / a.experts);
      task.expert = uniform(id % a.experts);
      task.work = table_of(a, a.tables == 1 ? 0 : task.rank);
    } else {
      const int table = uniform(id / a.most), at = uniform(id % a.most);
      if constexpr (MODE == Mode::FUSED) {
        if (!route<S * 64>(a, table, choice, at, at == 0 && j0 == 0)) return;
        task.rank = uniform(choice.record->rank);
        task.expert = uniform(choice.record->expert);
        task.count = uniform(choice.record->count);
        task.work = table_of(a, table);
      } else {
        if (!task.find(a, table, at)) return;
      }
    }
    // set n: gate (even) or up, of columns n / 2 * 16 .. (past the last one: that
    // one, and no results)
    const char* base[NS];
    int left[NS], off[NS];
#pragma unroll
    for (int n = 0; n < NS; ++n) {
      size_t j = j0 + n / 2 * 16;
      if (j >= a.hidden) j = a.hidden - 1;
      base[n] = uniform(
          (const char*)a.w[n & 1][task.rank] +
          ((size_t)task.expert * a.xw + j * a.ldw) * sizeof(V));
      left[n] = a.hidden - j < 16 ? (int)(a.hidden - j) : 16;
      off[n] = St::offset(base[n], a.ldw, left[n], r);
    }
    const unsigned chunks = (unsigned)((a.in + KC - 1) / KC);
    const unsigned c0 = uniform((unsigned)((uint64_t)chunks * wave / S)),
                   c1 = uniform((unsigned)((uint64_t)chunks * (wave + 1) / S));
    const uint32_t mine =
        uniform((uint32_t)(uintptr_t)lds + wave * (2 * kChunk));
    LDS char* const src = lds + wave * (2 * kChunk);
    auto ask = [&](int n, unsigned c, int buf) {
      St::ask(base[n], a.ldw, left[n], a.in, c, uniform(mine + buf * kChunk),
              lane);
    };
    auto begin = [&] {
      if (c0 < c1) {
        ask(0, c0, 0);
        ask(1, c0, 1);
      }
    };
    LDS int* const mine_list = (LDS int*)(lds + kLds);
    if constexpr (MODE == Mode::DIRECT) {
      begin();
      // the choices of all tables' tokens, one to a workgroup
      if (wave == 0)
        for (int n = blockIdx.x; n < a.tokens * a.tables; n += gridDim.x)
          keep_choice(a, n / a.tokens, n % a.tokens, lane);
      task.count = chosen_by<S>(a, task, mine_list);
      if (j0 == 0) {
        // (a record of every expert, a list of `tokens` pairs for each)
        const int at = a.tables == 1 ? (int)id : task.expert;
        if (t == 0) {
          const Record r = {task.rank, task.expert, at * a.tokens, task.count};
          ((Record*)(task.work + a.at.records))[at] = r;
          if (at == 0) *(int*)task.work = a.most;
        }
        for (int i = t; i < task.count; i += S * 64)
          ((int*)(task.work + a.at.pairs))[at * a.tokens + i] = mine_list[i];
      }
      if (task.count == 0) {
        landed<0>();
        return;
      }
    }
    const int count = task.count;
    for (int i0 = 0; i0 < count; i0 += MT * 16) {
      const int here = count - i0 < MT * 16 ? count - i0 : MT * 16;
      if (MODE != Mode::DIRECT || i0 > 0) begin();
      const XV* x[MT];
      int pair[MT];
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        int i = m * 16 + r;
        if (i >= here) i = here - 1;
        if constexpr (MODE == Mode::FUSED)
          pair[m] = choice.list[choice.record->first + i0 + i];
        else if constexpr (MODE == Mode::DIRECT)
          pair[m] = mine_list[i0 + i];
        else
          pair[m] = task.list[i0 + i];
        x[m] = (const XV*)a.x[task.rank] + (size_t)(pair[m] / a.top) * a.ldx +
               q * M::E;
      }
      f32x4 acc[MT][NS] = {};
      i32x4 fx[MT][U][NX];
      auto load = [&](unsigned c) {
        const int rest = rest_of<St>(a.in, c);
        auto all = [&](auto whole) {
#pragma unroll
          for (int m = 0; m < MT; ++m)
            if (m == 0 || m * 16 < here) {
#pragma unroll
              for (int u = 0; u < U; ++u)
                fetch_row<whole.value>(x[m] + (size_t)c * KC + u * K,
                                       rest - u * K - q * M::E, fx[m][u]);
            }
        };
        if (!SHIFT || rest == KC) {
          all(Yes());
        } else if (a.in >= M::E) {
          all(No());
        } else {
#pragma unroll
          for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
              for (int n = 0; n < NX; ++n)
                fx[m][u][n] = u == 0 && n == 0 && q == 0
                                  ? load_piece<XV>(x[m], a.in)
                                  : i32x4{0, 0, 0, 0};
        }
      };
      auto pin = [&] {
#pragma unroll
        for (int m = 0; m < MT; ++m)
          if (m == 0 || m * 16 < here) arrived(fx[m]);
      };
      auto use = [&](int n, unsigned c, int buf) {
        const int rest = rest_of<St>(a.in, c);
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const i32x4 w =
              St::take(src + buf * kChunk, u, r, q, off[n], rest);
#pragma unroll
          for (int m = 0; m < MT; ++m)
            if (m == 0 || m * 16 < here)
              acc[m][n] = M::up(w, fx[m][u], acc[m][n]);
        }
      };
      sweep<NS, St::kLoads>(c0, c1, load, pin, ask, use);
      if (S > 1) __syncthreads();
      finish(a, task, pair, here, j0, lds, wave, lane, acc);
      if (i0 + MT * 16 < count) __syncthreads();
    }
  }

  // Adds the wavefronts' sums in their order; of the results' MT * C tiles of 16
  // pairs and 16 columns wavefront w finishes those w, w + S ..
  static __device__ void finish(GivenMoe& a, const Task& task,
                                const int (&pairs)[MT], int here, size_t j0,
                                LDS char* lds, int wave, int lane,
                                const f32x4 (&acc)[MT][NS]) {
    const int r = lane & 15, q = lane >> 4;
    auto part = (f32x4(LDS*)[MT * NS][64])lds;
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int n = 0; n < NS; ++n) part[wave][m * NS + n][lane] = acc[m][n];
    if (S > 1)
      __syncthreads();
    else
      in_order();
#pragma unroll 1
    for (int x = wave; x < MT * C; x += S) {
      const int m = x / C, i = m * 16 + r, from = m * NS + x % C * 2;
      const size_t j = j0 + x % C * 16 + q * 4;
      if (m * 16 >= here || j >= held_of(a)) continue;
      f32x4 g = part[0][from][lane], u = part[0][from + 1][lane];
#pragma unroll
      for (int k = 1; k < S; ++k) {
        g += part[k][from][lane];
        u += part[k][from + 1][lane];
      }
      if (i >= here) continue;
      float h[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float gate = g[e], up = u[e];
        const bool there = j + e < a.hidden;
        if constexpr (W == Type::I8) {
          const size_t row = (size_t)task.expert * a.hidden + j + e;
          if (there) {
            gate *= a.s[0][task.rank][row];
            up *= a.s[1][task.rank][row];
          }
        }
        h[e] = there ? up : 0.f;
        g[e] = gate;
      }
      with_act(a.act, [&](auto act) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float v = act_of<act.value, true>(g[e]) * h[e];
          h[e] = j + e < a.hidden ? v : 0.f;
        }
      });
      int one = 0;       // (a choice by ?: put the array in scratch memory)
#pragma unroll
      for (int k = 0; k < MT; ++k) one |= m == k ? pairs[k] : 0;
      char* const row = task.work + a.at.hidden;
      if (M::kWhole || a.planes != (int)Hidden::PARTS) {
        f32x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = h[e];
        *(f32x4*)(row + ((size_t)one * runs_of(a) * 32 + j) * 4) = v;
      } else {
        // in their run of 32: [run][part][value]
        int part[2][3];
        split(h[0], h[1], part[0]);
        split(h[2], h[3], part[1]);
#pragma unroll
        for (int p = 0; p < 3; ++p) {
          i32x2 v = {part[0][p], part[1][p]};
          *(i32x2*)(row + ((((size_t)one * runs_of(a) + j / 32) * 3 + p) * 32 +
                           j % 32) * 2) = v;
        }
      }
    }
  }
};

// ---------------------------------------------------------------- down

// A lane group's hidden values of a step, from value k (of the step's first run)
// of a row of `hidden` on: zeros past what is held.
template <typename M, int FORM>
__device__ inline void fetch_hidden(const char* row, size_t k, size_t held,
                                    int q, i32x4 (&h)[M::pieces(FORM)]) {
  constexpr int kRuns = M::kWhole ? 1 : M::VB / 8,
                N = M::pieces(FORM) / kRuns;
#pragma unroll
  for (int g = 0; g < kRuns; ++g) {
    const size_t at = k + g * 32 + q * (M::kWhole ? 4 : 8);
    const char* from = FORM == (int)Hidden::PARTS
                           ? row + (k / 32 + g) * 192 + q * 16
                           : row + at * 4;
#pragma unroll
    for (int n = 0; n < N; ++n)
      h[g * N + n] =
          at < held ? *(const i32x4*)(from +
                                      n * (FORM == (int)Hidden::PARTS ? 64 : 16))
                    : i32x4{0, 0, 0, 0};
  }
}
// Values as they go to the matrix cores.
template <typename M>
__device__ inline void to_parts(const i32x4 (&h)[M::VB / 4],
                                i32x4 (&part)[M::kParts]) {
#pragma unroll
  for (int g = 0; g < M::VB / 8; ++g)
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const f32x4 v = __builtin_bit_cast(f32x4, h[g * 2 + k / 2]);
      int two[3];
      split(v[k % 2 * 2], v[k % 2 * 2 + 1], two);
#pragma unroll
      for (int p = 0; p < 3; ++p) part[g * 3 + p][k] = two[p];
    }
}
// Bytes of a row of hidden values.
template <int FORM>
__device__ inline size_t hidden_bytes(GivenMoe& a) {
  return runs_of(a) * (FORM == (int)Hidden::PARTS ? 192 : 128);
}

// weight * (wd h) of one pair and column, value by value in 32 bits: for results
// that are NaN, since where values are several parts an infinity may have met a part
// that is 0 or has the other sign.  (What is NaN by itself is soon found to be.)
template <typename M, int FORM>
__device__ inline float whole_result(GivenMoe& a, const char* work, int rank,
                                     int expert, int pair, size_t j) {
  const char* h = work + a.at.hidden + (size_t)pair * hidden_bytes<FORM>(a);
  const auto w = (const typename M::V*)a.w[2][rank] + (size_t)expert * a.xd +
                 j * a.ldd;
  float sum = 0.f;
  for (size_t k = 0; k < a.hidden && sum == sum; ++k) {
    float v;
    if constexpr (FORM == (int)Hidden::PARTS) {
      const auto part = (const unsigned short*)(h + k / 32 * 192) + k % 32;
      auto value = [&](int p) {
        return __builtin_bit_cast(float, (uint32_t)part[p * 32] << 16);
      };
      v = value(0);
      if (fabsf(v) < __builtin_inff()) v += value(1) + value(2);
    } else {
      v = ((const float*)h)[k];
    }
    sum += v * (float)w[k];
  }
  if constexpr (sizeof(typename M::V) == 1)
    sum *= a.s[2][rank][(size_t)expert * a.in + j];
  return sum * ((const float*)(work + a.at.weights))[pair];
}

// weight * (wd h) of the pairs that chose an expert: a workgroup takes 16 * NW
// columns (rows of wd) of one chosen expert, its S wavefronts a part of the
// contraction each; MT tiles of 16 pairs at a time.  The NW sets of 16 rows take
// turns and share the hidden values in registers: they come from L2 in 32 bits, 4 n
// bytes for the 16 NW values of a column of weights with n pairs, and are split
// there (as parts from memory they would be half as many bytes again: 100 tokens,
// 64 experts 2048 x 1024 145 us for the whole layer, 141 so; 16-bit y from two parts
// alone, 2^-16 off, 138).
template <Type W, Type X, bool SHIFT, int FORM, int MT, int NW, int S>
struct Down {
  using M = Mix<W, X>;
  using V = typename M::V;
  // (8-bit weights beside two tiles: 256 bytes would be 192 registers of parts, and
  // with 16-bit ones 512: 64 tokens, 2 of 8 experts 4096 x 8192 8-bit 177 us, bf16 295;
  // with two parts of a value, 2^-16 off, 166 and 271)
  static constexpr int kPieces = MT * M::kParts, NH = M::pieces(FORM);
  static constexpr bool kSplits = FORM == (int)Hidden::VALUES;
  static constexpr int kRow =
      kPieces > 10 ? 128 : M::row(kPieces, MT * NW, SHIFT);
  using St = Stream<V, kRow, SHIFT>;
  static constexpr int VB = M::VB, K = 4 * VB;
  static constexpr int U = St::kSteps, KC = U * K, kChunk = St::kChunk,
                       BJ = 16 * NW;
  static constexpr int kParts = S * MT * NW * 1024;
  static constexpr int kLds = std::max(S * 2 * kChunk, kParts);

  static __device__ void run(GivenMoe& a, LDS char* lds) {
    const int t = threadIdx.x, lane = t & 63, wave = uniform(t >> 6);
    const int r = lane & 15, q = lane >> 4;
    const unsigned tiles = (unsigned)((a.in + BJ - 1) / BJ);
    const unsigned id = uniform(blockIdx.x / tiles);
    const size_t j0 = (size_t)uniform(blockIdx.x % tiles) * BJ;
    Task task;
    if (!task.find(a, uniform(id / a.most), uniform(id % a.most))) return;
    const int rank = task.rank, expert = task.expert, count = task.count;
    const int* list = task.list;
    const char* hidden = task.work + a.at.hidden;
    const size_t held = held_of(a);

    // (sets past the last row: that row, and no results)
    const char* base[NW];
    int left[NW], off[NW];
#pragma unroll
    for (int n = 0; n < NW; ++n) {
      const size_t j = j0 + n * 16 < a.in ? j0 + n * 16 : a.in - 1;
      left[n] = a.in - j < 16 ? (int)(a.in - j) : 16;
      base[n] = uniform((const char*)a.w[2][rank] +
                        ((size_t)expert * a.xd + j * a.ldd) * sizeof(V));
      off[n] = St::offset(base[n], a.ldd, left[n], r);
    }
    const unsigned chunks = (unsigned)((a.hidden + KC - 1) / KC);
    const unsigned c0 = uniform((unsigned)((uint64_t)chunks * wave / S)),
                   c1 = uniform((unsigned)((uint64_t)chunks * (wave + 1) / S));
    const uint32_t mine =
        uniform((uint32_t)(uintptr_t)lds + wave * (2 * kChunk));
    LDS char* const src = lds + wave * (2 * kChunk);
    auto ask = [&](int n, unsigned c, int buf) {
      St::ask(base[n], a.ldd, left[n], a.hidden, c,
              uniform(mine + buf * kChunk), lane);
    };
    for (int i0 = 0; i0 < count; i0 += MT * 16) {
      const int here = count - i0 < MT * 16 ? count - i0 : MT * 16;
      if (c0 < c1) {
        ask(0, c0, 0);
        ask(1, c0, 1);
      }
      const char* row[MT];
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        int i = m * 16 + r;
        if (i >= here) i = here - 1;
        row[m] = hidden + (size_t)list[i0 + i] * hidden_bytes<FORM>(a);
      }
      f32x4 acc[MT][NW] = {};
      i32x4 h[MT][U][NH];
      i32x4 split_h[kSplits ? MT : 1][kSplits ? U : 1][M::kParts];
      auto& parts = *[&] {
        if constexpr (kSplits)
          return &split_h;
        else
          return &h;
      }();
      auto load = [&](unsigned c) {
#pragma unroll
        for (int m = 0; m < MT; ++m)
          if (m == 0 || m * 16 < here) {
#pragma unroll
            for (int u = 0; u < U; ++u)
              fetch_hidden<M, FORM>(row[m], (size_t)c * KC + u * K, held, q,
                                    h[m][u]);
          }
      };
      auto pin = [&] {
#pragma unroll
        for (int m = 0; m < MT; ++m)
          if (m == 0 || m * 16 < here) {
            arrived(h[m]);
            if constexpr (kSplits)
#pragma unroll
              for (int u = 0; u < U; ++u) to_parts<M>(h[m][u], split_h[m][u]);
          }
      };
      auto use = [&](int n, unsigned c, int buf) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const i32x4 v = St::take(src + buf * kChunk, u, r, q, off[n],
                                   rest_of<St>(a.hidden, c));
#pragma unroll
          for (int m = 0; m < MT; ++m)
            if (m == 0 || m * 16 < here)
              acc[m][n] = M::down(v, parts[m][u], acc[m][n]);
        }
      };
      sweep<NW, St::kLoads>(c0, c1, load, pin, ask, use);
      // the wavefronts' sums in their order
      if (S > 1) __syncthreads();
      auto part = (f32x4(LDS*)[MT * NW][64])lds;
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int n = 0; n < NW; ++n)
          part[wave][m * NW + n][lane] = acc[m][n];
      if (S > 1)
        __syncthreads();
      else
        in_order();
#pragma unroll 1
      for (int x = wave; x < MT * NW; x += S) {
        const int m = x / NW, n = x % NW, i = m * 16 + r;
        if (i >= here) continue;
        f32x4 v = part[0][x][lane];
#pragma unroll
        for (int k = 1; k < S; ++k) v += part[k][x][lane];
        const size_t j = j0 + n * 16 + q * 4;
        if (j >= a.in) continue;
        const int pair = list[i0 + i];
        if constexpr (W == Type::I8) {
          const float* s = a.s[2][rank] + (size_t)expert * a.in + j;
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] *= j + e < a.in ? s[e] : 0.f;
        }
        v *= task.weights[pair];
        float* to = (float*)(task.work + a.at.parts) +
                    (size_t)pair * a.pitch + j;
        *(f32x4*)to = v;
      }
      if (i0 + MT * 16 < count) __syncthreads();
    }
  }
};

// y = sum of weight * (wd h) + residual for at most 8 tokens, whole: a workgroup
// takes 8 columns of a rank and goes over all the chosen experts.  A unit is a
// chunk of one expert's 8 rows; a wavefront takes two at a time, one in the upper
// and one in the lower 8 of the matrix cores' rows, their pairs in the left and
// right 8 columns: of the product the two blocks that belong together count.
// A token's sums stay in LDS, a wavefront's own, and are joined in order.  One
// token, 8 experts 2048 x 1024: 11 us for 34 MB, of which half is the way to the
// first weights (records, pairs, hidden values); by expert and joined 15.
template <Type W, Type X, bool SHIFT, int FORM>
struct DownSmall {
  using M = Mix<W, X>;
  using V = typename M::V;
  // (of two turns; three parts of 512 bytes just fit)
  static constexpr int NH = M::pieces(FORM), kPieces = NH * (NH > 3 ? 2 : 1);
  using St = Stream<V, M::row(kPieces, 1, SHIFT), SHIFT>;
  static constexpr int VB = M::VB, K = 4 * VB;
  static constexpr int U = St::kSteps, KC = U * K, kChunk = St::kChunk;
  static constexpr int S = 8, kMost = kSmall * kTop;     // pairs
  static constexpr int kSums = S * 2 * kChunk;
  static constexpr int kRecords = kSums + S * kSmall * 8 * 4,
                       kList = kRecords + kMost * (int)sizeof(Record),
                       kWeights = kList + kMost * 4,
                       kLds = kWeights + kMost * 4;

  // One of a wavefront's two units.
  struct Half {
    unsigned unit, end;        // this one, and past the last
    unsigned chunk;
    int expert, first, count;
  };

  static __device__ void run(GivenMoe& a, LDS char* lds) {
    const int t = threadIdx.x, lane = t & 63, wave = uniform(t >> 6);
    const int r = lane & 15, q = lane >> 4, side = r >> 3;
    const unsigned tiles = (unsigned)((a.in + 7) / 8);
    const int rank = uniform(blockIdx.x / tiles);
    const size_t j0 = (size_t)uniform(blockIdx.x % tiles) * 8;
    const int left = a.in - j0 < 8 ? (int)(a.in - j0) : 8;
    const int pairs = a.tokens * a.top;
    char* const work = table_of(a, a.tables == 1 ? 0 : rank);
    const char* hidden = work + a.at.hidden;
    const size_t held = held_of(a);

    // the table's lists in LDS
    LDS Record* const records = (LDS Record*)(lds + kRecords);
    LDS int* const list = (LDS int*)(lds + kList);
    LDS float* const weights = (LDS float*)(lds + kWeights);
    LDS float* const mine = (LDS float*)(lds + kSums) + wave * (kSmall * 8);
    // (a.most * 4 <= 512 threads, and pairs are fewer; all loads go out at once)
    static_assert(kMost * 4 <= S * 64);
    const int* starts = (const int*)work + 1 + rank;
    const int low1 = starts[0], high1 = starts[1];
    int word = 0, one = 0;
    float share = 0.f;
    if (t < a.most * 4) word = ((const int*)(work + a.at.records))[t];
    if (t < pairs) {
      one = ((const int*)(work + a.at.pairs))[t];
      share = ((const float*)(work + a.at.weights))[t];
    }
    ((LDS int*)records)[t] = word;
    if (t < kMost) {
      list[t] = one;
      weights[t] = share;
    }
    mine[lane] = 0.f;
    // Asks for what follows the lists from the arguments.
    asm volatile("" ::"s"(a.w[2][rank]), "s"(a.xd), "s"(a.ldd), "s"(a.r[rank]),
                 "s"(a.y[rank]), "s"(a.ldy), "s"(a.ldr), "s"(a.s[2][rank]));
    const int low = uniform(low1), high = uniform(high1);
    __syncthreads();

    const unsigned chunks = (unsigned)((a.hidden + KC - 1) / KC);
    const unsigned units = (unsigned)(high - low) * chunks;
    const unsigned u0 = uniform((unsigned)((uint64_t)units * wave / S)),
                   u1 = uniform((unsigned)((uint64_t)units * (wave + 1) / S));
    const unsigned turns = (u1 - u0 + 1) / 2;
    const uint32_t buffer =
        uniform((uint32_t)(uintptr_t)lds + wave * (2 * kChunk));
    LDS char* const src = lds + wave * (2 * kChunk);
    auto set = [&](Half& x) {
      LDS Record* rec = records + low + x.unit / chunks;
      x.expert = uniform(rec->expert);
      x.first = uniform(rec->first);
      x.count = uniform(rec->count);
    };
    Half now[2];
    auto start = [&](Half& x, unsigned from, unsigned end) {
      x = {from, end, from % chunks, 0, 0, 0};
      if (from < end) set(x);
    };
    auto step = [&](Half& x) {
      if (x.unit >= x.end) return;
      ++x.unit;
      if (++x.chunk == chunks) {
        x.chunk = 0;
        if (x.unit < x.end) set(x);
      }
    };
    auto base = [&](const Half& x) {
      return uniform((const char*)a.w[2][rank] +
                     ((size_t)x.expert * a.xd + j0 * a.ldd) * sizeof(V));
    };
    // (a half that is through, the second one of an odd number, stays where it
    // is: its block of the product is left out)
    auto ask = [&](const Half (&x)[2], int buf) {
      const uint32_t to = uniform(buffer + buf * kChunk);
      St::template ask<0, 8>(base(x[0]), a.ldd, left, a.hidden, x[0].chunk, to,
                             lane);
      if (x[1].unit < x[1].end)
        St::template ask<8, 8>(base(x[1]), a.ldd, left, a.hidden, x[1].chunk,
                               to, lane);
    };
    auto fetch = [&](const Half (&x)[2], i32x4 (&h)[U][NH]) {
      const int count = side ? x[1].count : x[0].count,
                first = side ? x[1].first : x[0].first;
      const unsigned chunk = side ? x[1].chunk : x[0].chunk;
      // (lanes past the pairs load nothing, and their columns do not count)
      const bool some = (!side || x[1].unit < x[1].end) && (r & 7) < count;
      const int i = r & 7;
      const char* row =
          hidden + (some ? (size_t)list[first + i] : 0) *
                       hidden_bytes<FORM>(a);
#pragma unroll
      for (int u = 0; u < U; ++u)
        fetch_hidden<M, FORM>(row, (size_t)chunk * KC + u * K,
                              some ? held : 0, q, h[u]);
    };
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    // Adds one half's sums to its tokens': lane (r, q): pair r % 8, columns q %
    // 2 * 4 ..
    auto flush = [&](const Half& x, int which) {
      const int i = r & 7;
      if (side == which && q >> 1 == which) {
        if (i < x.count) {
          f32x4 v = acc;
          const int j = (q & 1) * 4;
          if constexpr (W == Type::I8) {
            const float* s =
                a.s[2][rank] + (size_t)x.expert * a.in + j0 + j;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] *= j + e < left ? s[e] : 0.f;
          }
          LDS f32x4* to =
              (LDS f32x4*)(mine + list[x.first + i] / a.top * 8 + j);
          *to += v * weights[list[x.first + i]];
        }
        acc = f32x4{0.f, 0.f, 0.f, 0.f};
      }
      in_order();
    };
    if (turns) {
      start(now[0], u0, u0 + turns);
      start(now[1], u0 + turns, u1);
      // two turns at a time: both are asked for at once
      auto turn = [&](const Half (&was)[2], const Half (&then)[2], int buf,
                      i32x4 (&h)[U][NH]) {
        const Half& own = side ? was[1] : was[0];
        const int off = St::offset(side ? base(was[1]) : base(was[0]), a.ldd,
                                   left, r & 7);
        const int rest = rest_of<St>(a.hidden, own.chunk);
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const i32x4 w = St::take(src + buf * kChunk, u, r, q, off, rest);
          if constexpr (FORM == (int)Hidden::VALUES) {
            i32x4 parts[M::kParts];
            to_parts<M>(h[u], parts);
            acc = M::down(w, parts, acc);
          } else {
            acc = M::down(w, h[u], acc);
          }
        }
#pragma unroll
        for (int s = 0; s < 2; ++s)
          if (was[s].unit < was[s].end &&
              (then[s].unit == then[s].end || then[s].chunk == 0))
            flush(was[s], s);
      };
#pragma unroll 1
      for (unsigned k = 0; k < turns; k += 2) {
        i32x4 h[2][U][NH];
        const bool two = k + 1 < turns;
        const Half one[2] = {now[0], now[1]};
        ask(now, 0);
        fetch(now, h[0]);
        step(now[0]);
        step(now[1]);
        const Half other[2] = {now[0], now[1]};
        if (two) {
          ask(now, 1);
          fetch(now, h[1]);
          step(now[0]);
          step(now[1]);
        }
        landed<0>();
        turn(one, other, 0, h[0]);
        if (two) turn(other, now, 1, h[1]);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      }
    }
    __syncthreads();
    using Out = typename M::XV;
    const int token = t / 8, col = t % 8;
    if (token >= a.tokens || col >= left) return;
    LDS float* const sums = (LDS float*)(lds + kSums);
    float v = 0.f;
#pragma unroll
    for (int k = 0; k < S; ++k) v += sums[k * (kSmall * 8) + t];
    const size_t j = j0 + col;
    if (!M::kWhole && v != v) {
      v = 0.f;
      for (int n = low; n < high && v == v; ++n)
        for (int i = 0; i < records[n].count; ++i) {
          const int pair = list[records[n].first + i];
          if (pair / a.top == token)
            v += whole_result<M, FORM>(a, work, rank, records[n].expert, pair,
                                       j);
        }
    }
    if (const void* res = a.r[rank]) {
      const size_t from = (size_t)token * a.ldr + j;
      v += a.out32 ? ((const float*)res)[from]
                   : (float)((const Out*)res)[from];
    }
    store_out<1>(a.y[rank], (size_t)token * a.ldy + j, &v, 1, a.out32, false,
                 Out());
  }
};

// y = the sum of a token's parts, in the order of its choices, + residual: four
// columns per thread.
template <Type W, Type X>
__global__ __launch_bounds__(256) void k_moe_join(MoeArgs) {
  GivenMoe& a = *(GivenMoe*)__builtin_amdgcn_kernarg_segment_ptr();
  using Out = typename Elem<X>::V;
  const size_t j = ((size_t)blockIdx.x * 256 + threadIdx.x) * 4;
  const int token = blockIdx.y, rank = blockIdx.z;
  if (j >= a.in) return;
  char* const work = table_of(a, a.tables == 1 ? 0 : rank);
  const int* owner = (const int*)(work + a.at.owner) + (size_t)token * a.top;
  const float* parts = (const float*)(work + a.at.parts) +
                       (size_t)token * a.top * a.pitch + j;
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  for (int k = 0; k < a.top; ++k) {
    const int own = owner[k];
    if (own < 0 || own % kRanks != rank) continue;
    f32x4 p = *(const f32x4*)(parts + (size_t)k * a.pitch);
    if (X != Type::F32)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (p[e] != p[e] && j + e < a.in) {
          auto result = [&](auto form) {
            return whole_result<Mix<W, X>, form.value>(
                a, work, rank, own / kRanks, token * a.top + k, j + e);
          };
          if (a.planes == (int)Hidden::PARTS)
            p[e] = result(std::integral_constant<int, (int)Hidden::PARTS>());
          else
            p[e] = result(std::integral_constant<int, (int)Hidden::VALUES>());
        }
    v += p;
  }
  float o[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) o[e] = v[e];
  const long rest = (long)a.in - (long)j;
  if (const void* res = a.r[rank]) {
    float p[4];
    const size_t from = (size_t)token * a.ldr + j;
    if (a.out32)
      fetch_vals<float, 4>((const float*)res + from, p, rest, false);
    else
      fetch_vals<Out, 4>((const Out*)res + from, p, rest, false);
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] += p[e];
  }
  store_out<4>(a.y[rank], (size_t)token * a.ldy + j, o, rest, a.out32, false,
               Out());
}

// ---------------------------------------------------------------- launches

template <Type W, Type X, bool SHIFT, Mode MODE, int MT, int C, int S>
__global__ __launch_bounds__(S * 64, 2) void k_moe_up(MoeArgs) {
  GivenMoe& a = *(GivenMoe*)__builtin_amdgcn_kernarg_segment_ptr();
  extern __shared__ char lds[];
  Up<W, X, SHIFT, MODE, MT, C, S>::run(a, (LDS char*)lds);
}

template <Type W, Type X, bool SHIFT, int FORM, int MT, int NW, int S>
__global__ __launch_bounds__(S * 64, 2) void k_moe_down(MoeArgs) {
  GivenMoe& a = *(GivenMoe*)__builtin_amdgcn_kernarg_segment_ptr();
  extern __shared__ char lds[];
  Down<W, X, SHIFT, FORM, MT, NW, S>::run(a, (LDS char*)lds);
}

template <Type W, Type X, bool SHIFT, int FORM>
__global__ __launch_bounds__(512) void k_moe_down_small(MoeArgs) {
  GivenMoe& a = *(GivenMoe*)__builtin_amdgcn_kernarg_segment_ptr();
  extern __shared__ char lds[];
  DownSmall<W, X, SHIFT, FORM>::run(a, (LDS char*)lds);
}

template <void (*K)(MoeArgs)>
hipError_t launch_moe(const MoeArgs& a, size_t groups, int threads,
                      size_t bytes, hipStream_t stream) {
  if (groups == 0) return hipSuccess;
  if (groups * threads > 0xffffffffu) return hipErrorInvalidConfiguration;
  if (bytes > 65536) {
    static std::atomic<uint64_t> asked{0};     // one bit per device
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    const uint64_t bit = dev < 64 ? (uint64_t)1 << dev : 0;
    if (!(asked.load(std::memory_order_relaxed) & bit)) {
      e = hipFuncSetAttribute((const void*)K,
                              hipFuncAttributeMaxDynamicSharedMemorySize,
                              160 * 1024);
      if (e != hipSuccess) return e;
      asked.fetch_or(bit, std::memory_order_relaxed);
    }
  }
  hipLaunchKernelGGL(K, dim3((unsigned)groups), dim3(threads), bytes, stream,
                     a);
  return hipGetLastError();
}

template <Type W, Type X, bool SHIFT, Mode MODE, int MT, int S>
hipError_t go_up(const MoeArgs& a, hipStream_t stream) {
  constexpr int C = columns_up(W, MODE == Mode::FUSED, SHIFT, MT);
  using K = Up<W, X, SHIFT, MODE, MT, C, S>;
  const size_t tiles = (a.hidden + K::BJ - 1) / K::BJ;
  const size_t choice =
      Choice::bytes(a.tokens * a.top,
                    a.experts * (a.tables == 1 ? a.ranks : 1));
  size_t groups = tiles * a.most * a.tables, bytes = K::kLds;
  if (MODE == Mode::FUSED) bytes += choice;
  if (MODE == Mode::DIRECT) {
    groups = tiles * a.experts * a.ranks;
    bytes += kDirectList * 4;
  }
  return launch_moe<k_moe_up<W, X, SHIFT, MODE, MT, C, S>>(
      a, groups, S * 64, bytes, stream);
}

template <Type W, Type X, Mode MODE, int MT>
hipError_t waves_up(const MoeArgs& a, hipStream_t stream) {
  if constexpr (MT < 4)
    if (!a.fast[0]) return go_up<W, X, true, MODE, MT, 4>(a, stream);
  return a.waves[0] == 4 ? go_up<W, X, false, MODE, MT, 4>(a, stream)
                         : go_up<W, X, false, MODE, MT, 2>(a, stream);
}

template <Type W, Type X>
hipError_t pick_up(const MoeArgs& a, hipStream_t stream) {
  switch ((Mode)a.mode) {
    case Mode::TABLE: return waves_up<W, X, Mode::TABLE, 1>(a, stream);
    case Mode::FUSED: return waves_up<W, X, Mode::FUSED, 1>(a, stream);
    default: break;
  }
  if (a.tiles[0] == 1) return waves_up<W, X, Mode::DIRECT, 1>(a, stream);
  if (a.tiles[0] == 2) return waves_up<W, X, Mode::DIRECT, 2>(a, stream);
  return waves_up<W, X, Mode::DIRECT, 4>(a, stream);
}

template <Type W, Type X, bool SHIFT, int FORM, int MT, int NW, int S>
hipError_t go_down(const MoeArgs& a, hipStream_t stream) {
  using K = Down<W, X, SHIFT, FORM, MT, NW, S>;
  return launch_moe<k_moe_down<W, X, SHIFT, FORM, MT, NW, S>>(
      a, (a.in + K::BJ - 1) / K::BJ * a.most * a.tables, S * 64, K::kLds,
      stream);
}

template <Type W, Type X, bool SHIFT, int FORM>
hipError_t go_small(const MoeArgs& a, hipStream_t stream) {
  return launch_moe<k_moe_down_small<W, X, SHIFT, FORM>>(
      a, (a.in + 7) / 8 * a.ranks, 512, DownSmall<W, X, SHIFT, FORM>::kLds,
      stream);
}

template <Type W, Type X, int FORM, int MT>
hipError_t waves_down(const MoeArgs& a, hipStream_t stream) {
  if (!a.fast[1])
    return a.sets == 2 ? go_down<W, X, true, FORM, MT, 2, 4>(a, stream)
                       : go_down<W, X, true, FORM, MT, 4, 4>(a, stream);
  if (a.sets == 2) return go_down<W, X, false, FORM, MT, 2, 4>(a, stream);
  return a.waves[1] == 4 ? go_down<W, X, false, FORM, MT, 4, 4>(a, stream)
                         : go_down<W, X, false, FORM, MT, 4, 2>(a, stream);
}

template <Type W, Type X, int FORM>
hipError_t pick_down(const MoeArgs& a, hipStream_t stream) {
  if (a.small)
    return a.fast[1] ? go_small<W, X, false, FORM>(a, stream)
                     : go_small<W, X, true, FORM>(a, stream);
  // (8-bit weights' parts come from memory for one tile of pairs only)
  if constexpr (W != Type::I8 || FORM != (int)Hidden::PARTS)
    if (a.tiles[1] == 2) return waves_down<W, X, FORM, 2>(a, stream);
  return waves_down<W, X, FORM, 1>(a, stream);
}

template <Type W, Type X>
hipError_t run_moe(const MoeArgs& a, hipStream_t stream) {
  hipError_t e = pick_up<W, X>(a, stream);
  if (e != hipSuccess) return e;
  if constexpr (X == Type::F32)
    e = pick_down<W, X, (int)Hidden::WHOLE>(a, stream);
  else
    e = a.planes == (int)Hidden::PARTS
            ? pick_down<W, X, (int)Hidden::PARTS>(a, stream)
            : pick_down<W, X, (int)Hidden::VALUES>(a, stream);
  if (e != hipSuccess || a.small) return e;
  hipLaunchKernelGGL((k_moe_join<W, X>),
                     dim3((unsigned)((a.in + 1023) / 1024), a.tokens, a.ranks),
                     dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace
}  // namespace moe
}  // namespace dpar
