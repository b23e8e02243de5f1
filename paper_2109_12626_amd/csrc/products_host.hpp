// What the entry points of the layer products share: argument and alias checks,
// the rules that choose a kernel, launches of at most kRanks ranks.
#pragma once

#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstdlib>
#include <new>
#include <vector>

#include "dpar.h"
#include "errors.hpp"
#include "products.hpp"

using dpar::products::Args;
using dpar::products::Form;
using dpar::products::kRanks;
using dpar::products::SlopeArgs;
using dpar::products::SumArgs;
using dpar::products::Type;

namespace {

inline int fail(int code, const char* fmt, ...)
    __attribute__((format(printf, 2, 3)));
inline int fail(int code, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  return dpar::set_error(code, buf);
}

// 256 rows of an operand lie within the kernels' 32-bit offsets (the fast
// loads; others use 64-bit addresses throughout).
constexpr size_t kFastPitch = (size_t)1 << 23;

// Addresses are below 2^48, so a matrix beyond that is none; it would overflow
// the sizes computed from it.
constexpr size_t kMostBytes = (size_t)1 << 48;

// One array argument: p matrices of rows x cols elements, `ld` elements
// apart.
struct Mat {
  const char* name;
  const void* const* at;
  size_t rows, cols, ld, esz;
  bool out;
  bool gaps;               // entries may be null (bias, residual)
  bool used;
  const void* const* twin[2] = {nullptr, nullptr};  // inputs it may be

  size_t extent() const {
    return rows && cols ? ((rows - 1) * ld + cols) * esz : 0;
  }
  // every row starts on 16 bytes
  bool aligned(int p) const {
    if (!used || !extent()) return true;
    uintptr_t bits = rows > 1 ? ld * esz : 0;
    for (int i = 0; i < p; ++i) bits |= (uintptr_t)at[i];
    return (bits & 15) == 0;
  }
  // rows of whole aligned 16-byte pieces, 256 of them within 32 bits
  bool fast(int p) const {
    return !used || (extent() && aligned(p) && cols * esz % 16 == 0 &&
                     ld < kFastPitch);
  }
  const void* rank(int i) const { return used ? at[i] : nullptr; }
};

struct Range {
  uintptr_t lo, hi;
  size_t width, pitch;
  int mat, rank;
};

// Whether two matrices share a byte; ranges overlap already.  Matrices of one
// row distance may lie side by side.
inline bool share(const Range& a, const Range& b) {
  if (a.pitch == b.pitch && a.pitch != 0) {
    const size_t d = (b.lo - a.lo) % a.pitch;   // b.lo >= a.lo
    if (d >= a.width && d + b.width <= a.pitch) return false;
  }
  return true;
}

inline int check_alias(const Mat* mats, int n, int p, const char* call) {
  thread_local std::vector<Range> r;
  r.clear();
  for (int k = 0; k < n; ++k) {
    const Mat& m = mats[k];
    if (!m.used || !m.extent()) continue;
    for (int i = 0; i < p; ++i)
      if (const uintptr_t a = (uintptr_t)m.at[i])
        r.push_back({a, a + m.extent(), m.cols * m.esz, m.ld * m.esz, k, i});
  }
  std::sort(r.begin(), r.end(), [](const Range& a, const Range& b) {
    return a.lo != b.lo ? a.lo < b.lo : a.mat < b.mat;
  });
  // the same matrix read by many ranks counts once
  r.erase(std::unique(r.begin(), r.end(),
                      [&](const Range& a, const Range& b) {
                        return !mats[a.mat].out && a.mat == b.mat &&
                               a.lo == b.lo;
                      }),
          r.end());
  for (size_t k = 0; k < r.size(); ++k)
    for (size_t l = k + 1; l < r.size() && r[l].lo < r[k].hi; ++l) {
      const Mat &a = mats[r[k].mat], &b = mats[r[l].mat];
      if (!a.out && !b.out) continue;
      if (!share(r[k], r[l])) continue;
      // an output in place of its rank's input
      const Range &o = a.out ? r[k] : r[l], &in = a.out ? r[l] : r[k];
      const Mat &mo = mats[o.mat], &mi = mats[in.mat];
      if (!mi.out && o.lo == in.lo && mo.ld == mi.ld &&
          (mo.twin[0] == mi.at || mo.twin[1] == mi.at) &&
          mi.at[o.rank] == mo.at[o.rank]) {
        // read by no other rank
        bool alone = true;
        for (int i = 0; i < p; ++i)
          if (i != o.rank && mi.at[i] == mo.at[o.rank]) alone = false;
        if (alone) continue;
      }
      return fail(DPAR_ERR_ALIAS, "%s: %s of rank %d overlaps %s of rank %d",
                  call, a.name, r[k].rank, b.name, r[l].rank);
    }
  return DPAR_SUCCESS;
}

inline int check_mats(const Mat* mats, int n, int p, const char* call) {
  for (int k = 0; k < n; ++k) {
    const Mat& m = mats[k];
    if (!m.used) continue;
    if (m.ld < m.cols && m.rows > 1)
      return fail(DPAR_ERR_INVALID_ARG, "%s: rows of %s overlap: distance "
                  "%zu, length %zu", call, m.name, m.ld, m.cols);
    if (!m.at) return fail(DPAR_ERR_INVALID_ARG, "%s: null array %s", call,
                           m.name);
    if (m.rows && m.cols &&
        std::max(m.ld, m.cols) > kMostBytes / m.esz / m.rows)
      return fail(DPAR_ERR_UNSUPPORTED, "%s: %s of 2^48 bytes or more", call,
                  m.name);
    const bool empty = m.extent() == 0;
    for (int i = 0; i < p; ++i) {
      const uintptr_t a = (uintptr_t)m.at[i];
      if (!a) {
        if (m.gaps || empty) continue;
        return fail(DPAR_ERR_INVALID_ARG, "%s: %s of rank %d is null", call,
                    m.name, i);
      }
      if (a % m.esz)
        return fail(DPAR_ERR_INVALID_ARG, "%s: %s of rank %d is not aligned "
                    "to its element", call, m.name, i);
      if (a >> 48)
        return fail(DPAR_ERR_UNSUPPORTED, "%s: address of %s of rank %d above "
                    "2^48", call, m.name, i);
    }
  }
  return check_alias(mats, n, p, call);
}

inline size_t size_of(Type t) {
  return t == Type::F32 ? 4 : t == Type::I8 ? 1 : 2;
}
inline const char* name_of(Type t) {
  return t == Type::F32    ? "float32"
         : t == Type::BF16 ? "bfloat16"
         : t == Type::F16  ? "float16"
                           : "int8";
}

constexpr size_t kMost = (size_t)1 << 31;     // rows, in, out
constexpr size_t kMostPitch = (size_t)1 << 38;

// Sums of more products of two 8-bit values may leave 32 bits.
constexpr size_t kMostInt8 = ((size_t)1 << 31) / (128 * 128) - 1;

// The options with row distances filled in.  int8: the entry point takes 8-bit
// operands (and no others).
inline int check_options(const char* call, int p, const dpar_product_t* opt,
                         dpar_product_t* o, Type* t, size_t* esz, size_t* osz,
                         bool int8 = false) {
  dpar::set_error(0, "");
  if (p < 1) return fail(DPAR_ERR_INVALID_ARG, "%s: p must be >= 1", call);
  if (!opt) return fail(DPAR_ERR_INVALID_ARG, "%s: null options", call);
  *o = *opt;
  switch (o->dtype) {
    case DPAR_FLOAT32: *t = Type::F32; break;
    case DPAR_BFLOAT16: *t = Type::BF16; break;
    case DPAR_FLOAT16: *t = Type::F16; break;
    case DPAR_INT8: *t = Type::I8; break;
    default:
      return fail(DPAR_ERR_UNSUPPORTED, "%s: dtype %d", call, (int)o->dtype);
  }
  if ((*t == Type::I8) != int8)
    return fail(DPAR_ERR_UNSUPPORTED, "%s: dtype %d", call, (int)o->dtype);
  if (int8) {
    if (o->out_dtype != DPAR_FLOAT32 && o->out_dtype != DPAR_BFLOAT16 &&
        o->out_dtype != DPAR_FLOAT16)
      return fail(DPAR_ERR_UNSUPPORTED, "%s: out_dtype %d", call,
                  (int)o->out_dtype);
    if (o->in > kMostInt8)
      return fail(DPAR_ERR_UNSUPPORTED, "%s: sums of more than %zu products",
                  call, kMostInt8);
  } else if (o->out_dtype != o->dtype && o->out_dtype != DPAR_FLOAT32) {
    return fail(DPAR_ERR_UNSUPPORTED, "%s: out_dtype %d with dtype %d", call,
                (int)o->out_dtype, (int)o->dtype);
  }
  if ((int)o->act < DPAR_ACT_NONE || (int)o->act > DPAR_ACT_SILU)
    return fail(DPAR_ERR_INVALID_ARG, "%s: unknown activation %d", call,
                (int)o->act);
  if (o->rows >= kMost || o->in >= kMost || o->out >= kMost)
    return fail(DPAR_ERR_UNSUPPORTED, "%s: a size beyond 2^31", call);
  *esz = size_of(*t);
  *osz = o->out_dtype == DPAR_FLOAT32 ? 4 : 2;
  size_t* const in[] = {&o->ldx, &o->ldw, &o->lddx, &o->lddw};
  size_t* const out[] = {&o->ldy, &o->ldr, &o->ldz};
  for (size_t* v : in)
    if (!*v) *v = o->in;
  for (size_t* v : out)
    if (!*v) *v = o->out;
  for (size_t v : {o->ldx, o->ldw, o->lddx, o->lddw, o->ldy, o->ldr, o->ldz})
    if (v > kMostPitch)
      return fail(DPAR_ERR_UNSUPPORTED, "%s: a row distance beyond 2^38",
                  call);
  // a single row has no distance (the kernels' offsets of rows that are not
  // there, held inside the matrix, would be off 16 bytes with an odd one)
  if (o->rows <= 1)
    o->ldx = o->lddx = o->in, o->ldy = o->ldr = o->ldz = o->out;
  if (o->out <= 1) o->ldw = o->lddw = o->in;
  return DPAR_SUCCESS;
}

// CUs of the current device (asked once per device).
inline int cu_count() {
  constexpr int kKnown = 64;
  static std::atomic<int> known[kKnown];
  int dev = 0, cus = 0;
  if (hipGetDevice(&dev) != hipSuccess) {
    (void)hipGetLastError();
    return 256;
  }
  if (dev < kKnown) cus = known[dev].load(std::memory_order_relaxed);
  if (cus > 0) return cus;
  if (hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount,
                            dev) != hipSuccess || cus < 1) {
    (void)hipGetLastError();
    return 256;
  }
  if (dev < kKnown) known[dev].store(cus, std::memory_order_relaxed);
  return cus;
}

// Ranks of the largest launch: p ranks in as few launches as they need, all
// about equal.
inline int ranks_per_launch(int p) {
  const int n = (p + kRanks - 1) / kRanks;
  return (p + n - 1) / n;
}

// How a product runs.
struct Shape {
  int waves, sets, tile, splits;
  size_t part;           // bytes of workspace
  double ns;             // estimate (tiles only)
};

// Time of one contraction tile (128 bytes of every row) of a workgroup on a
// CU, in ns: its share of the CU's rate when the CU is full, and the least it
// takes alone (memory latency over the two tiles in flight); workgroups
// resident.  Measured on an MI355X.
struct TileCost {
  double rate, alone;
  int resident;
};
// 64 x 64 with two and with four tiles in LDS, 128 x 128, 256 x 128, 256 x 256;
// the last two for 16-bit operands of whole aligned pieces only, and other
// operands have no four-buffer form.  8-bit operands go by the 16-bit ones' figures
// (a tile of as many bytes), which leave out that their results are twice as large
// a share: 7 x 875 x 1001 x 1000 linear 15.6 us by them, 27.8 measured.
constexpr int kTiles = 5;
constexpr size_t kTileRows[kTiles] = {64, 64, 128, 256, 256},
                 kTileCols[kTiles] = {64, 64, 128, 128, 256};
constexpr TileCost kFast16[kTiles] = {
    {220, 500, 5}, {270, 400, 2}, {610, 800, 2}, {1050, 950, 1},
    {1600, 1200, 1}};
constexpr TileCost kFast32[kTiles] = {
    {530, 700, 5}, {600, 600, 2}, {2100, 2200, 2}};
constexpr TileCost kSlow16[kTiles] = {{400, 1000, 4}, {}, {850, 1500, 2}};
constexpr TileCost kSlow32[kTiles] = {{650, 1000, 4}, {}, {2400, 2700, 2}};
// Joining a split contraction: a second launch, and its bytes (written by the
// first) per ns.
constexpr double kJoinNs = 4000, kJoinRate = 2300;
constexpr double kStartNs = 2000;      // first loads and last stores
constexpr size_t kMostPart = (size_t)256 << 20;

// Rows up to which the forward forms may take the few-rows kernel: 48 x 4096 x
// 8192 gated 29 us (tiles: 53); half of that in 32 bits (8 x 64 x 2048 x 4096
// 98 us, in tiles 89).
constexpr size_t kFewRows = 64;

inline Shape shape_of(Form f, Type t, int ranks, int pairs, size_t ni, size_t nj,
               size_t nc, int cus, bool split, bool fast) {
  if ((f == Form::LINEAR || f == Form::GATED) &&
      ni <= (t == Type::F32 ? kFewRows / 2 : kFewRows)) {
    // Sets of 16 weight rows per wavefront.  More share x's loads, fewer give
    // more wavefronts: 16 x 4096 x 8192 15.1 us with one set, 13.3 with two; 16
    // x 4096 x 4096 9.6 with one, 11.4 with two.  From 17 rows on four sets
    // need a workgroup per CU (40 x 4096 x 16384 28.7 us against 32.4 with two
    // and 36.5 in tiles); else two up to 32 rows (24 x 4096 x 8192 15.0 us, in
    // tiles 18.2), and tiles beyond (40 x 4096 x 8192 18.7 and 17.9).
    const size_t least = f == Form::GATED ? 2 : 1;
    auto groups = [&](size_t sets) {
      const size_t cols = 16 * sets / least;
      return (nj + cols - 1) / cols * ranks;
    };
    size_t sets = 0;
    if (ni <= 16)
      sets = groups(2 * least) >= (size_t)cus ? 2 * least : least;
    else if (groups(4) >= (size_t)cus)
      sets = 4;
    else if (ni <= 32)
      sets = 2;
    if (sets) {
      // Wavefronts per workgroup: 16 per CU in all (8 with more sets), half
      // of that once there are 4 and each has at most 4 chunks of 512 bytes.
      // 8 x 1 x 4096 x 2048 gated: 42.9 us with 4, 47.0 with 2, 45.7 with 8.
      const size_t chunks = nc * size_of(t) / 512;
      const size_t many = (size_t)cus * (sets > least ? 8 : 16);
      const size_t n = groups(sets);
      int w = 1;
      while (w < 8 && chunks >= (size_t)w * 2 &&
             (w < 4 ? n * w < many || chunks > (size_t)w * 4
                    : n * w < many / 2))
        w *= 2;
      return {w, (int)sets, 0, 1, 0, 0};
    }
  }
  const size_t kt = 128 / size_of(t);
  const size_t nk = (nc + kt - 1) / kt * (f == Form::DX ? pairs : 1);
  const size_t cells = ni * nj * ranks * (f == Form::DW ? pairs : 1) *
                       (f == Form::GATED ? 2 : 1);
  const TileCost* cost = t == Type::F32 ? (fast ? kFast32 : kSlow32)
                                        : fast ? kFast16 : kSlow16;
  Shape best = {0, 0, 0, 1, 0, 0};
  for (int tile = 0; tile < kTiles; ++tile) {
    if (!cost[tile].resident) continue;
    const size_t bm = kTileRows[tile],
                 bn = kTileCols[tile] / (f == Form::GATED ? 2 : 1);
    const double n = (double)((ni + bm - 1) / bm) * ((nj + bn - 1) / bn) *
                     ranks * (f == Form::DW ? pairs : 1);
    for (int s = 1; s <= (split ? 16 : 1); s += s < 4 ? 1 : s < 8 ? 2 : 4) {
      const size_t part = s > 1 ? (cells + (f == Form::DW ? ni * ranks * pairs
                                                          : 0)) * s * 4 : 0;
      if (s > 1 && (nk < (size_t)s * 2 || part > kMostPart)) break;
      const double wgs = n * s, steps = (double)((nk + s - 1) / s);
      const double turns = std::ceil(wgs / ((double)cus * cost[tile].resident));
      const double per = std::ceil(wgs / cus);
      double ns = kStartNs + steps * std::max(turns * cost[tile].alone,
                                              per * cost[tile].rate);
      if (s > 1) ns += kJoinNs + part / kJoinRate;
      if (best.ns == 0 || ns < best.ns) best = {0, 0, tile, s, part, ns};
    }
  }
  return best;
}

// An operand of a product as it is stored: `mats` matrices per rank.
struct Stored {
  int mats;
  size_t rows, cols, ld;
  bool fast;
};

struct Step {
  Form form;
  int pairs;
  size_t ni, nj, nc;
  Stored a, b;
};

// How a product runs, operands copied first (`copy_*`) or not.
struct Plan {
  Shape shape;
  bool fast, copy_a, copy_b;
  size_t ld_a, ld_b, bytes_a, bytes_b;   // of the copies
  size_t bytes() const { return bytes_a + bytes_b + shape.part; }
};

// Operands off 16 bytes are read at a third of the rate of aligned ones (38
// against 114 GB/s per CU from L2), again by every tile.  With enough reuse it
// pays to copy them once into the workspace, rows 128 bytes apart and filled
// with zeros, and to run the fast kernels: 2001 x 2001 x 2001 backward 160 ->
// 83 us.
constexpr double kCopyNs = 4000, kCopyRate = 1900;   // bytes of the copy per ns

inline Plan plan_of(const Step& s, Type t, int ranks, int cus, size_t room) {
  const size_t e = size_of(t);
  Plan n = {};
  n.fast = s.a.fast && s.b.fast && s.nc != 0;
  n.shape = shape_of(s.form, t, ranks, s.pairs, s.ni, s.nj, s.nc, cus,
                     room != 0, n.fast);
  if (n.fast || n.shape.waves || !room || !s.nc || !s.ni || !s.nj) return n;
  Plan c = n;
  c.fast = true;
  c.shape = shape_of(s.form, t, ranks, s.pairs, s.ni, s.nj, s.nc, cus, true,
                     true);
  c.copy_a = !s.a.fast, c.copy_b = !s.b.fast;
  const size_t line = 128 / e;
  c.ld_a = (s.a.cols + line - 1) / line * line;
  c.ld_b = (s.b.cols + line - 1) / line * line;
  if (c.copy_a) c.bytes_a = s.a.mats * (size_t)ranks * s.a.rows * c.ld_a * e;
  if (c.copy_b) c.bytes_b = s.b.mats * (size_t)ranks * s.b.rows * c.ld_b * e;
  if (c.bytes_a + c.bytes_b > 2 * kMostPart || c.ld_a >= kFastPitch ||
      c.ld_b >= kFastPitch || c.bytes() > room)
    return n;
  const double ns =
      c.shape.ns + kCopyNs + (double)(c.bytes_a + c.bytes_b) / kCopyRate;
  return ns < n.shape.ns ? c : n;
}

// The products of a call.
inline int steps_of(dpar_product_call_t call, const dpar_product_t& o, Type t,
             bool dx, bool dw, Step* s) {
  const size_t e = size_of(t);
  auto stored = [&](int mats, size_t rows, size_t cols, size_t ld) {
    const bool fast = rows && cols && cols * e % 16 == 0 &&
                      (rows == 1 || ld * e % 16 == 0) && ld < kFastPitch;
    return Stored{mats, rows, cols, ld, fast};
  };
  const bool gated = call == DPAR_GATED || call == DPAR_GATED_BACKWARD;
  const int m = gated ? 2 : 1;
  const Stored x = stored(1, o.rows, o.in, o.ldx),
               w = stored(m, o.out, o.in, o.ldw);
  int n = 0;
  switch (call) {
    case DPAR_LINEAR:
      s[n++] = {Form::LINEAR, 1, o.rows, o.out, o.in, x, w};
      break;
    case DPAR_GATED:
      s[n++] = {Form::GATED, 1, o.rows, o.out, o.in, x, w};
      break;
    default: {
      const bool slope = gated || o.act != DPAR_ACT_NONE;
      const Stored dz = stored(m, o.rows, o.out, slope ? o.ldz : o.ldy);
      if (dx) s[n++] = {Form::DX, m, o.rows, o.in, o.out, dz, w};
      if (dw) s[n++] = {Form::DW, m, o.out, o.in, o.rows, dz, x};
    }
  }
  return n;
}

// Bias gradients that the slopes' kernel sums (rounded slopes, 16-bit types):
// in how many parts of the rows, and the workspace of their sums.  Workgroups
// take 128 bytes of the columns, 64 rows at a time; where these are fewer than
// two per CU they share the rows, 64 at least to each, and dw's kernel joins
// the parts (2 x 129 x 1000 x 1363 gated fp16 37.7 us, with 128 rows to each
// 41.4).
struct SumPlan {
  int parts;
  size_t bytes;
};
inline bool sums_apart(Type t, bool slope) { return t != Type::F32 && slope; }
inline SumPlan sums_of(int p, int pairs, size_t rows, size_t out, int cus) {
  const size_t cols = dpar::products::kSumLine / 2;
  const size_t n = (out + cols - 1) / cols * ranks_per_launch(p),
               most = (size_t)cus * 2;
  const size_t parts =
      n ? std::min(std::min(most / n, rows / 64), (size_t)64) : 0;
  if (parts < 2) return {1, 0};
  const size_t bytes = parts * p * pairs * out * 4;
  return {(int)parts, (bytes + 127) / 128 * 128};
}

// Workspace of a call: its bias gradients', then its products' (in turn).
inline size_t workspace_of(dpar_product_call_t call, Type t, int p,
                    const dpar_product_t& o, int cus) {
  Step s[2];
  const int n = steps_of(call, o, t, true, true, s);
  const size_t any = ~(size_t)0;
  size_t most = 0;
  for (int k = 0; k < n; ++k) {
    most = std::max(most, plan_of(s[k], t, ranks_per_launch(p), cus,
                                  any).bytes());
    // also without copies (operands off 16 bytes at the call)
    s[k].a.fast = s[k].b.fast = false;
    const Shape slow = shape_of(s[k].form, t, ranks_per_launch(p), s[k].pairs,
                                s[k].ni, s[k].nj, s[k].nc, cus, true, false);
    most = std::max(most, slow.part);
  }
  const bool gated = call == DPAR_GATED_BACKWARD;
  if ((gated || call == DPAR_LINEAR_BACKWARD) &&
      sums_apart(t, gated || o.act != DPAR_ACT_NONE))
    most += sums_of(p, gated ? 2 : 1, o.rows, o.out, cus).bytes;
  return most;
}

// Whether a row of rank i's matrix has a byte in [lo, hi).
inline bool touches(const Mat& m, int i, uintptr_t lo, uintptr_t hi) {
  const uintptr_t a = (uintptr_t)m.at[i];
  if (!a || !m.extent() || a >= hi || a + m.extent() <= lo) return false;
  const size_t pitch = m.rows > 1 ? m.ld * m.esz : m.extent();
  // the last row that starts at or before lo (the first, if none does); what
  // it leaves, the next one's start decides
  const size_t r = lo > a ? (lo - a) / pitch : 0;
  const uintptr_t row = a + r * pitch;
  if (row < hi && row + m.cols * m.esz > lo) return true;
  return r + 1 < m.rows && row + pitch < hi;
}

inline int check_workspace(const char* call, dpar_product_call_t which, Type t, int p,
                    const dpar_product_t& o, const Mat* mats, int n, void* ws,
                    size_t bytes, int* cus) {
  *cus = cu_count();
  if (!ws) return DPAR_SUCCESS;
  const size_t need = workspace_of(which, t, p, o, *cus);
  if (bytes < need)
    return fail(DPAR_ERR_INVALID_ARG, "%s: workspace of %zu bytes, %zu needed",
                call, bytes, need);
  if ((uintptr_t)ws & 15)
    return fail(DPAR_ERR_INVALID_ARG, "%s: workspace not on 16 bytes", call);
  const uintptr_t lo = (uintptr_t)ws, hi = lo + need;
  if (need && (hi >> 48 || hi < lo))
    return fail(DPAR_ERR_UNSUPPORTED, "%s: workspace above 2^48", call);
  for (int k = 0; k < n && need; ++k)
    for (int i = 0; i < p && mats[k].used; ++i)
      if (touches(mats[k], i, lo, hi))
        return fail(DPAR_ERR_ALIAS, "%s: workspace overlaps %s of rank %d",
                    call, mats[k].name, i);
  return DPAR_SUCCESS;
}

inline int launched(const char* call, hipError_t e) {
  if (e == hipSuccess) return DPAR_SUCCESS;
  return fail(DPAR_ERR_HIP, "%s: %s", call, hipGetErrorString(e));
}

// Copies one operand of a launch's ranks and points the launch at the copies.
// One matrix read by every rank is copied once.
inline void add_copy(dpar::products::CopyArgs* c, const Stored& m, int ranks,
              size_t e, const void* (*at)[kRanks], size_t ld, char* to) {
  for (int k = 0; k < m.mats; ++k) {
    int n = 1;
    for (int r = 1; r < ranks; ++r)
      if (at[k][r] != at[k][0]) n = ranks;
    auto& job = c->job[c->jobs++];
    const size_t unit = e == 1 ? 1 : 2;
    job.rows = m.rows, job.cols = m.cols * e / unit, job.ld = m.ld * e / unit;
    job.pitch = ld * e, job.mats = n;
    job.to = to;
    const size_t one = m.rows * ld * e;
    for (int r = 0; r < ranks; ++r) {
      job.from[r] = at[k][r];
      at[k][r] = to + (n == 1 ? 0 : r * one);
    }
    to += n * one;
  }
}

// Whether calls print their plans.
inline bool logs() {
  const char* log = std::getenv("DPAR_LOG");
  return log && std::atoi(log) != 0;
}

// DPAR_LOG=1: one line per product on stderr with the kernel that runs.
inline void log_plan(const Step& s, Type t, int ranks, const Plan& n) {
  static const char* forms[] = {"linear", "gated", "dx", "dw"};
  std::fprintf(stderr,
               "dpar: product=%s %s ranks=%d rows=%zu cols=%zu sum=%zu "
               "pairs=%d operands=%s",
               forms[(int)s.form],
               name_of(t),
               ranks, s.ni, s.nj, s.nc, s.pairs,
               n.copy_a || n.copy_b ? "copied" : n.fast ? "aligned"
                                                        : "unaligned");
  if (n.shape.waves)
    std::fprintf(stderr, " kernel=few sets=%d waves=%d\n", n.shape.sets,
                 n.shape.waves);
  else
    std::fprintf(stderr, " kernel=%zux%zu%s splits=%d\n",
                 kTileRows[n.shape.tile], kTileCols[n.shape.tile],
                 n.shape.tile == 1 ? "x4" : "", n.shape.splits);
}

// Runs one product over all ranks.  a: everything but the addresses, which
// `fill` writes for a rank; s: the product with its operands' alignment.
// `launch` and `copy` start the kernels of the operands' type.
template <typename Launch, typename Copy, typename Fill>
int run_product(const char* call, Type t, int p, const Step& s, Args* a,
                void* ws, size_t bytes, int cus, hipStream_t stream,
                Launch launch, Copy copy, Fill fill) {
  const int per = ranks_per_launch(p);
  const Plan n = plan_of(s, t, per, cus, ws ? bytes : 0);
  const size_t e = size_of(t);
  if (logs()) log_plan(s, t, per, n);
  a->ni = s.ni, a->nj = s.nj, a->nc = s.nc;
  a->pairs = s.pairs;
  a->lda = n.copy_a ? n.ld_a : s.a.ld;
  a->ldb = n.copy_b ? n.ld_b : s.b.ld;
  // values that may be loaded along a row of results' operands
  a->na = n.copy_a && s.form == Form::DW ? n.ld_a : s.ni;
  a->nb = n.copy_b && (s.form == Form::DW || s.form == Form::DX) ? n.ld_b
                                                                 : s.nj;
  a->fast = n.fast;
  a->waves = n.shape.waves;
  a->sets = n.shape.sets;
  a->tile = n.shape.tile;
  a->splits = n.shape.splits;
  char* const work = (char*)ws;
  a->part = (float*)(work + n.bytes_a + n.bytes_b);
  for (int r0 = 0; r0 < p; r0 += per) {
    a->ranks = std::min(per, p - r0);
    for (int k = 0; k < a->ranks; ++k) fill(k, r0 + k);
    if (n.copy_a || n.copy_b) {
      dpar::products::CopyArgs c = {};
      if (n.copy_a) add_copy(&c, s.a, a->ranks, e, a->a, n.ld_a, work);
      if (n.copy_b)
        add_copy(&c, s.b, a->ranks, e, a->b, n.ld_b, work + n.bytes_a);
      const int rc = launched(call, copy(c, stream));
      if (rc) return rc;
    }
    const int rc = launched(call, launch(s.form, *a, stream));
    if (rc) return rc;
  }
  return DPAR_SUCCESS;
}

template <typename Body>
int guarded(const char* call, Body body) {
  try {
    return body();
  } catch (const std::bad_alloc&) {
    return fail(DPAR_ERR_NOMEM, "%s: out of host memory", call);
  } catch (...) {
    return fail(DPAR_ERR_HIP, "%s: unexpected failure", call);
  }
}

// Addresses of the array arguments as the checks take them.
inline const void* const* in_array(void* const* a) { return (const void* const*)a; }

}  // namespace
