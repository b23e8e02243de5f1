// C entry points of the layer products: argument and alias checks, the rules
// that choose a kernel, launches of at most kRanks ranks.
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

int fail(int code, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
int fail(int code, const char* fmt, ...) {
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
bool share(const Range& a, const Range& b) {
  if (a.pitch == b.pitch && a.pitch != 0) {
    const size_t d = (b.lo - a.lo) % a.pitch;   // b.lo >= a.lo
    if (d >= a.width && d + b.width <= a.pitch) return false;
  }
  return true;
}

int check_alias(const Mat* mats, int n, int p, const char* call) {
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

int check_mats(const Mat* mats, int n, int p, const char* call) {
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

constexpr size_t kMost = (size_t)1 << 31;     // rows, in, out
constexpr size_t kMostPitch = (size_t)1 << 38;

// The options with row distances filled in.
int check_options(const char* call, int p, const dpar_product_t* opt,
                  dpar_product_t* o, Type* t, size_t* esz, size_t* osz) {
  dpar::set_error(0, "");
  if (p < 1) return fail(DPAR_ERR_INVALID_ARG, "%s: p must be >= 1", call);
  if (!opt) return fail(DPAR_ERR_INVALID_ARG, "%s: null options", call);
  *o = *opt;
  switch (o->dtype) {
    case DPAR_FLOAT32: *t = Type::F32; break;
    case DPAR_BFLOAT16: *t = Type::BF16; break;
    case DPAR_FLOAT16: *t = Type::F16; break;
    default:
      return fail(DPAR_ERR_UNSUPPORTED, "%s: dtype %d", call, (int)o->dtype);
  }
  if (o->out_dtype != o->dtype && o->out_dtype != DPAR_FLOAT32)
    return fail(DPAR_ERR_UNSUPPORTED, "%s: out_dtype %d with dtype %d", call,
                (int)o->out_dtype, (int)o->dtype);
  if ((int)o->act < DPAR_ACT_NONE || (int)o->act > DPAR_ACT_SILU)
    return fail(DPAR_ERR_INVALID_ARG, "%s: unknown activation %d", call,
                (int)o->act);
  if (o->rows >= kMost || o->in >= kMost || o->out >= kMost)
    return fail(DPAR_ERR_UNSUPPORTED, "%s: a size beyond 2^31", call);
  *esz = o->dtype == DPAR_FLOAT32 ? 4 : 2;
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
int cu_count() {
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
int ranks_per_launch(int p) {
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
// operands have no four-buffer form.
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

Shape shape_of(Form f, Type t, int ranks, int pairs, size_t ni, size_t nj,
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
      const size_t chunks = nc / (t == Type::F32 ? 128 : 256);
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
  const size_t kt = t == Type::F32 ? 32 : 64;
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

Plan plan_of(const Step& s, Type t, int ranks, int cus, size_t room) {
  const size_t e = t == Type::F32 ? 4 : 2;
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
int steps_of(dpar_product_call_t call, const dpar_product_t& o, Type t,
             bool dx, bool dw, Step* s) {
  const size_t e = t == Type::F32 ? 4 : 2;
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
bool sums_apart(Type t, bool slope) { return t != Type::F32 && slope; }
SumPlan sums_of(int p, int pairs, size_t rows, size_t out, int cus) {
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
size_t workspace_of(dpar_product_call_t call, Type t, int p,
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
bool touches(const Mat& m, int i, uintptr_t lo, uintptr_t hi) {
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

int check_workspace(const char* call, dpar_product_call_t which, Type t, int p,
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

int launched(const char* call, hipError_t e) {
  if (e == hipSuccess) return DPAR_SUCCESS;
  return fail(DPAR_ERR_HIP, "%s: %s", call, hipGetErrorString(e));
}

// Copies one operand of a launch's ranks and points the launch at the copies.
// One matrix read by every rank is copied once.
void add_copy(dpar::products::CopyArgs* c, const Stored& m, int ranks,
              size_t e, const void* (*at)[kRanks], size_t ld, char* to) {
  for (int k = 0; k < m.mats; ++k) {
    int n = 1;
    for (int r = 1; r < ranks; ++r)
      if (at[k][r] != at[k][0]) n = ranks;
    auto& job = c->job[c->jobs++];
    job.rows = m.rows, job.cols = m.cols * e / 2, job.ld = m.ld * e / 2;
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

// DPAR_LOG=1: one line per product on stderr with the kernel that runs.
void log_plan(const Step& s, Type t, int ranks, const Plan& n) {
  static const char* forms[] = {"linear", "gated", "dx", "dw"};
  std::fprintf(stderr,
               "dpar: product=%s %s ranks=%d rows=%zu cols=%zu sum=%zu "
               "pairs=%d operands=%s",
               forms[(int)s.form],
               t == Type::F32 ? "float32" : t == Type::BF16 ? "bfloat16"
                                                            : "float16",
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
template <typename Fill>
int run_product(const char* call, Type t, int p, const Step& s, Args* a,
                void* ws, size_t bytes, int cus, hipStream_t stream,
                Fill fill) {
  const int per = ranks_per_launch(p);
  const Plan n = plan_of(s, t, per, cus, ws ? bytes : 0);
  const size_t e = t == Type::F32 ? 4 : 2;
  const char* log = std::getenv("DPAR_LOG");
  if (log && std::atoi(log) != 0) log_plan(s, t, per, n);
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
      const int rc = launched(call, dpar::products::launch_copy(c, stream));
      if (rc) return rc;
    }
    hipError_t err;
    switch (t) {
      case Type::BF16:
        err = dpar::products::launch_bf16(s.form, *a, stream);
        break;
      case Type::F16:
        err = dpar::products::launch_f16(s.form, *a, stream);
        break;
      default: err = dpar::products::launch_f32(s.form, *a, stream);
    }
    const int rc = launched(call, err);
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
const void* const* in_array(void* const* a) { return (const void* const*)a; }

int linear_impl(const void* const* x, const void* const* w,
                const void* const* bias, const void* const* residual,
                void* const* y, void* const* z, int p,
                const dpar_product_t* opt, void* ws, size_t bytes,
                hipStream_t stream) {
  const char* call = "dpar_linear";
  dpar_product_t o;
  Type t;
  size_t e, eo;
  int rc = check_options(call, p, opt, &o, &t, &e, &eo);
  if (rc) return rc;
  Mat m[] = {
      {"x", x, o.rows, o.in, o.ldx, e, false, false, true},
      {"w", w, o.out, o.in, o.ldw, e, false, false, true},
      {"bias", bias, 1, o.out, o.out, e, false, true, bias != nullptr},
      {"residual", residual, o.rows, o.out, o.ldr, eo, false, true,
       residual != nullptr},
      {"y", in_array(y), o.rows, o.out, o.ldy, eo, true, false, true},
      {"z", in_array(z), o.rows, o.out, o.ldz, e, true, false, z != nullptr}};
  // (each thread reads the residuals of its results before it stores these)
  m[4].twin[0] = residual;
  if ((rc = check_mats(m, 6, p, call))) return rc;
  int cus;
  if ((rc = check_workspace(call, DPAR_LINEAR, t, p, o, m, 6, ws, bytes,
                            &cus)))
    return rc;
  if (!o.rows || !o.out) return DPAR_SUCCESS;
  Args a = {};
  a.ldo = o.ldy, a.ldk = o.ldz, a.lde = o.ldr;
  a.act = o.act, a.out32 = eo == 4;
  Step s;
  steps_of(DPAR_LINEAR, o, t, false, false, &s);
  s.a.fast = m[0].fast(p), s.b.fast = m[1].fast(p);
  a.wide_out = m[2].aligned(p) && m[3].aligned(p) && m[4].aligned(p) &&
               m[5].aligned(p);
  return run_product(call, t, p, s, &a, ws, bytes, cus, stream,
                     [&](int k, int i) {
                       a.a[0][k] = m[0].rank(i);
                       a.b[0][k] = m[1].rank(i);
                       a.e[0][k] = m[2].rank(i);
                       a.e[1][k] = m[3].rank(i);
                       a.o[0][k] = (void*)m[4].rank(i);
                       a.o[1][k] = (void*)m[5].rank(i);
                     });
}

int gated_impl(const void* const* x, const void* const* wg,
               const void* const* wu, const void* const* bg,
               const void* const* bu, void* const* h, void* const* g,
               void* const* u, int p, const dpar_product_t* opt, void* ws,
               size_t bytes, hipStream_t stream) {
  const char* call = "dpar_gated";
  dpar_product_t o;
  Type t;
  size_t e, eo;
  int rc = check_options(call, p, opt, &o, &t, &e, &eo);
  if (rc) return rc;
  if (!g != !u)
    return fail(DPAR_ERR_INVALID_ARG, "%s: g without u or u without g", call);
  const Mat m[] = {
      {"x", x, o.rows, o.in, o.ldx, e, false, false, true},
      {"wg", wg, o.out, o.in, o.ldw, e, false, false, true},
      {"wu", wu, o.out, o.in, o.ldw, e, false, false, true},
      {"bg", bg, 1, o.out, o.out, e, false, true, bg != nullptr},
      {"bu", bu, 1, o.out, o.out, e, false, true, bu != nullptr},
      {"h", in_array(h), o.rows, o.out, o.ldy, eo, true, false, true},
      {"g", in_array(g), o.rows, o.out, o.ldz, e, true, false, g != nullptr},
      {"u", in_array(u), o.rows, o.out, o.ldz, e, true, false, u != nullptr}};
  if ((rc = check_mats(m, 8, p, call))) return rc;
  int cus;
  if ((rc = check_workspace(call, DPAR_GATED, t, p, o, m, 8, ws, bytes,
                            &cus)))
    return rc;
  if (!o.rows || !o.out) return DPAR_SUCCESS;
  Args a = {};
  a.ldo = o.ldy, a.ldk = o.ldz;
  a.act = o.act, a.out32 = eo == 4;
  Step s;
  steps_of(DPAR_GATED, o, t, false, false, &s);
  s.a.fast = m[0].fast(p), s.b.fast = m[1].fast(p) && m[2].fast(p);
  a.wide_out = m[3].aligned(p) && m[4].aligned(p) && m[5].aligned(p) &&
               m[6].aligned(p) && m[7].aligned(p);
  return run_product(call, t, p, s, &a, ws, bytes, cus, stream,
                     [&](int k, int i) {
                       a.a[0][k] = m[0].rank(i);
                       a.b[0][k] = m[1].rank(i);
                       a.b[1][k] = m[2].rank(i);
                       a.e[0][k] = m[3].rank(i);
                       a.e[1][k] = m[4].rank(i);
                       a.o[0][k] = (void*)m[5].rank(i);
                       a.o[1][k] = (void*)m[6].rank(i);
                       a.u[0][k] = (void*)m[7].rank(i);
                     });
}

hipError_t launch_slope(Type t, const SlopeArgs& a, hipStream_t stream) {
  switch (t) {
    case Type::BF16: return dpar::products::launch_slope_bf16(a, stream);
    case Type::F16: return dpar::products::launch_slope_f16(a, stream);
    default: return dpar::products::launch_slope_f32(a, stream);
  }
}

hipError_t launch_sums(Type t, const SumArgs& a, hipStream_t stream) {
  return t == Type::BF16 ? dpar::products::launch_sums_bf16(a, stream)
                         : dpar::products::launch_sums_f16(a, stream);
}

// Both backward calls; pairs: 1 (dpar_linear_backward) or 2.
struct Back {
  const void* const* dy;
  const void* const* x;
  const void* const* w[2];
  const void* const* z[2];     // z; g, u
  void* const* dx;
  void* const* dw[2];
  void* const* db[2];
  void* const* dz[2];
};

int backward_impl(const char* call, int pairs, const Back& b, int p,
                  const dpar_product_t* opt, void* ws, size_t bytes,
                  hipStream_t stream) {
  dpar_product_t o;
  Type t;
  size_t e, eo;
  int rc = check_options(call, p, opt, &o, &t, &e, &eo);
  if (rc) return rc;
  const bool gated = pairs == 2;
  const bool slope = gated || o.act != DPAR_ACT_NONE;
  const bool dx = b.dx != nullptr, dw = b.dw[0] != nullptr,
             db = b.db[0] != nullptr;
  if (gated && (!b.dw[0] != !b.dw[1] || !b.db[0] != !b.db[1]))
    return fail(DPAR_ERR_INVALID_ARG, "%s: the gradients of one projection "
                "without the other's", call);
  if (db && !dw)
    return fail(DPAR_ERR_UNSUPPORTED, "%s: bias gradients without the weights' "
                "gradients", call);
  static const char* names[2][4] = {{"w", "z", "dz", "dw"},
                                    {"wg", "g", "dg", "dwg"}};
  static const char* names2[4] = {"wu", "u", "du", "dwu"};
  const char* const* n1 = names[gated];
  Mat m[14] = {
      {gated ? "dh" : "dy", b.dy, o.rows, o.out, o.ldy, e, false, false, true},
      {"x", b.x, o.rows, o.in, o.ldx, e, false, false, dw},
      {n1[0], b.w[0], o.out, o.in, o.ldw, e, false, false, dx},
      {names2[0], b.w[1], o.out, o.in, o.ldw, e, false, false, dx && gated},
      {n1[1], b.z[0], o.rows, o.out, o.ldz, e, false, false, slope},
      {names2[1], b.z[1], o.rows, o.out, o.ldz, e, false, false, gated},
      {n1[2], in_array(b.dz[0]), o.rows, o.out, o.ldz, e, true, false, slope},
      {names2[2], in_array(b.dz[1]), o.rows, o.out, o.ldz, e, true, false,
       gated},
      {"dx", in_array(b.dx), o.rows, o.in, o.lddx, eo, true, false, dx},
      {n1[3], in_array(b.dw[0]), o.out, o.in, o.lddw, eo, true, false, dw},
      {names2[3], in_array(b.dw[1]), o.out, o.in, o.lddw, eo, true, false,
       dw && gated},
      {gated ? "dbg" : "dbias", in_array(b.db[0]), 1, o.out, o.out, eo, true,
       false, db},
      {"dbu", in_array(b.db[1]), 1, o.out, o.out, eo, true, false,
       db && gated}};
  constexpr int kMats = 13;
  m[6].twin[0] = b.z[0], m[6].twin[1] = b.dy;
  if (gated) m[7].twin[0] = b.z[1];
  if ((rc = check_mats(m, kMats, p, call))) return rc;
  int cus;
  if ((rc = check_workspace(call,
                            gated ? DPAR_GATED_BACKWARD : DPAR_LINEAR_BACKWARD,
                            t, p, o, m, kMats, ws, bytes, &cus)))
    return rc;

  const bool apart = db && sums_apart(t, slope);
  const float* parts_at = nullptr;
  int parts = 1;
  if (o.out && (apart || (slope && o.rows))) {
    SumArgs q = {};
    SlopeArgs& s = q.s;
    s.rows = o.rows, s.cols = o.out, s.ldy = o.ldy, s.ldz = o.ldz;
    s.act = o.act, s.gated = gated;
    s.wide = m[0].aligned(p);
    for (int k = 4; k < 8; ++k) s.wide &= m[k].aligned(p);
    q.out32 = eo == 4, q.all = p, q.parts = 1;
    if (apart && ws && o.in) {
      const SumPlan n = sums_of(p, pairs, o.rows, o.out, cus);
      q.parts = parts = n.parts, q.part = (float*)ws;
      if (parts > 1) parts_at = q.part;
      ws = (char*)ws + n.bytes, bytes -= n.bytes;
    }
    const int per = ranks_per_launch(p);
    for (int r0 = 0; r0 < p; r0 += per) {
      s.ranks = std::min(per, p - r0), q.first = r0;
      for (int k = 0; k < s.ranks; ++k) {
        s.dy[k] = m[0].rank(r0 + k);
        s.z[k] = m[4].rank(r0 + k);
        s.u[k] = m[5].rank(r0 + k);
        s.dz[k] = (void*)m[6].rank(r0 + k);
        s.du[k] = (void*)m[7].rank(r0 + k);
        q.db[0][k] = (void*)m[11].rank(r0 + k);
        q.db[1][k] = (void*)m[12].rank(r0 + k);
      }
      if ((rc = launched(call, apart ? launch_sums(t, q, stream)
                                     : launch_slope(t, s, stream))))
        return rc;
    }
  }
  // with no activation the products read dy itself
  const Mat& d0 = slope ? m[6] : m[0];
  const Mat& d1 = m[7];
  const dpar_product_call_t which =
      gated ? DPAR_GATED_BACKWARD : DPAR_LINEAR_BACKWARD;
  const bool dz_fast = d0.fast(p) && d1.fast(p);
  if (dx && o.rows && o.in) {
    Args a = {};
    a.ldo = o.lddx, a.out32 = eo == 4;
    a.wide_out = m[8].aligned(p);
    Step s;
    steps_of(which, o, t, true, false, &s);
    s.a.fast = dz_fast, s.b.fast = m[2].fast(p) && m[3].fast(p);
    rc = run_product(call, t, p, s, &a, ws, bytes, cus, stream,
                     [&](int k, int i) {
                       a.a[0][k] = d0.rank(i);
                       a.a[1][k] = d1.rank(i);
                       a.b[0][k] = m[2].rank(i);
                       a.b[1][k] = m[3].rank(i);
                       a.o[0][k] = (void*)m[8].rank(i);
                     });
    if (rc) return rc;
  }
  if (dw && o.out && (o.in || (db && !apart))) {
    Args a = {};
    a.ldo = o.lddw, a.out32 = eo == 4, a.sums = db && !apart;
    a.sum = parts_at, a.parts = parts, a.all = p;
    a.wide_out = m[9].aligned(p) && m[10].aligned(p);
    Step s;
    steps_of(which, o, t, false, true, &s);
    s.a.fast = dz_fast, s.b.fast = m[1].fast(p);
    rc = run_product(call, t, p, s, &a, ws, bytes, cus, stream,
                     [&](int k, int i) {
                       a.a[0][k] = d0.rank(i);
                       a.a[1][k] = d1.rank(i);
                       a.b[0][k] = m[1].rank(i);
                       a.o[0][k] = (void*)m[9].rank(i);
                       a.o[1][k] = (void*)m[10].rank(i);
                       if (k == 0) a.first = i;
                       if (!a.sums && !a.sum) return;
                       a.u[0][k] = (void*)m[11].rank(i);
                       a.u[1][k] = (void*)m[12].rank(i);
                     });
    if (rc) return rc;
  }
  return DPAR_SUCCESS;
}

}  // namespace

extern "C" {

int dpar_linear(const void* const* x, const void* const* w,
                const void* const* bias, const void* const* residual,
                void* const* y, void* const* z, int p,
                const dpar_product_t* opt, void* workspace,
                size_t workspace_bytes, hipStream_t stream) {
  return guarded("dpar_linear", [&] {
    return linear_impl(x, w, bias, residual, y, z, p, opt, workspace,
                       workspace_bytes, stream);
  });
}

int dpar_linear_backward(const void* const* dy, const void* const* x,
                         const void* const* w, const void* const* z,
                         void* const* dx, void* const* dw, void* const* dbias,
                         void* const* dz, int p, const dpar_product_t* opt,
                         void* workspace, size_t workspace_bytes,
                         hipStream_t stream) {
  return guarded("dpar_linear_backward", [&] {
    const Back b = {dy, x, {w, nullptr}, {z, nullptr}, dx, {dw, nullptr},
                    {dbias, nullptr}, {dz, nullptr}};
    return backward_impl("dpar_linear_backward", 1, b, p, opt, workspace,
                         workspace_bytes, stream);
  });
}

int dpar_gated(const void* const* x, const void* const* wg,
               const void* const* wu, const void* const* bg,
               const void* const* bu, void* const* h, void* const* g,
               void* const* u, int p, const dpar_product_t* opt,
               void* workspace, size_t workspace_bytes, hipStream_t stream) {
  return guarded("dpar_gated", [&] {
    return gated_impl(x, wg, wu, bg, bu, h, g, u, p, opt, workspace,
                      workspace_bytes, stream);
  });
}

int dpar_gated_backward(const void* const* dh, const void* const* x,
                        const void* const* wg, const void* const* wu,
                        const void* const* g, const void* const* u,
                        void* const* dx, void* const* dwg, void* const* dwu,
                        void* const* dbg, void* const* dbu, void* const* dg,
                        void* const* du, int p, const dpar_product_t* opt,
                        void* workspace, size_t workspace_bytes,
                        hipStream_t stream) {
  return guarded("dpar_gated_backward", [&] {
    const Back b = {dh, x, {wg, wu}, {g, u}, dx, {dwg, dwu}, {dbg, dbu},
                    {dg, du}};
    return backward_impl("dpar_gated_backward", 2, b, p, opt, workspace,
                         workspace_bytes, stream);
  });
}

int dpar_product_workspace(dpar_product_call_t call, int p,
                           const dpar_product_t* opt, size_t* bytes) {
  return guarded("dpar_product_workspace", [&] {
    const char* name = "dpar_product_workspace";
    dpar_product_t o;
    Type t;
    size_t e, eo;
    const int rc = check_options(name, p, opt, &o, &t, &e, &eo);
    if (rc) return rc;
    if ((int)call < DPAR_LINEAR || (int)call > DPAR_GATED_BACKWARD)
      return fail(DPAR_ERR_INVALID_ARG, "%s: unknown call %d", name,
                  (int)call);
    if (!bytes) return fail(DPAR_ERR_INVALID_ARG, "%s: null result", name);
    *bytes = workspace_of(call, t, p, o, cu_count());
    return (int)DPAR_SUCCESS;
  });
}

}  // extern "C"
