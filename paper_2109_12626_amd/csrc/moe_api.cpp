// C entry points of the mixture-of-experts layer.
#include "moe.hpp"
#include "products_host.hpp"

namespace {

namespace moe = dpar::moe;

struct Options {
  dpar_moe_t o;              // with distances filled in
  Type t, w;
  size_t e, ew, eo, all;     // element sizes; experts of all ranks
};

int check_moe(const char* call, int p, const dpar_moe_t* opt, Options* c) {
  dpar::set_error(0, "");
  if (p < 1) return fail(DPAR_ERR_INVALID_ARG, "%s: p must be >= 1", call);
  if (!opt) return fail(DPAR_ERR_INVALID_ARG, "%s: null options", call);
  dpar_moe_t& o = c->o = *opt;
  switch (o.dtype) {
    case DPAR_FLOAT32: c->t = Type::F32; break;
    case DPAR_BFLOAT16: c->t = Type::BF16; break;
    case DPAR_FLOAT16: c->t = Type::F16; break;
    default:
      return fail(DPAR_ERR_UNSUPPORTED, "%s: dtype %d", call, (int)o.dtype);
  }
  c->w = c->t;
  if (o.weight_dtype == DPAR_INT8 && c->t != Type::F32)
    c->w = Type::I8;
  else if (o.weight_dtype != o.dtype)
    return fail(DPAR_ERR_UNSUPPORTED, "%s: weight_dtype %d with dtype %d", call,
                (int)o.weight_dtype, (int)o.dtype);
  if (o.out_dtype != o.dtype && o.out_dtype != DPAR_FLOAT32)
    return fail(DPAR_ERR_UNSUPPORTED, "%s: out_dtype %d with dtype %d", call,
                (int)o.out_dtype, (int)o.dtype);
  if ((int)o.act < DPAR_ACT_NONE || (int)o.act > DPAR_ACT_SILU)
    return fail(DPAR_ERR_INVALID_ARG, "%s: unknown activation %d", call,
                (int)o.act);
  if ((int)o.route < DPAR_ROUTE_SOFTMAX || (int)o.route > DPAR_ROUTE_SIGMOID)
    return fail(DPAR_ERR_INVALID_ARG, "%s: unknown route %d", call,
                (int)o.route);
  if (o.experts < 1 || o.top < 1)
    return fail(DPAR_ERR_INVALID_ARG, "%s: no experts, or none chosen", call);
  if (o.tokens > (size_t)moe::kTokens || o.top > moe::kTop ||
      o.experts > (size_t)moe::kExperts ||
      o.experts * p > (size_t)moe::kExperts)
    return fail(DPAR_ERR_UNSUPPORTED, "%s: %zu tokens, top %d, %d x %zu "
                "experts: beyond %d, %d, %d", call, o.tokens, o.top, p,
                o.experts, moe::kTokens, moe::kTop, moe::kExperts);
  c->all = o.experts * p;
  if ((size_t)o.top > c->all)
    return fail(DPAR_ERR_INVALID_ARG, "%s: %d chosen of %zu experts", call,
                o.top, c->all);
  if (o.in >= kMost || o.hidden >= kMost)
    return fail(DPAR_ERR_UNSUPPORTED, "%s: a size beyond 2^31", call);
  c->e = size_of(c->t), c->ew = size_of(c->w);
  c->eo = o.out_dtype == DPAR_FLOAT32 ? 4 : 2;
  if (!o.ldx || o.tokens <= 1) o.ldx = o.in;
  if (!o.ldl || o.tokens <= 1) o.ldl = c->all;
  if (!o.ldy || o.tokens <= 1) o.ldy = o.in;
  if (!o.ldr || o.tokens <= 1) o.ldr = o.in;
  if (!o.ldw || o.hidden <= 1) o.ldw = o.in;
  if (!o.ldd || o.in <= 1) o.ldd = o.hidden;
  for (size_t v : {o.ldx, o.ldl, o.ldw, o.ldd, o.ldy, o.ldr, o.xw, o.xd})
    if (v > kMostPitch)
      return fail(DPAR_ERR_UNSUPPORTED, "%s: a distance beyond 2^38", call);
  // (16 rows of a matrix lie within the kernels' 32-bit offsets)
  if (o.ldw >= kFastPitch || o.ldd >= kFastPitch)
    return fail(DPAR_ERR_UNSUPPORTED, "%s: rows of the weights 2^23 values or "
                "more apart", call);
  if (o.ldw < o.in || o.ldd < o.hidden)
    return fail(DPAR_ERR_INVALID_ARG, "%s: rows of the weights overlap", call);
  if (!o.xw || o.experts <= 1) o.xw = o.hidden * o.ldw;
  if (!o.xd || o.experts <= 1) o.xd = o.in * o.ldd;
  return DPAR_SUCCESS;
}

// Records of a table for the experts of `ranks` ranks.
int most_of(const dpar_moe_t& o, size_t ranks) {
  return (int)std::min(o.experts * ranks, o.tokens * (size_t)o.top);
}

int ranks_of(int p) {
  const int n = (p + moe::kRanks - 1) / moe::kRanks;
  return (p + n - 1) / n;
}

// Distance of the pairs' results, in 32-bit values.
size_t pitch_of(const dpar_moe_t& o) { return (o.in + 3) / 4 * 4; }

moe::Layout layout_of(const Options& c, int p) {
  const size_t pairs = c.o.tokens * c.o.top;
  auto up = [](size_t v) { return (v + 127) / 128 * 128; };
  moe::Layout l;
  l.records = up(moe::kStarts * 4);
  // (Mode::DIRECT: every expert has a record and room for all tokens)
  const size_t own = c.o.experts * ranks_of(p),
               direct = c.all <= (size_t)moe::kDirect ? own : 0;
  l.pairs = l.records +
            up(std::max((size_t)most_of(c.o, ranks_of(p)), direct) *
               sizeof(moe::Record));
  l.weights = l.pairs + up(std::max(pairs, direct * c.o.tokens) * 4);
  l.owner = l.weights + up(pairs * 4);
  l.hidden = l.owner + up(pairs * 4);
  // (room for the parts of 16-bit calls where y has 32 bits)
  l.parts = l.hidden + up(pairs * ((c.o.hidden + 31) / 32 * 32) *
                          (c.t != Type::F32 && c.eo == 4 ? 6 : 4));
  l.bytes = l.parts + up(pairs * pitch_of(c.o) * 4);
  return l;
}

// Wavefronts per workgroup, 2 or 4, for a matrix of `chunks` chunks of 512 bytes
// a row, with n workgroups that have work: 4 for 16 or more chunks (64 tokens, 2 of
// 8 experts 4096 x 4096 bf16: 141 us, with 2 in up 147, in down 158), else where two
// do not fill the card (100 tokens, a given 4 of 64 experts 2048 x 1024 bf16: 141
// us, with 4 in up 147; 64 tokens, 2 of 8 experts 2048 x 1024 fp32: 57, with 2 in up
// 75).
int waves_of(size_t n, size_t chunks, int cus) {
  return chunks >= 16 || (chunks >= 4 && n * 2 < (size_t)cus * 8) ? 4 : 2;
}

// DPAR_LOG=1: the layer, its choice and its kernels.
void log_layer(const Options& c, const moe::Args& a, int ranks) {
  std::fprintf(stderr,
               "dpar: moe %s weights=%s ranks=%d tokens=%d in=%zu hidden=%zu "
               "experts=%zu top=%d tables=%d choice=%s up=%dx%d waves=%d%s "
               "down=",
               name_of(c.t), name_of(c.w), ranks, a.tokens, a.in, a.hidden,
               c.all, a.top, a.tables,
               a.mode == (int)moe::Mode::FUSED    ? "fused"
               : a.mode == (int)moe::Mode::DIRECT ? "direct"
                                                  : "apart",
               a.tiles[0] * 16,
               16 * moe::columns_up(c.w, a.mode == (int)moe::Mode::FUSED,
                                    !a.fast[0], a.tiles[0]),
               a.waves[0], a.fast[0] ? "" : " unaligned");
  if (a.small)
    std::fprintf(stderr, "small%s\n", a.fast[1] ? "" : " unaligned");
  else
    std::fprintf(stderr, "%dx%d waves=%d%s\n", a.tiles[1] * 16, a.sets * 16,
                 a.waves[1], a.fast[1] ? "" : " unaligned");
}

int moe_impl(const void* const* x, const void* const* logits,
             const void* const* wg, const void* const* wu,
             const void* const* wd, const void* const* sg,
             const void* const* su, const void* const* sd,
             const void* const* residual, void* const* y, void* const* index,
             void* const* weight, int p, const dpar_moe_t* opt, void* ws,
             size_t bytes, hipStream_t stream) {
  const char* call = "dpar_moe";
  Options c;
  int rc = check_moe(call, p, opt, &c);
  if (rc) return rc;
  const dpar_moe_t& o = c.o;
  const bool eight = c.w == Type::I8, given = !logits;
  if (eight ? !sg || !su || !sd : sg || su || sd)
    return fail(DPAR_ERR_INVALID_ARG, "%s: scales belong to 8-bit weights, all "
                "three", call);
  if (given && (!index || !weight))
    return fail(DPAR_ERR_INVALID_ARG, "%s: neither logits nor a choice", call);
  const size_t n = o.experts, span_w = o.hidden ? (o.hidden - 1) * o.ldw + o.in
                                                : 0,
               span_d = o.in ? (o.in - 1) * o.ldd + o.hidden : 0;
  const size_t top = o.top;
  Mat m[] = {
      {"x", x, o.tokens, o.in, o.ldx, c.e, false, false, true},
      {"logits", logits, o.tokens, c.all, o.ldl, 4, false, false, !given},
      {"wg", wg, n, o.in ? span_w : 0, o.xw, c.ew, false, false, true},
      {"wu", wu, n, o.in ? span_w : 0, o.xw, c.ew, false, false, true},
      {"wd", wd, n, o.hidden ? span_d : 0, o.xd, c.ew, false, false, true},
      {"sg", sg, 1, n * o.hidden, n * o.hidden, 4, false, false, eight},
      {"su", su, 1, n * o.hidden, n * o.hidden, 4, false, false, eight},
      {"sd", sd, 1, n * o.in, n * o.in, 4, false, false, eight},
      {"residual", residual, o.tokens, o.in, o.ldr, c.eo, false, true,
       residual != nullptr},
      {"y", in_array(y), o.tokens, o.in, o.ldy, c.eo, true, false, true},
      {"index", in_array(index), o.tokens, top, top, 4, !given, !given,
       index != nullptr},
      {"weight", in_array(weight), o.tokens, top, top, 4, !given, !given,
       weight != nullptr}};
  constexpr int kMats = 12;
  m[9].twin[0] = residual;
  if ((rc = check_mats(m, kMats, p, call))) return rc;
  const moe::Layout at = layout_of(c, p);
  if (!o.tokens) return DPAR_SUCCESS;
  if (!ws || bytes < at.bytes * p)
    return fail(DPAR_ERR_INVALID_ARG, "%s: workspace of %zu bytes, %zu needed",
                call, ws ? bytes : 0, at.bytes * p);
  if ((uintptr_t)ws & 15)
    return fail(DPAR_ERR_INVALID_ARG, "%s: workspace not on 16 bytes", call);
  const uintptr_t lo = (uintptr_t)ws, hi = lo + at.bytes * p;
  if (hi >> 48 || hi < lo)
    return fail(DPAR_ERR_UNSUPPORTED, "%s: workspace above 2^48", call);
  for (int k = 0; k < kMats; ++k)
    for (int i = 0; i < p && m[k].used; ++i)
      if (touches(m[k], i, lo, hi))
        return fail(DPAR_ERR_ALIAS, "%s: workspace overlaps %s of rank %d",
                    call, m[k].name, i);

  const int cus = cu_count();
  const int per = ranks_of(p);
  moe::Args a = {};
  a.in = o.in, a.hidden = o.hidden;
  a.ldx = o.ldx, a.ldl = o.ldl, a.ldw = o.ldw, a.ldd = o.ldd;
  a.xw = o.xw, a.xd = o.xd, a.ldy = o.ldy, a.ldr = o.ldr;
  a.pitch = pitch_of(o);
  a.work = (char*)ws, a.at = at;
  a.scale = o.weight_scale;
  a.tokens = (int)o.tokens, a.experts = (int)o.experts, a.top = o.top;
  a.all = p;
  a.act = o.act, a.route = o.route, a.normalize = o.normalize != 0;
  a.given = given, a.out32 = c.eo == 4;
  // one table if all ranks make the same choice
  bool same = true;
  for (int i = 1; i < p; ++i)
    same = same && (given ? index[i] == index[0] && weight[i] == weight[0]
                          : logits[i] == logits[0]);
  a.tables = same ? 1 : per;
  a.most = most_of(o, same ? per : 1);
  // weights of whole aligned pieces
  auto fast = [&](size_t cols, size_t ld, size_t far, int k0, int k1) {
    uintptr_t bits = cols * c.ew | ld * c.ew | (n > 1 ? far * c.ew : 0);
    for (int k = k0; k < k1; ++k)
      for (int i = 0; i < p; ++i) bits |= (uintptr_t)m[k].at[i];
    return bits % 16 == 0;
  };
  a.fast[0] = fast(o.in, o.ldw, o.xw, 2, 4);
  a.fast[1] = fast(o.hidden, o.ldd, o.xd, 4, 5);
  const size_t chosen = std::min(c.all, o.tokens * top);
  // Tiles of 16 pairs at a time, by an expert's share of them if all have alike;
  // more take another turn over its matrices (2 of 8 experts 4096 x 4096 bf16: up of
  // 128 tokens 193 us with 4, 225 with 2, of 64 tokens 141 with 2, 149 with 4, 177
  // with 1; down of 128 tokens 193 with 2, 222 with 1).  A choice that prefers one
  // expert pays for its turns: 193 us, with one of the two for every token 271.
  const size_t mean = o.tokens * top / c.all;
  a.tiles[0] = mean <= 8 ? 1 : mean <= 24 || !a.fast[0] ? 2 : 4;
  a.tiles[1] = mean <= 8 ? 1 : 2;
  const size_t blocks = o.tokens <= (size_t)moe::kSmall
                            ? (size_t)a.most * a.tables : ~(size_t)0 / kMost;
  // Down by token, a workgroup per CU (8 of 64 experts 2048 x 1024 bf16: one token
  // 27.7 us, by expert and joined 32.2; on 4 and 8 ranks, with as many times the
  // workgroups, 34.9 and 40.8 by token, 31.0 and 30.5 by expert; 8 tokens 103.5 and
  // 103.7, 8-bit weights 78 and 75.5, with a fourth of the pairs 34 and 37.7; 4 tokens
  // through 2 of 8 experts 1024 x 4096, where 16-bit results leave no room for parts
  // of hidden values, below, 44.7 and 44.7, 8-bit 40.9 and 37.2).
  a.small = o.hidden && o.tokens <= (size_t)moe::kSmall &&
            (o.in + 7) / 8 * per <= (size_t)cus * (o.tokens == 1 ? 2 : 1) &&
            (o.tokens == 1 || c.t == Type::F32 ||
             ((o.hidden + 31) / 32 * 32 <= 2 * a.pitch &&
              (!eight || o.tokens * top <= 24)));
  // Each workgroup of up may make the choice for itself: 1 token, 8 of 64 experts
  // 2048 x 1024 bf16 27.7 us, 30.0 with a launch for it; 8 tokens (4096 workgroups)
  // 117 and 103.5.  Where most experts have 3 tokens, each may find those of its own
  // expert: 33 tokens, 3 of 20 experts 1001 x 501 fp16 32.8 us, 37.1 with a launch;
  // 64 tokens, 2 of 8 experts 4096 x 4096 bf16 141 and 181 (which has one tile at a
  // time); 100 tokens of 4 given experts of 64 141 and 144.  (From logits, of which
  // every workgroup reads all, those are 177 and 151.)
  using moe::Mode;
  Mode mode = Mode::TABLE;
  if (o.in && o.hidden && c.all <= 256 &&
      (o.hidden + 15) / 16 * blocks <= (size_t)cus * 4)
    mode = Mode::FUSED;
  else if (o.in && o.hidden && !a.small && c.all <= (size_t)moe::kDirect &&
           o.tokens * top >= 3 * c.all)
    mode = Mode::DIRECT;
  a.mode = (int)mode;
  if (mode == Mode::DIRECT) a.most = (int)n;     // (of one rank's table)
  // (others have at most 8 pairs an expert on the average: of 2048 pairs and
  // more than 256 experts)
  if (mode != Mode::DIRECT) a.tiles[0] = 1;
  const size_t up = 16 * moe::columns_up(c.w, mode == Mode::FUSED, !a.fast[0],
                                         a.tiles[0]);
  a.waves[0] = waves_of((o.hidden + up - 1) / up * chosen, o.in * c.ew / 512,
                        cus);
  // Fewer columns where that fills the card: 33 tokens, 3 of 20 experts 1001 x 501
  // fp16 32.8 us with 32 of them, 33.8 with 64; 3 of 8 experts 4001 x 4001 215 and
  // 207.
  a.sets = (o.in + 63) / 64 * chosen < (size_t)cus * 3 / 2 ? 2 : 4;
  a.waves[1] = waves_of((o.in + 16 * a.sets - 1) / (16 * a.sets) * chosen,
                        o.hidden * c.ew / 512, cus);
  // (rows off 16 bytes, and few columns, have one form each)
  if (!a.fast[0]) a.waves[0] = 4;
  if (!a.fast[1] || a.sets == 2) a.waves[1] = 4;
  // Parts, where there is room for them (by token no pair's result is kept), are
  // half as many bytes again as values, which every workgroup has to split (one token
  // 27.8 and 28.2 us, 8-bit weights 23.5 and 25.0, fp16 29.1 and 30.3).  Two tiles of
  // pairs beside 8-bit weights have registers for values alone (64 tokens, 2 of 8
  // experts 4096 x 8192: 177 us, parts and one tile 208).
  const size_t room = (a.small ? at.bytes : at.parts) - at.hidden;
  a.planes = (int)(c.t == Type::F32 ? moe::Hidden::WHOLE
                   : o.tokens * top * ((o.hidden + 31) / 32) * 192 <= room &&
                           (a.small || !eight || a.tiles[1] == 1)
                       ? moe::Hidden::PARTS
                       : moe::Hidden::VALUES);
  if (logs()) log_layer(c, a, per);
  const size_t groups =
      std::max(std::max((o.hidden + 15) / 16, (o.in + 31) / 32) * n * per,
               (o.in + 7) / 8 * per);
  if (groups > 0xffffffffu / 512)
    return fail(DPAR_ERR_UNSUPPORTED, "%s: %zu workgroups in a launch", call,
                groups);
  for (int r0 = 0; r0 < p; r0 += per) {
    a.ranks = std::min(per, p - r0), a.first = r0;
    if (!same) a.tables = a.ranks;
    if (mode == Mode::DIRECT && same) a.most = (int)n * a.ranks;
    for (int k = 0; k < a.ranks; ++k) {
      const int i = r0 + k;
      a.x[k] = m[0].rank(i);
      a.logits[k] = (const float*)m[1].rank(i);
      for (int j = 0; j < 3; ++j) {
        a.w[j][k] = m[2 + j].rank(i);
        a.s[j][k] = (const float*)m[5 + j].rank(i);
      }
      a.r[k] = m[8].rank(i);
      a.y[k] = (void*)m[9].rank(i);
      a.index[k] = (int*)m[10].rank(i);
      a.weight[k] = (float*)m[11].rank(i);
    }
    if (mode == Mode::TABLE &&
        (rc = launched(call, moe::launch_route(a, stream))))
      return rc;
    if (!o.in) continue;
    const hipError_t e = c.t == Type::BF16  ? moe::launch_bf16(eight, a, stream)
                         : c.t == Type::F16 ? moe::launch_f16(eight, a, stream)
                                            : moe::launch_f32(a, stream);
    if ((rc = launched(call, e))) return rc;
  }
  return DPAR_SUCCESS;
}

}  // namespace

extern "C" {

int dpar_moe(const void* const* x, const void* const* logits,
             const void* const* wg, const void* const* wu,
             const void* const* wd, const void* const* sg,
             const void* const* su, const void* const* sd,
             const void* const* residual, void* const* y, void* const* index,
             void* const* weight, int p, const dpar_moe_t* opt,
             void* workspace, size_t workspace_bytes, hipStream_t stream) {
  return guarded("dpar_moe", [&] {
    return moe_impl(x, logits, wg, wu, wd, sg, su, sd, residual, y, index,
                    weight, p, opt, workspace, workspace_bytes, stream);
  });
}

int dpar_moe_workspace(int p, const dpar_moe_t* opt, size_t* bytes) {
  return guarded("dpar_moe_workspace", [&] {
    const char* call = "dpar_moe_workspace";
    Options c;
    const int rc = check_moe(call, p, opt, &c);
    if (rc) return rc;
    if (!bytes) return fail(DPAR_ERR_INVALID_ARG, "%s: null result", call);
    *bytes = c.o.tokens ? layout_of(c, p).bytes * p : 0;
    return (int)DPAR_SUCCESS;
  });
}

}  // extern "C"
