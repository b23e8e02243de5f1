// C entry points of the layer products in 16 and 32 bits.
#include "products_host.hpp"

namespace {

// A product in 16 or 32 bits.
template <typename Fill>
int run_float(const char* call, Type t, int p, const Step& s, Args* a,
              void* ws, size_t bytes, int cus, hipStream_t stream, Fill fill) {
  using namespace dpar::products;
  return run_product(call, t, p, s, a, ws, bytes, cus, stream,
                     t == Type::BF16  ? launch_bf16
                     : t == Type::F16 ? launch_f16
                                      : launch_f32,
                     launch_copy, fill);
}

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
  return run_float(call, t, p, s, &a, ws, bytes, cus, stream,
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
  return run_float(call, t, p, s, &a, ws, bytes, cus, stream,
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
    rc = run_float(call, t, p, s, &a, ws, bytes, cus, stream,
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
    rc = run_float(call, t, p, s, &a, ws, bytes, cus, stream,
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
    const bool int8 = opt && opt->dtype == DPAR_INT8;
    const int rc = check_options(name, p, opt, &o, &t, &e, &eo, int8);
    if (rc) return rc;
    if ((int)call < DPAR_LINEAR || (int)call > DPAR_GATED_BACKWARD)
      return fail(DPAR_ERR_INVALID_ARG, "%s: unknown call %d", name,
                  (int)call);
    if (int8 && call != DPAR_LINEAR && call != DPAR_GATED)
      return fail(DPAR_ERR_UNSUPPORTED, "%s: call %d of 8-bit operands", name,
                  (int)call);
    if (!bytes) return fail(DPAR_ERR_INVALID_ARG, "%s: null result", name);
    *bytes = workspace_of(call, t, p, o, cu_count());
    return (int)DPAR_SUCCESS;
  });
}

}  // extern "C"
