// C entry points of the 8-bit layer products and of rows' way there.
#include "products_host.hpp"

namespace {

using dpar::products::QuantizeArgs;

// A product of 8-bit operands.
template <typename Fill>
int run_int8(const char* call, int p, const Step& s, Args* a, void* ws,
             size_t bytes, int cus, hipStream_t stream, Fill fill) {
  return run_product(call, Type::I8, p, s, a, ws, bytes, cus, stream,
                     dpar::products::launch_int8,
                     dpar::products::launch_copy_int8, fill);
}

int type_code(dpar_dtype_t t) {
  return (int)(t == DPAR_FLOAT32    ? Type::F32
               : t == DPAR_BFLOAT16 ? Type::BF16
                                    : Type::F16);
}

int linear_impl(const void* const* x, const void* const* sx,
                const void* const* w, const void* const* sw,
                const void* const* bias, const void* const* residual,
                void* const* y, int p, const dpar_product_t* opt, void* ws,
                size_t bytes, hipStream_t stream) {
  const char* call = "dpar_linear_int8";
  dpar_product_t o;
  Type t;
  size_t e, eo;
  int rc = check_options(call, p, opt, &o, &t, &e, &eo, true);
  if (rc) return rc;
  Mat m[] = {
      {"x", x, o.rows, o.in, o.ldx, 1, false, false, true},
      {"sx", sx, 1, o.rows, o.rows, 4, false, false, true},
      {"w", w, o.out, o.in, o.ldw, 1, false, false, true},
      {"sw", sw, 1, o.out, o.out, 4, false, false, true},
      {"bias", bias, 1, o.out, o.out, eo, false, true, bias != nullptr},
      {"residual", residual, o.rows, o.out, o.ldr, eo, false, true,
       residual != nullptr},
      {"y", in_array(y), o.rows, o.out, o.ldy, eo, true, false, true}};
  constexpr int n = 7;
  m[6].twin[0] = residual;
  if ((rc = check_mats(m, n, p, call))) return rc;
  int cus;
  if ((rc = check_workspace(call, DPAR_LINEAR, t, p, o, m, n, ws, bytes,
                            &cus)))
    return rc;
  if (!o.rows || !o.out) return DPAR_SUCCESS;
  Args a = {};
  a.ldo = o.ldy, a.lde = o.ldr;
  a.act = o.act, a.out32 = eo == 4, a.out_type = type_code(o.out_dtype);
  Step s;
  steps_of(DPAR_LINEAR, o, t, false, false, &s);
  s.a.fast = m[0].fast(p), s.b.fast = m[2].fast(p);
  a.wide_out = 1;
  for (int k = 3; k < n; ++k) a.wide_out &= m[k].aligned(p);
  return run_int8(call, p, s, &a, ws, bytes, cus, stream, [&](int k, int i) {
    a.a[0][k] = m[0].rank(i);
    a.a[1][k] = m[1].rank(i);
    a.b[0][k] = m[2].rank(i);
    a.u[0][k] = (void*)m[3].rank(i);
    a.e[0][k] = m[4].rank(i);
    a.e[1][k] = m[5].rank(i);
    a.o[0][k] = (void*)m[6].rank(i);
  });
}

int gated_impl(const void* const* x, const void* const* sx,
               const void* const* wg, const void* const* sg,
               const void* const* wu, const void* const* su,
               const void* const* bg, const void* const* bu, void* const* h,
               int p, const dpar_product_t* opt, void* ws, size_t bytes,
               hipStream_t stream) {
  const char* call = "dpar_gated_int8";
  dpar_product_t o;
  Type t;
  size_t e, eo;
  int rc = check_options(call, p, opt, &o, &t, &e, &eo, true);
  if (rc) return rc;
  const Mat m[] = {
      {"x", x, o.rows, o.in, o.ldx, 1, false, false, true},
      {"sx", sx, 1, o.rows, o.rows, 4, false, false, true},
      {"wg", wg, o.out, o.in, o.ldw, 1, false, false, true},
      {"wu", wu, o.out, o.in, o.ldw, 1, false, false, true},
      {"sg", sg, 1, o.out, o.out, 4, false, false, true},
      {"su", su, 1, o.out, o.out, 4, false, false, true},
      {"bg", bg, 1, o.out, o.out, eo, false, true, bg != nullptr},
      {"bu", bu, 1, o.out, o.out, eo, false, true, bu != nullptr},
      {"h", in_array(h), o.rows, o.out, o.ldy, eo, true, false, true}};
  constexpr int n = 9;
  if ((rc = check_mats(m, n, p, call))) return rc;
  int cus;
  if ((rc = check_workspace(call, DPAR_GATED, t, p, o, m, n, ws, bytes,
                            &cus)))
    return rc;
  if (!o.rows || !o.out) return DPAR_SUCCESS;
  Args a = {};
  a.ldo = o.ldy;
  a.act = o.act, a.out32 = eo == 4, a.out_type = type_code(o.out_dtype);
  Step s;
  steps_of(DPAR_GATED, o, t, false, false, &s);
  s.a.fast = m[0].fast(p), s.b.fast = m[2].fast(p) && m[3].fast(p);
  a.wide_out = 1;
  for (int k = 4; k < n; ++k) a.wide_out &= m[k].aligned(p);
  return run_int8(call, p, s, &a, ws, bytes, cus, stream, [&](int k, int i) {
    a.a[0][k] = m[0].rank(i);
    a.a[1][k] = m[1].rank(i);
    a.b[0][k] = m[2].rank(i);
    a.b[1][k] = m[3].rank(i);
    a.u[0][k] = (void*)m[4].rank(i);
    a.u[1][k] = (void*)m[5].rank(i);
    a.e[0][k] = m[6].rank(i);
    a.e[1][k] = m[7].rank(i);
    a.o[0][k] = (void*)m[8].rank(i);
  });
}

int quantize_impl(const void* const* x, void* const* q, void* const* scale,
                  int p, const dpar_quantize_t* opt, hipStream_t stream) {
  const char* call = "dpar_quantize";
  dpar::set_error(0, "");
  if (p < 1) return fail(DPAR_ERR_INVALID_ARG, "%s: p must be >= 1", call);
  if (!opt) return fail(DPAR_ERR_INVALID_ARG, "%s: null options", call);
  dpar_quantize_t o = *opt;
  if (o.dtype != DPAR_FLOAT32 && o.dtype != DPAR_BFLOAT16 &&
      o.dtype != DPAR_FLOAT16)
    return fail(DPAR_ERR_UNSUPPORTED, "%s: dtype %d", call, (int)o.dtype);
  if (o.rows >= kMost || o.cols >= kMost)
    return fail(DPAR_ERR_UNSUPPORTED, "%s: a size beyond 2^31", call);
  if (!o.ldx || o.rows <= 1) o.ldx = o.cols;
  if (!o.ldq || o.rows <= 1) o.ldq = o.cols;
  if (o.ldx > kMostPitch || o.ldq > kMostPitch)
    return fail(DPAR_ERR_UNSUPPORTED, "%s: a row distance beyond 2^38", call);
  const size_t e = o.dtype == DPAR_FLOAT32 ? 4 : 2;
  const Mat m[] = {
      {"x", x, o.rows, o.cols, o.ldx, e, false, false, true},
      {"q", in_array(q), o.rows, o.cols, o.ldq, 1, true, false, true},
      {"scale", in_array(scale), 1, o.rows, o.rows, 4, true, false, true}};
  const int rc = check_mats(m, 3, p, call);
  if (rc || !o.rows) return rc;
  const int per = ranks_per_launch(p);
  if (logs())
    std::fprintf(stderr, "dpar: quantize %s ranks=%d rows=%zu cols=%zu\n",
                 name_of((Type)type_code(o.dtype)), per, o.rows, o.cols);
  for (int r0 = 0; r0 < p; r0 += per) {
    QuantizeArgs a = {};
    a.rows = o.rows, a.cols = o.cols, a.ldx = o.ldx, a.ldq = o.ldq;
    a.type = type_code(o.dtype);
    a.ranks = std::min(per, p - r0);
    for (int k = 0; k < a.ranks; ++k) {
      a.x[k] = m[0].rank(r0 + k);
      a.q[k] = (signed char*)m[1].rank(r0 + k);
      a.scale[k] = (float*)m[2].rank(r0 + k);
    }
    const int r = launched(call, dpar::products::launch_quantize(a, stream));
    if (r) return r;
  }
  return DPAR_SUCCESS;
}

}  // namespace

extern "C" {

int dpar_quantize(const void* const* x, void* const* q, void* const* scale,
                  int p, const dpar_quantize_t* opt, hipStream_t stream) {
  return guarded("dpar_quantize", [&] {
    return quantize_impl(x, q, scale, p, opt, stream);
  });
}

int dpar_linear_int8(const void* const* x, const void* const* sx,
                     const void* const* w, const void* const* sw,
                     const void* const* bias, const void* const* residual,
                     void* const* y, int p, const dpar_product_t* opt,
                     void* workspace, size_t workspace_bytes,
                     hipStream_t stream) {
  return guarded("dpar_linear_int8", [&] {
    return linear_impl(x, sx, w, sw, bias, residual, y, p, opt, workspace,
                       workspace_bytes, stream);
  });
}

int dpar_gated_int8(const void* const* x, const void* const* sx,
                    const void* const* wg, const void* const* sg,
                    const void* const* wu, const void* const* su,
                    const void* const* bg, const void* const* bu,
                    void* const* h, int p, const dpar_product_t* opt,
                    void* workspace, size_t workspace_bytes,
                    hipStream_t stream) {
  return guarded("dpar_gated_int8", [&] {
    return gated_impl(x, sx, wg, sg, wu, su, bg, bu, h, p, opt, workspace,
                      workspace_bytes, stream);
  });
}

}  // extern "C"
