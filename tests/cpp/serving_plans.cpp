// The entry points of the 8-bit products and of the mixture-of-experts layer
// (int8_api.cpp, moe_api.cpp) with launches that do nothing: which kernels each
// call takes, without a device.
//
// Reads lines "int8 gated p rows in out out_dtype far shift workspace" and "moe p
// tokens in hidden experts top dtype weight_dtype out_dtype far apart" (the C
// values; far: elements between rows; apart: every rank has logits of its own)
// and prints a line "int8 form fast waves sets tile splits rows" or "moe type
// eight mode fast0 tiles0 waves0 small fast1 tiles1 waves1 sets planes" per
// launch, "route" for one of its own, and "rc code".
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <string>
#include <vector>

#include "dpar.h"
#include "errors.hpp"
#include "moe.hpp"

extern "C" {
hipError_t hipGetDevice(int* d) {
  *d = 0;
  return hipSuccess;
}
hipError_t hipDeviceGetAttribute(int* v, hipDeviceAttribute_t, int) {
  *v = 256;
  return hipSuccess;
}
hipError_t hipGetLastError() { return hipSuccess; }
const char* hipGetErrorString(hipError_t) { return ""; }
}

namespace dpar {
static std::string g_text;
int set_error(int code, const char* text) {
  g_text = text;
  return code;
}
namespace products {
hipError_t launch_int8(Form f, const Args& a, hipStream_t) {
  std::printf("int8 %d %d %d %d %d %d %zu\n", (int)f, a.fast, a.waves, a.sets,
              a.tile, a.splits, a.ni);
  return hipSuccess;
}
hipError_t launch_copy_int8(const CopyArgs&, hipStream_t) {
  return hipSuccess;
}
hipError_t launch_quantize(const QuantizeArgs&, hipStream_t) {
  return hipSuccess;
}
// (products_api.cpp, for the workspace query)
hipError_t launch_copy(const CopyArgs&, hipStream_t) { return hipSuccess; }
hipError_t launch_bf16(Form, const Args&, hipStream_t) { return hipSuccess; }
hipError_t launch_f16(Form, const Args&, hipStream_t) { return hipSuccess; }
hipError_t launch_f32(Form, const Args&, hipStream_t) { return hipSuccess; }
hipError_t launch_slope_bf16(const SlopeArgs&, hipStream_t) {
  return hipSuccess;
}
hipError_t launch_slope_f16(const SlopeArgs&, hipStream_t) {
  return hipSuccess;
}
hipError_t launch_slope_f32(const SlopeArgs&, hipStream_t) {
  return hipSuccess;
}
hipError_t launch_sums_bf16(const SumArgs&, hipStream_t) { return hipSuccess; }
hipError_t launch_sums_f16(const SumArgs&, hipStream_t) { return hipSuccess; }
}  // namespace products
namespace moe {
static hipError_t note(int type, bool eight, const Args& a) {
  std::printf("moe %d %d %d %d %d %d %d %d %d %d %d %d\n", type, (int)eight,
              a.mode, a.fast[0], a.tiles[0], a.waves[0], a.small, a.fast[1],
              a.tiles[1], a.waves[1], a.sets, a.planes);
  return hipSuccess;
}
hipError_t launch_route(const Args&, hipStream_t) {
  std::printf("route\n");
  return hipSuccess;
}
hipError_t launch_bf16(bool eight, const Args& a, hipStream_t) {
  return note(3, eight, a);
}
hipError_t launch_f16(bool eight, const Args& a, hipStream_t) {
  return note(4, eight, a);
}
hipError_t launch_f32(const Args& a, hipStream_t) { return note(1, false, a); }
}  // namespace moe
}  // namespace dpar

namespace {

// Addresses of p pieces of `bytes` each, a call's k-th array in 2^41 bytes of
// its own.
std::vector<void*> at(int k, int p, size_t bytes, size_t shift) {
  std::vector<void*> v;
  for (int i = 0; i < p; ++i)
    v.push_back((void*)(((uintptr_t)(k + 1) << 41) + i * bytes + shift));
  return v;
}
const void* const* in(const std::vector<void*>& v) {
  return (const void* const*)v.data();
}

int run_int8() {
  int gated, p, out, ws;
  size_t rows, n_in, n_out, far, shift;
  if (std::scanf("%d %d %zu %zu %zu %d %zu %zu %d", &gated, &p, &rows, &n_in,
                 &n_out, &out, &far, &shift, &ws) != 9)
    return 1;
  const size_t eo = out == DPAR_FLOAT32 ? 4 : 2;
  const dpar_product_t o = {rows, n_in, n_out, DPAR_INT8, (dpar_dtype_t)out,
                            DPAR_ACT_NONE, n_in + far, n_in + far,
                            n_out + far, n_out + far, 0, 0, 0};
  size_t n = 0;
  int rc = ws ? dpar_product_workspace(gated ? DPAR_GATED : DPAR_LINEAR, p, &o,
                                       &n)
              : 0;
  void* work = n ? (void*)((uintptr_t)60 << 41) : nullptr;
  const auto x = at(0, p, rows * (n_in + far), shift),
             w = at(1, p, n_out * (n_in + far), shift),
             u = at(2, p, n_out * (n_in + far), shift),
             sx = at(3, p, rows * 4, 0), sw = at(4, p, n_out * 4, 0),
             su = at(5, p, n_out * 4, 0);
  auto y = at(6, p, rows * (n_out + far) * eo, 0);
  if (!rc)
    rc = gated ? dpar_gated_int8(in(x), in(sx), in(w), in(sw), in(u), in(su),
                                 nullptr, nullptr, y.data(), p, &o, work, n,
                                 nullptr)
               : dpar_linear_int8(in(x), in(sx), in(w), in(sw), nullptr,
                                  nullptr, y.data(), p, &o, work, n, nullptr);
  return rc;
}

int run_moe() {
  int p, top, dtype, wtype, out, apart;
  size_t tokens, n_in, hidden, experts, far;
  if (std::scanf("%d %zu %zu %zu %zu %d %d %d %d %zu %d", &p, &tokens, &n_in,
                 &hidden, &experts, &top, &dtype, &wtype, &out, &far,
                 &apart) != 11)
    return 1;
  const size_t e = dtype == DPAR_FLOAT32 ? 4 : 2,
               ew = wtype == DPAR_INT8 ? 1 : e,
               eo = out == DPAR_FLOAT32 ? 4 : 2;
  dpar_moe_t o = {};
  o.tokens = tokens, o.in = n_in, o.hidden = hidden, o.experts = experts;
  o.top = top, o.dtype = (dpar_dtype_t)dtype;
  o.weight_dtype = (dpar_dtype_t)wtype, o.out_dtype = (dpar_dtype_t)out;
  o.act = DPAR_ACT_SILU, o.normalize = 1, o.weight_scale = 1.f;
  o.ldw = n_in + far, o.ldd = hidden + far;
  size_t n = 0;
  int rc = dpar_moe_workspace(p, &o, &n);
  if (rc) return rc;
  const auto w = [&](int k, size_t r, size_t c) {
    return at(k, p, experts * r * (c + far) * ew, 0);
  };
  const bool eight = wtype == DPAR_INT8;
  const auto x = at(0, 1, 1, 0), logits = at(1, p, 1 << 20, 0),
             wg = w(2, hidden, n_in), wu = w(3, hidden, n_in),
             wd = w(4, n_in, hidden), sg = at(5, p, experts * hidden * 4, 0),
             su = at(6, p, experts * hidden * 4, 0),
             sd = at(7, p, experts * n_in * 4, 0);
  auto y = at(8, p, tokens * n_in * eo, 0);
  std::vector<const void*> xs(p, x[0]), ls(p, logits[0]);
  return dpar_moe(xs.data(), apart ? in(logits) : ls.data(), in(wg), in(wu),
                  in(wd), eight ? in(sg) : nullptr, eight ? in(su) : nullptr,
                  eight ? in(sd) : nullptr, nullptr, y.data(), nullptr,
                  nullptr, p, &o, (void*)((uintptr_t)60 << 41), n, nullptr);
}

}  // namespace

int main() {
  char what[8];
  while (std::scanf("%7s", what) == 1) {
    const int rc = std::strcmp(what, "moe") ? run_int8() : run_moe();
    std::printf("rc %d %s\n", rc, rc ? dpar::g_text.c_str() : "");
  }
  return 0;
}
