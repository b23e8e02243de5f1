// The layer products' entry points (products_api.cpp) with launches that do
// nothing: which kernel each product of a call takes, without a device.
//
// Reads lines "call p rows in out dtype out_dtype act far shift workspace bias"
// (the C values; far: elements between rows, shift: elements before the first,
// workspace: 1 if the call gets the one it asks for, bias: 1 if it has biases
// or is asked for their gradients) and prints for each the
// library's plan lines (DPAR_LOG), a line "launch form type fast waves sets
// tile splits rows sums" per launch, and "rc code".
#include <unistd.h>

#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <string>
#include <vector>

#include "dpar.h"
#include "errors.hpp"
#include "products.hpp"

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
static hipError_t note(Form f, Type t, const Args& a) {
  std::printf("launch %d %d %d %d %d %d %d %zu %d\n", (int)f, (int)t, a.fast,
              a.waves, a.sets, a.tile, a.splits, a.ni, a.sums);
  return hipSuccess;
}
hipError_t launch_copy(const CopyArgs&, hipStream_t) { return hipSuccess; }
hipError_t launch_bf16(Form f, const Args& a, hipStream_t) {
  return note(f, Type::BF16, a);
}
hipError_t launch_f16(Form f, const Args& a, hipStream_t) {
  return note(f, Type::F16, a);
}
hipError_t launch_f32(Form f, const Args& a, hipStream_t) {
  return note(f, Type::F32, a);
}
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
}  // namespace dpar

namespace {

// Addresses of p matrices of rows x cols, each call's k-th array in 2^40 bytes
// of its own.
std::vector<void*> at(int k, int p, size_t rows, size_t ld, size_t shift,
                      size_t e) {
  std::vector<void*> v;
  for (int i = 0; i < p; ++i)
    v.push_back((void*)(((uintptr_t)(k + 1) << 40) +
                        ((size_t)i * rows * ld + shift) * e));
  return v;
}

const void* const* in(const std::vector<void*>& v) {
  return (const void* const*)v.data();
}

}  // namespace

int main() {
  setvbuf(stdout, nullptr, _IONBF, 0);
  dup2(1, 2);
  setenv("DPAR_LOG", "1", 1);
  int call, p, dtype, out, act, ws, bias;
  size_t rows, n_in, n_out, far, shift;
  while (std::scanf("%d %d %zu %zu %zu %d %d %d %zu %zu %d %d",
                    &call, &p, &rows, &n_in, &n_out, &dtype, &out, &act, &far,
                    &shift, &ws, &bias) == 12) {
    const size_t e = dtype == DPAR_FLOAT32 ? 4 : 2,
                 eo = out == DPAR_FLOAT32 ? 4 : 2;
    dpar_product_t o = {rows, n_in, n_out, (dpar_dtype_t)dtype,
                        (dpar_dtype_t)out, (dpar_act_t)act, n_in + far,
                        n_in + far, n_out + far, n_out + far, n_out + far,
                        n_in + far, n_in + far};
    auto x = [&](int k, size_t es) {
      return at(k, p, rows, n_in + far, shift, es);
    };
    auto w = [&](int k, size_t es) {
      return at(k, p, n_out, n_in + far, shift, es);
    };
    auto y = [&](int k, size_t es) {
      return at(k, p, rows, n_out + far, shift, es);
    };
    std::vector<void*> biases[2];
    auto b = [&](int k, size_t es) -> void* const* {
      if (!bias) return nullptr;
      biases[k % 2] = at(k, p, 1, n_out, shift, es);
      return biases[k % 2].data();
    };
    size_t n = 0;
    int rc = ws ? dpar_product_workspace((dpar_product_call_t)call, p, &o, &n)
                : 0;
    void* work = n ? (void*)((uintptr_t)60 << 40) : nullptr;
    switch (rc ? -1 : call) {
      case DPAR_LINEAR:
        rc = dpar_linear(in(x(0, e)), in(w(1, e)), b(2, e), nullptr,
                         y(3, eo).data(), y(4, e).data(), p, &o, work, n,
                         nullptr);
        break;
      case DPAR_LINEAR_BACKWARD:
        rc = dpar_linear_backward(
            in(y(0, e)), in(x(1, e)), in(w(2, e)), in(y(3, e)),
            x(4, eo).data(), w(5, eo).data(), b(6, eo), y(7, e).data(),
            p, &o, work, n, nullptr);
        break;
      case DPAR_GATED:
        rc = dpar_gated(in(x(0, e)), in(w(1, e)), in(w(2, e)), b(3, e),
                        b(4, e), y(5, eo).data(), y(6, e).data(),
                        y(7, e).data(), p, &o, work, n, nullptr);
        break;
      case DPAR_GATED_BACKWARD:
        rc = dpar_gated_backward(
            in(y(0, e)), in(x(1, e)), in(w(2, e)), in(w(3, e)), in(y(4, e)),
            in(y(5, e)), x(6, eo).data(), w(7, eo).data(), w(8, eo).data(),
            b(9, eo), b(10, eo), y(11, e).data(),
            y(12, e).data(), p, &o, work, n, nullptr);
    }
    std::printf("rc %d %s\n", rc, rc ? dpar::g_text.c_str() : "");
  }
  return 0;
}
