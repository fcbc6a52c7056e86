// C ABI of the matrix operators (optorch_matrix.h): argument checks, then the kernels of k_linear.hip and k_ortho.hip on the
// caller's stream.  Nothing here allocates on the device; only optorch_ortho_bind synchronises.
#include <hip/hip_runtime.h>

#include <string>

#include "matrix.h"

using namespace oseq;

static thread_local std::string g_mat_error;

int oseq_mat_err(int code, const std::string& m);
int oseq_mat_err(int code, const std::string& m) {
  try { g_mat_error = m; } catch (...) {}
  return code;
}

// every entry runs inside this: no C++ exception (host memory running out) leaves the library
template <class F> static auto guarded(F&& f) -> decltype(f()) {
  try { return f(); } catch (...) { return oseq_mat_err(OPTORCH_E_INVALID, "out of host memory"); }
}

static int mat_launched(const char* what) {
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return oseq_mat_err(OPTORCH_E_HIP, std::string(what) + ": " + hipGetErrorString(e));
  return OPTORCH_OK;
}

extern "C" const char* optorch_matrix_last_error(void) { return g_mat_error.c_str(); }

static bool precision_ok(int32_t p) { return p == OPTORCH_FP32 || p == OPTORCH_BF16 || p == OPTORCH_FP16; }
static int bytes_of(int32_t p) { return p == OPTORCH_FP32 ? 4 : 2; }

// ---- linear layers -----------------------------------------------------------------------------------------------------

// Offsets inside a tile are 32-bit: 256 rows take less than 2^31 bytes.  A row of fp32 values laid out as planes takes 8
// bytes a value.
static constexpr int64_t kMaxFeatures = (1 << 22) - 8, kMaxFeatures32 = (1 << 20) - 16;

static int linear_check(const optorch_linear_t* a, bool backward) {
  if (!a) return oseq_mat_err(OPTORCH_E_INVALID, "null arguments");
  if (!precision_ok(a->precision)) return oseq_mat_err(OPTORCH_E_INVALID, "unknown precision");
  if (a->activation < OPTORCH_ACT_NONE || a->activation > OPTORCH_ACT_SILU) return oseq_mat_err(OPTORCH_E_INVALID, "unknown activation");
  if (a->rows < 0 || a->rows > 0x7fffff00) return oseq_mat_err(OPTORCH_E_INVALID, "rows must be 0 .. 2^31 - 256");
  if (a->in_features < 1 || a->out_features < 1 || a->in_features > kMaxFeatures || a->out_features > kMaxFeatures)
    return oseq_mat_err(OPTORCH_E_INVALID, "in_features and out_features must be 1 .. 2^22 - 8");
  if (a->precision == OPTORCH_FP32 && (a->in_features > kMaxFeatures32 || a->out_features > kMaxFeatures32))
    return oseq_mat_err(OPTORCH_E_INVALID, "in fp32 in_features and out_features must be 1 .. 2^20 - 16");
  const int esize = bytes_of(a->precision);
  // a matrix that is used: present, its rows apart, its elements aligned
  auto matrix = [&](const void* p, int64_t ld, int32_t cols, const char* name) {
    if (!p) return oseq_mat_err(OPTORCH_E_INVALID, std::string("null ") + name);
    if (ld < cols || ld > kMaxFeatures) return oseq_mat_err(OPTORCH_E_INVALID, std::string("leading dimension of ") + name + " must be its columns .. 2^22 - 8");
    if ((uintptr_t)p % esize) return oseq_mat_err(OPTORCH_E_INVALID, std::string(name) + " is not aligned to its elements");
    return (int)OPTORCH_OK;
  };
  auto vector = [&](const float* p, const char* name) {
    return (uintptr_t)p % 4 ? oseq_mat_err(OPTORCH_E_INVALID, std::string(name) + " is not aligned to its elements") : (int)OPTORCH_OK;
  };
  int rc = OPTORCH_OK;
  const int32_t in = a->in_features, out = a->out_features;
  const bool some = a->rows > 0;  // (an empty batch has no matrices of its own)
  if (!backward) {
    if (some && rc == OPTORCH_OK) rc = matrix(a->x, a->ldx, in, "x");
    if (rc == OPTORCH_OK) rc = matrix(a->w, a->ldw, in, "w");
    if (some && rc == OPTORCH_OK) rc = matrix(a->y, a->ldy, out, "y");
    if (some && rc == OPTORCH_OK && a->residual) rc = matrix(a->residual, a->ldr, out, "residual");
    if (some && rc == OPTORCH_OK && a->z) rc = matrix(a->z, a->ldz, out, "z");
    if (rc == OPTORCH_OK) rc = vector(a->bias, "bias");
    return rc;
  }
  if (!a->dx && !a->dw && !a->dbias) return oseq_mat_err(OPTORCH_E_INVALID, "no gradient asked for");
  if (some && rc == OPTORCH_OK) rc = matrix(a->dy, a->lddy, out, "dy");
  if (some && rc == OPTORCH_OK && a->activation != OPTORCH_ACT_NONE) rc = matrix(a->z, a->ldz, out, "z");
  if (some && rc == OPTORCH_OK && a->dw) rc = matrix(a->x, a->ldx, in, "x");
  if (rc == OPTORCH_OK && a->dw) rc = matrix(a->dw, a->lddw, in, "dw");
  if (some && rc == OPTORCH_OK && a->dx) rc = matrix(a->w, a->ldw, in, "w");
  if (some && rc == OPTORCH_OK && a->dx) rc = matrix(a->dx, a->lddx, in, "dx");
  if (rc == OPTORCH_OK) rc = vector(a->dbias, "dbias");
  return rc;
}

// What the call writes against everything that it reads or writes besides
static int linear_overlaps(const optorch_linear_t* a, bool backward, uint64_t workspace_bytes) {
  struct Named { const char* name; Place p; bool written; } list[10];
  int n = 0;
  const int e = bytes_of(a->precision);
  auto add = [&](const char* name, const void* p, int64_t rows, int64_t cols, int64_t ld, int bytes, bool written) {
    if (p && rows > 0 && cols > 0) list[n++] = Named{name, place_in(p, rows, cols, ld, bytes), written};
  };
  const int64_t rows = a->rows, in = a->in_features, out = a->out_features;
  const bool slope = a->activation != OPTORCH_ACT_NONE;
  if (!backward || a->dw) add("x", a->x, rows, in, a->ldx, e, false);
  if (!backward || a->dx) add("w", a->w, out, in, a->ldw, e, false);
  if (!backward || slope) add("z", a->z, rows, out, a->ldz, e, !backward);
  if (!backward) {
    add("bias", a->bias, 1, out, out, 4, false);
    add("residual", a->residual, rows, out, a->ldr, e, false);
    add("y", a->y, rows, out, a->ldy, e, true);
  } else {
    add("dy", a->dy, rows, out, a->lddy, e, false);
    add("dx", a->dx, rows, in, a->lddx, e, true);
    add("dw", a->dw, out, in, a->lddw, e, true);
    add("dbias", a->dbias, 1, out, out, 4, true);
  }
  add("workspace", workspace_bytes ? a->workspace : nullptr, 1, (int64_t)workspace_bytes, (int64_t)workspace_bytes, 1, true);
  for (int i = 0; i < n; ++i)
    for (int j = i + 1; j < n; ++j) {
      const Named &p = list[i], &q = list[j];
      if (!(p.written || q.written) || !overlap(p.p, q.p)) continue;
      if (!backward && p.p.at == (uintptr_t)a->residual && q.p.at == (uintptr_t)a->y && same_place(p.p, q.p)) continue;
      return oseq_mat_err(OPTORCH_E_INVALID, std::string(p.name) + " and " + q.name + " overlap");
    }
  return OPTORCH_OK;
}

extern "C" int64_t optorch_linear_workspace(const optorch_linear_t* a, int32_t backward) {
  return guarded([&]() -> int64_t {
    const int rc = linear_check(a, backward != 0);
    if (rc != OPTORCH_OK) return rc;
    return a->rows ? (int64_t)plan_linear(*a, backward != 0).bytes : 0;
  });
}

// How a product of the call is cut, for the tests that name a kernel by its tile (not part of the API): 1000 * values of a
// tile's edge + parts; product 0: y, 1: dx, 2: dw.  0: straight from memory.
namespace oseq {
int linear_shape(const optorch_linear_t* a, bool backward, int product);
int linear_shape(const optorch_linear_t* a, bool backward, int product) {
  const LinearPlan p = plan_linear(*a, backward);
  const ProductShape s = product == 0 ? p.y : product == 1 ? p.dx : p.dw;
  return p.straight ? 0 : 2000 * s.wave + s.parts;
}
}  // namespace oseq

static int linear_run(const optorch_linear_t* a, bool backward) {
  const int rc = linear_check(a, backward);
  if (rc != OPTORCH_OK) return rc;
  LinearPlan p = {};
  if (a->rows) {
    p = plan_linear(*a, backward);
    if (p.bytes && !a->workspace) return oseq_mat_err(OPTORCH_E_INVALID, "null workspace");
    if (p.bytes > a->workspace_bytes) return oseq_mat_err(OPTORCH_E_BUDGET, "workspace too small: " + std::to_string(p.bytes) + " bytes are needed");
    if (p.bytes && (uintptr_t)a->workspace % 256) return oseq_mat_err(OPTORCH_E_INVALID, "workspace must be 256-byte aligned");
  }
  const int apart = linear_overlaps(a, backward, p.bytes);
  if (apart != OPTORCH_OK) return apart;
  if (!backward && a->rows) launch_linear_forward(*a, p);
  if (backward) launch_linear_backward(*a, p);
  return mat_launched(backward ? "linear_backward" : "linear_forward");
}

extern "C" int optorch_linear_forward(const optorch_linear_t* a) { return guarded([&] { return linear_run(a, false); }); }
extern "C" int optorch_linear_backward(const optorch_linear_t* a) { return guarded([&] { return linear_run(a, true); }); }
