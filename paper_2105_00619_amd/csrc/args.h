// Checks of arguments that the C entries of the matrix operators share.  Every failure leaves its message for
// optorch_matrix_last_error and returns its code.
#pragma once
#include <hip/hip_runtime.h>
#include <math.h>
#include <string.h>

#include <string>

#include "matrix.h"

int oseq_mat_err(int code, const std::string& m);  // matrix.cpp

namespace oseq {

// every entry runs inside this: no C++ exception (host memory running out) leaves the library
template <class F> inline auto guarded(F&& f) -> decltype(f()) {
  try { return f(); } catch (...) { return oseq_mat_err(OPTORCH_E_INVALID, "out of host memory"); }
}

inline int mat_launched(const char* what) {
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return oseq_mat_err(OPTORCH_E_HIP, std::string(what) + ": " + hipGetErrorString(e));
  return OPTORCH_OK;
}

inline bool precision_ok(int32_t p) { return p == OPTORCH_FP32 || p == OPTORCH_BF16 || p == OPTORCH_FP16; }
inline int bytes_of(int32_t p) { return p == OPTORCH_FP32 ? 4 : 2; }

// Offsets inside a tile are 32-bit: 256 rows take less than 2^31 bytes.  A row of fp32 values laid out as planes takes 8
// bytes a value.
constexpr int64_t kMaxFeatures = (1 << 22) - 8, kMaxFeatures32 = (1 << 20) - 16;

// a matrix that is used: present, its rows apart, its elements aligned
inline int check_matrix(const void* p, int64_t ld, int64_t cols, int esize, const char* name) {
  if (!p) return oseq_mat_err(OPTORCH_E_INVALID, std::string("null ") + name);
  if (ld < cols || ld > kMaxFeatures) return oseq_mat_err(OPTORCH_E_INVALID, std::string("leading dimension of ") + name + " must be its columns .. 2^22 - 8");
  if ((uintptr_t)p % esize) return oseq_mat_err(OPTORCH_E_INVALID, std::string(name) + " is not aligned to its elements");
  return OPTORCH_OK;
}
inline int check_vector(const void* p, const char* name) {
  return (uintptr_t)p % 4 ? oseq_mat_err(OPTORCH_E_INVALID, std::string(name) + " is not aligned to its elements") : (int)OPTORCH_OK;
}
inline int check_workspace(const void* p, uint64_t given, uint64_t bytes) {
  if (bytes && !p) return oseq_mat_err(OPTORCH_E_INVALID, "null workspace");
  if (bytes > given) return oseq_mat_err(OPTORCH_E_BUDGET, "workspace too small: " + std::to_string(bytes) + " bytes are needed");
  if (bytes && (uintptr_t)p % 256) return oseq_mat_err(OPTORCH_E_INVALID, "workspace must be 256-byte aligned");
  return OPTORCH_OK;
}

// What a call writes against everything that it reads or writes besides
struct Operands {
  static constexpr int MOST = 16;
  struct Named {
    const char* name; Place p; bool written;
    bool is(const char* n) const { return strcmp(name, n) == 0; }
  } list[MOST];
  int n = 0;
  void add(const char* name, const void* p, int64_t rows, int64_t cols, int64_t ld, int bytes, bool written) {
    if (p && rows > 0 && cols > 0) list[n++] = Named{name, place_in(p, rows, cols, ld, bytes), written};
  }
  void vector(const char* name, const void* p, int64_t n, int bytes, bool written) { add(name, p, 1, n, n, bytes, written); }
  // allowed(p, q): a pair that may lie in the same place
  template <class F> int apart(F&& allowed) const {
    for (int i = 0; i < n; ++i)
      for (int j = i + 1; j < n; ++j) {
        const Named &p = list[i], &q = list[j];
        if (!(p.written || q.written) || !overlap(p.p, q.p) || allowed(p, q)) continue;
        return oseq_mat_err(OPTORCH_E_INVALID, std::string(p.name) + " and " + q.name + " overlap");
      }
    return OPTORCH_OK;
  }
};

}  // namespace oseq
