// Host-callable launchers of the matrix operators (k_linear.hip, k_ortho.hip).  All launches are asynchronous on `st`.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <vector>

#include "kernels.h"
#include "optorch_matrix.h"

namespace oseq {

inline int64_t up8(int64_t n) { return (n + 7) & ~(int64_t)7; }
inline uint64_t up256(uint64_t n) { return (n + 255) & ~(uint64_t)255; }

// Where a matrix lies: rows of `width` bytes, `pitch` bytes apart
struct Place {
  uintptr_t at; int64_t rows, width, pitch;
  uintptr_t end() const { return at + (uintptr_t)((rows - 1) * pitch + width); }
};
inline Place place_in(const void* p, int64_t rows, int64_t cols, int64_t ld, int bytes) {
  return Place{(uintptr_t)p, rows, cols * bytes, ld * bytes};
}
// Whether two matrices share a byte.  Rows that lie between each other's do not.
inline bool overlap(const Place& a, const Place& b) {
  if (a.rows <= 0 || b.rows <= 0 || a.end() <= b.at || b.end() <= a.at) return false;
  if (a.rows < b.rows) return overlap(b, a);
  for (int64_t r = 0; r < b.rows; ++r) {
    // the first of a's rows that ends behind the beginning of this one of b's
    const int64_t s = (int64_t)(b.at + (uintptr_t)(r * b.pitch)) - (int64_t)a.at;
    const int64_t i = s < a.width ? 0 : (s - a.width) / a.pitch + 1;
    if (i < a.rows && i * a.pitch < s + b.width) return true;
  }
  return false;
}
inline bool same_place(const Place& a, const Place& b) {
  return a.at == b.at && (a.pitch == b.pitch || a.rows <= 1) && a.width == b.width;
}

// How a product M x N over K is cut: block tiles of 2 * wave x 2 * wave, the reduction in `parts`
struct ProductShape { int wave, parts; };

// What a linear layer's call does with its workspace: where each piece begins, and how the products run
struct LinearPlan {
  bool straight;                    // forward: both operands straight from memory, no workspace
  bool pack_x, pack_w, make_dz;     // operands that are laid out anew (fp32, or not aligned for 16-byte loads)
  uint64_t off_x, off_w, off_dz, off_sums, off_parts, bytes;
  int64_t dz_second;                // dz in two planes: values from the first to the second, else 0
  int sum_blocks;                   // blocks of rows whose dbias sums are kept apart
  ProductShape y, dx, dw;
};
LinearPlan plan_linear(const optorch_linear_t& a, bool backward);
void launch_linear_forward(const optorch_linear_t& a, const LinearPlan& p);
void launch_linear_backward(const optorch_linear_t& a, const LinearPlan& p);

// ---- orthogonalised updates: what the host plans and the kernels read ----

// One matrix of the list.  X, its iterate, has the shorter side as rows (tall matrices are transposed on the way in and out),
// padded with zeros to multiples of 32, in two fp16 planes (mat_core.h); everything else is m x m, m the shorter side.
struct OrthoMat {
  int64_t offset, ld;      // in the caller's flat vectors
  int32_t rows, cols, m, n;  // m, n: padded shorter and longer side
  int32_t tall, chunk0, chunks, unused;  // rows > cols; its pieces in the passes over all elements
  uint64_t x[2], chain;    // bytes into the workspace: the iterate (two buffers), the m x m buffers
};
enum { OB_A = 0, OB_P, OB_C, OB_Q0, OB_Q1, OB_COUNT };

// A piece of a matrix: 8192 places of X, as 1024 groups of eight (first: of the groups, row by row), or of a tall one 128
// columns from `first` on of 64 rows from `row` on
struct OrthoChunk { int32_t mat, first, row; };
constexpr int ORTHO_GROUPS = 1024;

// one block's tile of a product (mat < 0: nothing); slot >= 0: a part of the sum, kept apart
struct OrthoWork { int32_t mat, tm, tn, k0, k1, slot; };
// a tile whose sum is in `parts` slots from `slot` on
struct OrthoJoin { int32_t mat, tm, tn, slot, parts; };

// dst = alpha * (a b) + beta * extra + diag * identity, all of it in planes (extra < 0: none)
struct OrthoOp { int32_t a, b, dst, extra; float alpha, beta, diag; };

// Lists of small matrices: all steps on A between two iterates in one launch
constexpr int ORTHO_SMALL = 128;                   // padded shorter side at most
constexpr int ORTHO_RESTART = 3;                   // steps between two iterates at most
constexpr int ORTHO_SEGMENT_OPS = 4 * ORTHO_RESTART - 3;
struct OrthoOps { int n; OrthoOp op[ORTHO_SEGMENT_OPS]; };

// the blocks of one kind of product, in launch order, with wavefront tiles of w
struct OrthoList {
  int w = 32, n = 0, joins = 0, slots = 0;
  uint64_t work0 = 0, join0 = 0;
};

enum { OL_GRAM = 0, OL_CHAIN, OL_APPLY };
struct OrthoLaunch {
  int kind, src;       // src: the iterate that is read
  int ops; OrthoOp op[2];
  bool last;           // OL_APPLY: to the caller's output
};

// What the result is stored as says how exact the steps have to be (ortho.cpp): fp32, fp16 or an update of fp32 weights; bf16
enum { OUT_OTHER = 0, OUT_BF16, OUT_COUNT };

struct OrthoTables {   // device pointers and sizes, by value to every kernel
  char* ws;
  const OrthoMat* mats; int nmat;
  const OrthoChunk* chunks; int nchunks;
  double* partial; double* scale; int32_t* bad; int32_t* skip; float* slots;
};

struct OrthoPlanHost {
  std::vector<OrthoMat> mats;
  std::vector<OrthoChunk> chunks;
  std::vector<OrthoWork> works;   // all lists, one behind the other
  std::vector<OrthoJoin> joins;
  OrthoList gram, chain, apply, last[2];  // last: Q X to the caller's vectors; [1]: to weights
  std::vector<OrthoLaunch> launches[OUT_COUNT];
  int most_m = 0;                        // the largest padded shorter side
  float eps = 1e-7f, first_scale = 1.f;  // first_scale: power of two of the first iterate's planes
  int64_t span = 0;
  uint64_t off_mats = 0, off_chunks = 0, off_works = 0, off_joins = 0, off_partial = 0, off_scale = 0, off_bad = 0, off_slots = 0,
           bytes = 0;
};

struct OrthoRun {  // one call
  int g_precision; const void* g;
  int o_precision; void* o;      // orthogonalize
  bool muon;
  optorch_muon_t m;
};
void launch_ortho(hipStream_t st, const OrthoPlanHost& p, char* ws, const OrthoRun& r);

}  // namespace oseq
