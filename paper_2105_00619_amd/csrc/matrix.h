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

// How a product M x N over K is cut: block tiles of 2 * wave x 2 * wave, the reduction in `parts`
struct ProductShape { int wave, parts; };

// What a linear layer's call does with its workspace: where each piece begins, and how the products run
struct LinearPlan {
  bool pack_x, pack_w, pack_dy, make_dz;  // operands that are laid out anew (fp32, or not aligned for 16-byte loads)
  uint64_t off_x, off_w, off_dz, off_sums, off_parts, bytes;
  int sum_blocks;                   // blocks of rows whose dbias sums are kept apart
  ProductShape y, dx, dw;
};
LinearPlan plan_linear(const optorch_linear_t& a, bool backward);
void launch_linear_forward(const optorch_linear_t& a, const LinearPlan& p);
void launch_linear_backward(const optorch_linear_t& a, const LinearPlan& p);

// ---- orthogonalised updates: what the host plans and the kernels read ----

// One matrix of the list.  X, its iterate, is kept as it lies in memory (rows x cols), padded with zeros to multiples of 32,
// in two fp16 planes (mat_core.h); everything else is m x m, m the shorter side.
struct OrthoMat {
  int64_t offset, ld;      // in the caller's flat vectors
  int32_t rows, cols, rp, cp, mp, tall;  // rp, cp, mp: padded rows, columns, shorter side; tall: rows > cols
  uint64_t x[2], chain;    // bytes into the workspace: the iterate (two buffers), the m x m buffers
  int32_t chunk0, chunks;  // its pieces in the passes over all elements
};
enum { OB_A = 0, OB_P, OB_C, OB_Q0, OB_Q1, OB_COUNT };

struct OrthoChunk { int32_t mat, first; };  // 8192 values: groups of eight from `first` on
constexpr int ORTHO_GROUPS = 1024;          // groups of a chunk

// one block's tile of a product
struct OrthoWork { int32_t mat, tm, tn, k0, k1, slot; };  // slot >= 0: a part of the sum, kept apart
// a tile whose sum is in `parts` slots from `slot` on
struct OrthoJoin { int32_t mat, tm, tn, slot, parts; };

// dst = alpha * (a b) + beta * extra + diag * identity, all of it in planes (extra < 0: none)
struct OrthoOp { int32_t a, b, dst, extra; float alpha, beta, diag; };

struct OrthoList { uint64_t off; int32_t n; };  // OrthoWork entries at off in the workspace

enum { OL_GRAM = 0, OL_CHAIN, OL_APPLY };
struct OrthoLaunch {
  int kind, src;       // src: the iterate that is read
  int ops; OrthoOp op[2];
  bool last;           // OL_APPLY: to the caller's output
};

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
  OrthoList gram[2] = {}, chain = {}, apply[2] = {};  // [0] wide, [1] tall; off: index into works
  int w_gram = 32, w_chain = 32, w_apply = 32;        // wavefront tiles
  std::vector<OrthoLaunch> launches;
  float eps = 1e-7f, first_scale = 1.f;  // first_scale: power of two of the first iterate's planes
  int64_t span = 0;
  uint64_t off_mats = 0, off_chunks = 0, off_works = 0, off_joins = 0, off_partial = 0, off_scale = 0, off_bad = 0, off_slots = 0,
           bytes = 0;
  int slots = 0;
};

struct OrthoRun {  // one call
  int g_precision; const void* g;
  int o_precision; void* o;      // orthogonalize
  bool muon;
  optorch_muon_t m;
};
void launch_ortho(hipStream_t st, const OrthoPlanHost& p, char* ws, const OrthoRun& r);

}  // namespace oseq
