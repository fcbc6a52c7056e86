// Orthogonalised updates: the kernels of the plan made in ortho.cpp.  Every launch does its part for all matrices of the list; a
// block finds its matrix and tile in a table.
//   norms    sum of squares of each piece of a matrix, in 64 bits
//   scales   1 / max(norm, eps) per matrix, and whether all its elements are finite
//   planes   the first iterate: elements times the scale as two fp16 planes, padded with zeros; momentum is updated on the way
//   products X X^T, then m x m products (half of the tiles: they are symmetric), then Q X (ortho.cpp)
#include <math.h>

#include "mat_core.h"
#include "matrix.h"

namespace oseq {

namespace {

using namespace mat;

// a value in two fp16 planes
__device__ __forceinline__ void split8(const float (&v)[8], Vec<f16_t, 8>& hi, Vec<f16_t, 8>& lo) {
  hi = round_vec<f16_t, 8>(v);
  float l[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) l[e] = v[e] - (float)hi.v[e];
  lo = round_vec<f16_t, 8>(l);
}
// eight neighbouring columns from c on of a row in two planes (mat_core.h)
__device__ __forceinline__ void store_planes(f16_t* row, int c, const float (&v)[8]) {
  Vec<f16_t, 8> hi, lo;
  split8(v, hi, lo);
  f16_t* p = row + place_of<2>(c);
  *reinterpret_cast<Vec<f16_t, 8>*>(p) = hi;
  *reinterpret_cast<Vec<f16_t, 8>*>(p + 32) = lo;
}
__device__ __forceinline__ void load_planes(const f16_t* row, int c, float (&v)[8]) {
  const f16_t* p = row + place_of<2>(c);
  float l[8];
  load_f32<f16_t, 8>(p, v);
  load_f32<f16_t, 8>(p + 32, l);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] += l[e];
}

// eight neighbouring values, n of them inside, at any address
template <class T> struct Loose8 { T v[8]; } __attribute__((packed, aligned(alignof(T))));
template <class T> __device__ __forceinline__ void get8(const T* p, int n, float (&v)[8]) {
  if (n == 8) {
    const Loose8<T> t = *reinterpret_cast<const Loose8<T>*>(p);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = to_f32(t.v[e]);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < n ? to_f32(p[e]) : 0.f;
  }
}
template <class T> __device__ __forceinline__ void put8(T* p, int n, const float (&v)[8]) {
  if (n == 8) {
    *reinterpret_cast<Loose8<T>*>(p) = __builtin_bit_cast(Loose8<T>, round_vec<T, 8>(v));
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) p[e] = from_f32<T>(v[e]);
  }
}

// what the first iterate is made of
struct Source {
  const void* g; float* v;
  float grad_scale, momentum; int nesterov;
};
// u of eight neighbouring elements; vn: the new momentum
template <class G, bool MUON>
__device__ __forceinline__ void source8(const Source& s, int64_t at, int n, float (&u)[8], float (&vn)[8]) {
  get8((const G*)s.g + at, n, u);
  if (MUON) {
    get8((const float*)s.v + at, n, vn);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float g = u[e] * s.grad_scale;
      vn[e] = __fmaf_rn(s.momentum, vn[e], g);
      u[e] = s.nesterov ? __fmaf_rn(s.momentum, vn[e], g) : vn[e];
    }
  }
}

// f(place in the flat vectors, n, row of X, column) for groups of eight neighbouring columns of a piece, n of them inside (0: none);
// a tall matrix' groups run along its own columns: row and column of the transposed group's first value
template <class F> __device__ __forceinline__ void groups_of(const OrthoChunk& c, const OrthoMat& m, F&& f) {
  if (m.tall) {
    const int col = c.first + (threadIdx.x & 15) * 8;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int r = c.row + k * 16 + (threadIdx.x >> 4);
      f(m.offset + r * m.ld + col, r < m.rows ? min(8, m.cols - col) : 0, col, r);
    }
  } else {
    const int c8 = m.n / 8, last = min(c.first + ORTHO_GROUPS, m.m * c8);
    for (int g = c.first + threadIdx.x; g < last; g += 256) {
      const int r = g / c8, col = (g - r * c8) * 8;
      f(m.offset + r * m.ld + col, r < m.rows ? min(8, m.cols - col) : 0, r, col);
    }
  }
}

template <class G, bool MUON>
__global__ void __launch_bounds__(256) norms_kernel(OrthoTables t, Source s) {
  __shared__ double part[4];
  const OrthoChunk c = t.chunks[blockIdx.x];
  double sum = 0.;
  groups_of(c, t.mats[c.mat], [&](int64_t at, int n, int, int) {
    if (n <= 0) return;
    float u[8], vn[8];
    source8<G, MUON>(s, at, n, u, vn);
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) sum = fma((double)u[e], (double)u[e], sum);
  });
#pragma unroll
  for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x == 0) t.partial[blockIdx.x] = (part[0] + part[1]) + (part[2] + part[3]);
}

__global__ void __launch_bounds__(256) scales_kernel(OrthoTables t, float eps, double times) {
  __shared__ double part[4];
  const OrthoMat& m = t.mats[blockIdx.x];
  double sum = 0.;
  for (int i = threadIdx.x; i < m.chunks; i += 256) sum += t.partial[m.chunk0 + i];
#pragma unroll
  for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    sum = (part[0] + part[1]) + (part[2] + part[3]);
    const double norm = sqrt(sum);
    t.scale[blockIdx.x] = times / (norm < (double)eps ? (double)eps : norm);  // (NaN stays NaN)
    t.bad[blockIdx.x] = sum <= 1.7976931348623157e308 ? 0 : 1;
  }
}

template <class G, bool MUON>
__global__ void __launch_bounds__(256) planes_kernel(OrthoTables t, Source s, int32_t* skipped) {
  __shared__ float turn[128][65];  // a tall matrix' piece on its way to its transposed place
  const OrthoChunk c = t.chunks[blockIdx.x];
  const OrthoMat& m = t.mats[c.mat];
  bool skip = false;
  if (MUON) {
    bool any = false;
    for (int i = threadIdx.x; i < t.nmat; i += 256) any |= t.bad[i] != 0;
    skip = __syncthreads_or(any);
    if (blockIdx.x == 0 && threadIdx.x == 0) {
      t.skip[0] = skip;
      if (skipped) *skipped = skip;
    }
  }
  const double scale = t.scale[c.mat];
  f16_t* x = (f16_t*)(t.ws + m.x[0]);
  groups_of(c, m, [&](int64_t at, int n, int r, int col) {
    float u[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, vn[8];
    if (n > 0) {
      source8<G, MUON>(s, at, n, u, vn);
      if (MUON && !skip) put8(s.v + at, n, vn);
#pragma unroll
      for (int e = 0; e < 8; ++e) u[e] = e < n ? (float)((double)u[e] * scale) : 0.f;
    }
    if (m.tall) {
#pragma unroll
      for (int e = 0; e < 8; ++e) turn[r - c.first + e][col - c.row] = u[e];
    } else {
      store_planes(x + (int64_t)r * 2 * m.n, col, u);
    }
  });
  if (!m.tall) return;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int g = threadIdx.x + k * 256, r = g >> 3, col = (g & 7) * 8;
    float u[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) u[e] = turn[r][col + e];
    if (c.first + r < m.m && c.row + col < m.n) store_planes(x + (int64_t)(c.first + r) * 2 * m.n, c.row + col, u);
  }
}

// ---- the products ------------------------------------------------------------------------------------------------------
__device__ __forceinline__ f16_t* chain_at(const OrthoTables& t, const OrthoMat& m, int buf) {
  return (f16_t*)(t.ws + m.chain) + (int64_t)buf * 2 * m.m * m.m;
}

// dst = alpha * sum + beta * extra + diag * identity at eight neighbouring places of a symmetric matrix
struct Eight { float v[8]; };
__device__ __forceinline__ Eight extra_of(const OrthoTables& t, const OrthoMat& m, const OrthoOp& op, int r, int c) {
  Eight x = {};
  if (op.extra >= 0) load_planes(chain_at(t, m, op.extra) + (int64_t)r * 2 * m.m, c, x.v);
  return x;
}
__device__ __forceinline__ void combine(const OrthoOp& op, int r, int c, float (&v)[8], const Eight& x) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    v[e] = __fmaf_rn(op.alpha, v[e], op.beta * x.v[e]);
    if (r == c + e) v[e] += op.diag;
  }
}
__device__ __forceinline__ void chain_store(const OrthoTables& t, const OrthoMat& m, const OrthoOp& op, int r, int c, const float (&v)[8]) {
  store_planes(chain_at(t, m, op.dst) + (int64_t)r * 2 * m.m, c, v);
}

// a finished tile of a symmetric matrix, or a part of its sum
template <class G>
__device__ __forceinline__ void symmetric_out(unsigned char* smem, const OrthoTables& t, const OrthoMat& m, const OrthoWork& w, const OrthoOp& op,
                                              int slot0, int rows, int cols, const typename G::Acc& acc) {
  const int r0 = w.tm * G::EDGE, c0 = w.tn * G::EDGE;
  if (w.slot >= 0) {
    float* s = t.slots + (int64_t)(slot0 + w.slot) * (G::EDGE * G::EDGE);
    G::template out<false, false>(smem, acc, rows, cols, [](int, int, int) { return 0; },
                           [&](int, int r, int c, float (&v)[8], int, int) { store_f32<float, 8>(s + r * G::EDGE + c, v); });
  } else {
    G::out_symmetric(smem, acc, rows, cols, w.tm != w.tn, [&](int r, int c) { return extra_of(t, m, op, r0 + r, c0 + c); },
                     [&](int r, int c, float (&v)[8], const Eight& x) { combine(op, r0 + r, c0 + c, v, x); },
                     [&](int r, int c, float (&v)[8]) { chain_store(t, m, op, r0 + r, c0 + c, v); },
                     [&](int c, int r, float (&v)[8]) { chain_store(t, m, op, c0 + c, r0 + r, v); });
  }
}

#define ORTHO_BOUNDS(W) __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(W == 128 ? 1 : 2, W == 128 ? 1 : 8)))

// X X^T
template <int W>
__global__ void ORTHO_BOUNDS(W) gram_kernel(OrthoTables t, const OrthoWork* __restrict__ works, int src, OrthoOp op) {
  typedef Tile<f16_t, 2, W, false, false> G;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  const OrthoWork w = works[blockIdx.x];
  if (w.mat < 0) return;
  const OrthoMat& m = t.mats[w.mat];
  const f16_t* x = (const f16_t*)(t.ws + m.x[src]) + 2 * w.k0;
  const int ld = 2 * m.n, r0 = w.tm * G::EDGE, c0 = w.tn * G::EDGE;
  const int rows = min(G::EDGE, m.m - r0), cols = min(G::EDGE, m.m - c0);
  typename G::Acc acc;
  G::product(smem, Operand<f16_t>{x + (int64_t)r0 * ld, ld, rows}, Operand<f16_t>{x + (int64_t)c0 * ld, ld, cols}, w.k1 - w.k0, acc);
  symmetric_out<G>(smem, t, m, w, op, 0, rows, cols, acc);
}

// The parts of a tile's sum, added in order: a block has 32 x 32 values.  The second half of the blocks: of the second operation.
__global__ void __launch_bounds__(256) join_kernel(OrthoTables t, const OrthoJoin* __restrict__ joins, int njoins, int slots, int edge,
                                                   OrthoOp op0, OrthoOp op1) {
  __shared__ float area[32][33];
  const int per = edge / 32, sub = blockIdx.x % (per * per), tile = blockIdx.x / (per * per);
  const bool second = tile >= njoins;
  const OrthoOp op = second ? op1 : op0;
  const OrthoJoin j = joins[second ? tile - njoins : tile];
  const OrthoMat& m = t.mats[j.mat];
  const int sr = sub / per * 32, sc = sub % per * 32, r0 = j.tm * edge + sr, c0 = j.tn * edge + sc;
  if (r0 >= m.m || c0 >= m.m) return;
  const int q = threadIdx.x & 127, lr = q >> 2, lc = (q & 3) * 8, half = threadIdx.x >> 7;
  {
    const int r = threadIdx.x >> 3, c = (threadIdx.x & 7) * 4;
    const float* s = t.slots + (int64_t)(j.slot + (second ? slots : 0)) * edge * edge + (sr + r) * edge + sc + c;
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    for (int p = 0; p < j.parts; ++p) {
      float x[4];
      load_f32<float, 4>(s + (int64_t)p * edge * edge, x);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += x[e];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) area[r][c + e] = v[e];
  }
  __syncthreads();
  float v[8];
  if (half == 0) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = area[lr][lc + e];
    combine(op, r0 + lr, c0 + lc, v, extra_of(t, m, op, r0 + lr, c0 + lc));
    chain_store(t, m, op, r0 + lr, c0 + lc, v);
  } else if (j.tm != j.tn) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = area[lc + e][lr];
    combine(op, c0 + lr, r0 + lc, v, extra_of(t, m, op, c0 + lr, r0 + lc));
    chain_store(t, m, op, c0 + lr, r0 + lc, v);
  }
}

// products of the m x m matrices; the second half of the blocks: the second operation
template <int W>
__global__ void ORTHO_BOUNDS(W) chain_kernel(OrthoTables t, const OrthoWork* __restrict__ works, int n, int slots, OrthoOp op0, OrthoOp op1) {
  typedef Tile<f16_t, 2, W, false, false> G;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  const bool second = (int)blockIdx.x >= n;
  const OrthoWork w = works[second ? blockIdx.x - n : blockIdx.x];
  if (w.mat < 0) return;
  const OrthoOp op = second ? op1 : op0;
  const OrthoMat& m = t.mats[w.mat];
  const int ld = 2 * m.m, r0 = w.tm * G::EDGE, c0 = w.tn * G::EDGE;
  const int rows = min(G::EDGE, m.m - r0), cols = min(G::EDGE, m.m - c0);
  typename G::Acc acc;
  G::product(smem, Operand<f16_t>{chain_at(t, m, op.a) + (int64_t)r0 * ld + 2 * w.k0, ld, rows},
             Operand<f16_t>{chain_at(t, m, op.b) + (int64_t)c0 * ld + 2 * w.k0, ld, cols}, w.k1 - w.k0, acc);
  symmetric_out<G>(smem, t, m, w, op, second ? slots : 0, rows, cols, acc);
}

struct Target {
  void* o;                               // orthogonalize
  float* w; void* w16; int w16_bf16;     // muon
  float keep, lr; int scale_mode;        // keep: 1 - lr * weight_decay
};
enum { TO_PLANES = -1 };  // else the precision of o, or 3: muon

// Q X.  OUT: TO_PLANES, the precision of o, or 3 (weights)
template <int W, int OUT>
__global__ void ORTHO_BOUNDS(W) apply_kernel(OrthoTables t, const OrthoWork* __restrict__ works, int src, OrthoOp op, Target out) {
  typedef Tile<f16_t, 2, W, false, true> G;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  if (OUT == 3 && t.skip[0]) return;
  const OrthoWork w = works[blockIdx.x];
  if (w.mat < 0) return;
  const OrthoMat& m = t.mats[w.mat];
  const int r0 = w.tm * G::EDGE, c0 = w.tn * G::EDGE;
  const int rows = min(G::EDGE, m.m - r0), cols = min(G::EDGE, m.n - c0);
  typename G::Acc acc;
  G::product(smem, Operand<f16_t>{chain_at(t, m, op.a) + (int64_t)r0 * 2 * m.m, 2 * m.m, rows},
             Operand<f16_t>{(const f16_t*)(t.ws + m.x[src]) + 2 * c0, 2 * m.n, cols}, m.m, acc);
  float lr = 0.f;
  if (OUT == 3) {
    const double ratio = out.scale_mode == OPTORCH_SCALE_ASPECT ? fmax(1., (double)m.rows / m.cols)
                         : out.scale_mode == OPTORCH_SCALE_RMS ? 0.04 * max(m.rows, m.cols) : 1.;
    lr = (float)(out.lr * sqrt(ratio));
  }
  // eight neighbouring columns of the caller's matrix: its weights, and what becomes of them
  auto ask = [&](int r, int c) {
    Eight x = {};
    const int n = min(8, m.cols - c);
    if (OUT == 3 && r < m.rows && n > 0) get8((const float*)out.w + m.offset + r * m.ld + c, n, x.v);
    return x;
  };
  auto give = [&](int r, int c, float (&v)[8], const Eight& x) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] *= op.alpha;
    if (OUT == TO_PLANES) {
      store_planes((f16_t*)(t.ws + m.x[src ^ 1]) + (int64_t)r * 2 * m.n, c, v);
      return;
    }
    const int n = min(8, m.cols - c);
    if (r >= m.rows || n <= 0) return;
    const int64_t at = m.offset + r * m.ld + c;
    if (OUT == OPTORCH_FP32) put8((float*)out.o + at, n, v);
    if (OUT == OPTORCH_BF16) put8((bf16_t*)out.o + at, n, v);
    if (OUT == OPTORCH_FP16) put8((f16_t*)out.o + at, n, v);
    if (OUT == 3) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = __fmaf_rn(-lr, v[e], x.v[e] * out.keep);
      put8(out.w + at, n, v);
      if (out.w16) {
        if (out.w16_bf16) put8((bf16_t*)out.w16 + at, n, v);
        else put8((f16_t*)out.w16 + at, n, v);
      }
    }
  };
  if (OUT != TO_PLANES && m.tall)
    G::template out<true, false>(smem, acc, rows, cols, [&](int c, int r, int) { return ask(c0 + c, r0 + r); },
                          [&](int, int c, int r, float (&v)[8], int, const Eight& x) { give(c0 + c, r0 + r, v, x); });
  else
    G::template out<false, false>(smem, acc, rows, cols, [&](int r, int c, int) { return ask(r0 + r, c0 + c); },
                           [&](int, int r, int c, float (&v)[8], int, const Eight& x) { give(r0 + r, c0 + c, v, x); });
}

template <class K, class... A> void run(K k, int n, size_t lds, hipStream_t st, A... a) {
  if (lds > 65536) (void)hipFuncSetAttribute((const void*)k, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  OSEQ_LAUNCH(k, dim3(n), dim3(256), lds, st, a...);
}
template <int W> constexpr size_t lds_of() { return Tile<f16_t, 2, W, false, false>::LDS; }

template <int OUT> void run_apply(hipStream_t st, const OrthoTables& t, const OrthoList& l, const OrthoWork* w, const OrthoLaunch& c, const Target& o) {
  if (l.w == 128) run(apply_kernel<128, OUT>, l.n, lds_of<128>(), st, t, w, c.src, c.op[0], o);
  else if (l.w == 64) run(apply_kernel<64, OUT>, l.n, lds_of<64>(), st, t, w, c.src, c.op[0], o);
  else run(apply_kernel<32, OUT>, l.n, lds_of<32>(), st, t, w, c.src, c.op[0], o);
}

template <class G, bool MUON> void run_elements(hipStream_t st, const OrthoTables& t, const OrthoPlanHost& p, const Source& s, int32_t* skipped) {
  OSEQ_LAUNCH((norms_kernel<G, MUON>), dim3(t.nchunks), dim3(256), 0, st, t, s);
  OSEQ_LAUNCH(scales_kernel, dim3(t.nmat), dim3(256), 0, st, t, p.eps, (double)p.first_scale);
  OSEQ_LAUNCH((planes_kernel<G, MUON>), dim3(t.nchunks), dim3(256), 0, st, t, s, skipped);
}

}  // namespace

void launch_ortho(hipStream_t st, const OrthoPlanHost& p, char* ws, const OrthoRun& r) {
  OrthoTables t;
  t.ws = ws;
  t.mats = (const OrthoMat*)(ws + p.off_mats); t.nmat = (int)p.mats.size();
  t.chunks = (const OrthoChunk*)(ws + p.off_chunks); t.nchunks = (int)p.chunks.size();
  t.partial = (double*)(ws + p.off_partial);
  t.scale = (double*)(ws + p.off_scale);
  t.bad = (int32_t*)(ws + p.off_bad); t.skip = t.bad + t.nmat;
  t.slots = (float*)(ws + p.off_slots);
  Source s = {};
  s.g = r.g;
  if (r.muon) { s.v = r.m.v; s.grad_scale = r.m.grad_scale; s.momentum = r.m.momentum; s.nesterov = r.m.nesterov; }
  if (r.muon) {
    if (r.g_precision == OPTORCH_FP32) run_elements<float, true>(st, t, p, s, r.m.skipped);
    else if (r.g_precision == OPTORCH_BF16) run_elements<bf16_t, true>(st, t, p, s, r.m.skipped);
    else run_elements<f16_t, true>(st, t, p, s, r.m.skipped);
  } else {
    if (r.g_precision == OPTORCH_FP32) run_elements<float, false>(st, t, p, s, nullptr);
    else if (r.g_precision == OPTORCH_BF16) run_elements<bf16_t, false>(st, t, p, s, nullptr);
    else run_elements<f16_t, false>(st, t, p, s, nullptr);
  }
  Target o = {};
  o.o = r.o;
  if (r.muon) {
    o.w = r.m.w; o.w16 = r.m.w16; o.w16_bf16 = r.m.w16_precision == OPTORCH_BF16;
    o.keep = (float)(1.0 - (double)r.m.lr * r.m.weight_decay); o.lr = r.m.lr; o.scale_mode = r.m.scale_mode;
  }
  const OrthoWork* works = (const OrthoWork*)(ws + p.off_works);
  const OrthoJoin* joins = (const OrthoJoin*)(ws + p.off_joins);
  auto join = [&](const OrthoList& l, const OrthoLaunch& c) {
    if (!l.joins) return;
    const int edge = 2 * l.w, per = edge / 32;
    run(join_kernel, l.joins * c.ops * per * per, 0, st, t, joins + l.join0, l.joins, l.slots, edge, c.op[0], c.op[1]);
  };
  // what is stored in fp32 as it is takes the more exact steps
  for (const OrthoLaunch& c : p.launches[!r.muon && r.o_precision == OPTORCH_FP32]) {
    if (c.kind == OL_GRAM) {
      const OrthoWork* w = works + p.gram.work0;
      if (p.gram.w == 128) run(gram_kernel<128>, p.gram.n, lds_of<128>(), st, t, w, c.src, c.op[0]);
      else if (p.gram.w == 64) run(gram_kernel<64>, p.gram.n, lds_of<64>(), st, t, w, c.src, c.op[0]);
      else run(gram_kernel<32>, p.gram.n, lds_of<32>(), st, t, w, c.src, c.op[0]);
      join(p.gram, c);
    } else if (c.kind == OL_CHAIN) {
      const OrthoList& l = p.chain;
      const OrthoWork* w = works + l.work0;
      if (l.w == 128) run(chain_kernel<128>, l.n * c.ops, lds_of<128>(), st, t, w, l.n, l.slots, c.op[0], c.op[1]);
      else if (l.w == 64) run(chain_kernel<64>, l.n * c.ops, lds_of<64>(), st, t, w, l.n, l.slots, c.op[0], c.op[1]);
      else run(chain_kernel<32>, l.n * c.ops, lds_of<32>(), st, t, w, l.n, l.slots, c.op[0], c.op[1]);
      join(l, c);
    } else {
      const OrthoWork* w = works + p.apply.work0;
      if (!c.last) run_apply<TO_PLANES>(st, t, p.apply, w, c, o);
      else if (r.muon) run_apply<3>(st, t, p.apply, w, c, o);
      else if (r.o_precision == OPTORCH_FP32) run_apply<OPTORCH_FP32>(st, t, p.apply, w, c, o);
      else if (r.o_precision == OPTORCH_BF16) run_apply<OPTORCH_BF16>(st, t, p.apply, w, c, o);
      else run_apply<OPTORCH_FP16>(st, t, p.apply, w, c, o);
    }
  }
}

}  // namespace oseq
