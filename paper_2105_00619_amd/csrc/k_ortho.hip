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

template <class T> __device__ __forceinline__ void get8(const T* p, int n, float (&v)[8]) {
  if (n == 8 && ((uintptr_t)p & 15) == 0) {
    load_f32<T, 8>(p, v);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < n ? to_f32(p[e]) : 0.f;
  }
}
template <class T> __device__ __forceinline__ void put8(T* p, int n, const float (&v)[8]) {
  if (n == 8 && ((uintptr_t)p & 15) == 0) {
    store_f32<T, 8>(p, v);
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

template <class G, bool MUON>
__global__ void __launch_bounds__(256) norms_kernel(OrthoTables t, Source s) {
  __shared__ double part[4];
  const OrthoChunk c = t.chunks[blockIdx.x];
  const OrthoMat& m = t.mats[c.mat];
  const int c8 = m.cp / 8, last = min(c.first + ORTHO_GROUPS, m.rows * c8);
  double sum = 0.;
  for (int g = c.first + threadIdx.x; g < last; g += 256) {
    const int r = g / c8, col = (g - r * c8) * 8;
    float u[8], vn[8];
    source8<G, MUON>(s, m.offset + r * m.ld + col, min(8, m.cols - col), u, vn);
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (col + e < m.cols) sum = fma((double)u[e], (double)u[e], sum);
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x == 0) t.partial[blockIdx.x] = (part[0] + part[1]) + (part[2] + part[3]);
}

__global__ void __launch_bounds__(64) scales_kernel(OrthoTables t, float eps, double times) {
  const OrthoMat& m = t.mats[blockIdx.x];
  double sum = 0.;
  for (int i = threadIdx.x; i < m.chunks; i += 64) sum += t.partial[m.chunk0 + i];
#pragma unroll
  for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
  if (threadIdx.x == 0) {
    const double norm = sqrt(sum);
    t.scale[blockIdx.x] = times / (norm < (double)eps ? (double)eps : norm);  // (NaN stays NaN)
    t.bad[blockIdx.x] = sum <= 1.7976931348623157e308 ? 0 : 1;
  }
}

template <class G, bool MUON>
__global__ void __launch_bounds__(256) planes_kernel(OrthoTables t, Source s, int32_t* skipped) {
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
  const int c8 = m.cp / 8, last = min(c.first + ORTHO_GROUPS, m.rp * c8);
  const double scale = t.scale[c.mat];
  f16_t* x = (f16_t*)(t.ws + m.x[0]);
  for (int g = c.first + threadIdx.x; g < last; g += 256) {
    const int r = g / c8, col = (g - r * c8) * 8, n = r < m.rows ? min(8, m.cols - col) : 0;
    float u[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, vn[8];
    if (n > 0) {
      const int64_t at = m.offset + r * m.ld + col;
      source8<G, MUON>(s, at, n, u, vn);
      if (MUON && !skip) put8(s.v + at, n, vn);
#pragma unroll
      for (int e = 0; e < 8; ++e) u[e] = e < n ? (float)((double)u[e] * scale) : 0.f;
    }
    store_planes(x + (int64_t)r * 2 * m.cp, col, u);
  }
}

// ---- the products ------------------------------------------------------------------------------------------------------
__device__ __forceinline__ f16_t* chain_at(const OrthoTables& t, const OrthoMat& m, int buf) {
  return (f16_t*)(t.ws + m.chain) + (int64_t)buf * 2 * m.mp * m.mp;
}

// dst = alpha * sum + beta * extra + diag * identity at eight neighbouring places of a symmetric matrix's planes
__device__ __forceinline__ void chain_store(const OrthoTables& t, const OrthoMat& m, const OrthoOp& op, int r, int c, float (&v)[8]) {
  const int64_t row = (int64_t)r * 2 * m.mp;
  float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (op.extra >= 0) load_planes(chain_at(t, m, op.extra) + row, c, x);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    v[e] = __fmaf_rn(op.alpha, v[e], op.beta * x[e]);
    if (r == c + e) v[e] += op.diag;
  }
  store_planes(chain_at(t, m, op.dst) + row, c, v);
}

template <int W, bool TALL>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(W == 128 ? 1 : 2, W == 128 ? 1 : 8)))
gram_kernel(OrthoTables t, const OrthoWork* __restrict__ works, int src, OrthoOp op) {
  typedef Tile<f16_t, 2, W, TALL, TALL> G;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  const OrthoWork w = works[blockIdx.x];
  const OrthoMat& m = t.mats[w.mat];
  const f16_t* x = (const f16_t*)(t.ws + m.x[src]);
  const int ld = 2 * m.cp, r0 = w.tm * G::EDGE, c0 = w.tn * G::EDGE;
  const int rows = min(G::EDGE, m.mp - r0), cols = min(G::EDGE, m.mp - c0);
  Operand<f16_t> a{x + (TALL ? (int64_t)w.k0 * ld + 2 * r0 : (int64_t)r0 * ld + 2 * w.k0), ld, rows};
  Operand<f16_t> b{x + (TALL ? (int64_t)w.k0 * ld + 2 * c0 : (int64_t)c0 * ld + 2 * w.k0), ld, cols};
  typename G::Acc acc;
  G::product(smem, a, b, w.k1 - w.k0, acc);
  if (w.slot >= 0) {
    float* s = t.slots + (int64_t)w.slot * (G::EDGE * G::EDGE);
    G::out(smem, acc, rows, cols, [&](int, int r, int c, float (&v)[8], int) { store_f32<float, 8>(s + r * G::EDGE + c, v); },
           [](int, int, float (&)[8], int) {}, false);
  } else {
    G::out(smem, acc, rows, cols, [&](int, int r, int c, float (&v)[8], int) { chain_store(t, m, op, r0 + r, c0 + c, v); },
           [&](int c, int r, float (&v)[8], int) { chain_store(t, m, op, c0 + c, r0 + r, v); }, w.tm != w.tn);
  }
}

// The parts of a tile of X X^T, added in order: a block has 32 x 32 values
__global__ void __launch_bounds__(256) gram_join_kernel(OrthoTables t, const OrthoJoin* __restrict__ joins, int edge, OrthoOp op) {
  __shared__ float area[32][33];
  const int per = edge / 32, sub = blockIdx.x % (per * per);
  const OrthoJoin j = joins[blockIdx.x / (per * per)];
  const OrthoMat& m = t.mats[j.mat];
  const int sr = sub / per * 32, sc = sub % per * 32, r0 = j.tm * edge + sr, c0 = j.tn * edge + sc;
  if (r0 >= m.mp || c0 >= m.mp) return;
  for (int i = threadIdx.x; i < 1024; i += 256) {
    const int r = i >> 5, c = i & 31;
    const float* s = t.slots + (int64_t)j.slot * edge * edge + (sr + r) * edge + sc + c;
    float v = 0.f;
    if (r0 + r < m.mp && c0 + c < m.mp)
      for (int p = 0; p < j.parts; ++p) v += s[(int64_t)p * edge * edge];
    area[r][c] = v;
  }
  __syncthreads();
  const int half = threadIdx.x >> 7, q = threadIdx.x & 127, r = q >> 2, c = (q & 3) * 8;
  float v[8];
  if (half == 0) {
    if (r0 + r < m.mp && c0 + c < m.mp) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = area[r][c + e];
      chain_store(t, m, op, r0 + r, c0 + c, v);
    }
  } else if (j.tm != j.tn) {
    if (c0 + r < m.mp && r0 + c < m.mp) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = area[c + e][r];
      chain_store(t, m, op, c0 + r, r0 + c, v);
    }
  }
}

template <int W>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(W == 128 ? 1 : 2, W == 128 ? 1 : 8)))
chain_kernel(OrthoTables t, const OrthoWork* __restrict__ works, int n, OrthoOp op0, OrthoOp op1) {
  typedef Tile<f16_t, 2, W, false, false> G;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  const bool second = (int)blockIdx.x >= n;
  const OrthoWork w = works[second ? blockIdx.x - n : blockIdx.x];
  const OrthoOp op = second ? op1 : op0;
  const OrthoMat& m = t.mats[w.mat];
  const int ld = 2 * m.mp, r0 = w.tm * G::EDGE, c0 = w.tn * G::EDGE;
  const int rows = min(G::EDGE, m.mp - r0), cols = min(G::EDGE, m.mp - c0);
  Operand<f16_t> a{chain_at(t, m, op.a) + (int64_t)r0 * ld, ld, rows};
  Operand<f16_t> b{chain_at(t, m, op.b) + (int64_t)c0 * ld, ld, cols};
  typename G::Acc acc;
  G::product(smem, a, b, m.mp, acc);
  G::out(smem, acc, rows, cols, [&](int, int r, int c, float (&v)[8], int) { chain_store(t, m, op, r0 + r, c0 + c, v); },
         [&](int c, int r, float (&v)[8], int) { chain_store(t, m, op, c0 + c, r0 + r, v); }, w.tm != w.tn);
}

struct Target {
  void* o;                               // orthogonalize
  float* w; void* w16; int w16_bf16;     // muon
  float keep, lr; int scale_mode;        // keep: 1 - lr * weight_decay
};
enum { TO_PLANES = -1 };  // else the precision of o, or 3: muon

// OUT: TO_PLANES, the precision of o, or 3 (weights)
template <int W, bool TALL, int OUT>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(W == 128 ? 1 : 2, W == 128 ? 1 : 8)))
apply_kernel(OrthoTables t, const OrthoWork* __restrict__ works, int src, OrthoOp op, Target out) {
  typedef Tile<f16_t, 2, W, false, !TALL> G;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  if (OUT == 3 && t.skip[0]) return;
  const OrthoWork w = works[blockIdx.x];
  const OrthoMat& m = t.mats[w.mat];
  const f16_t* x = (const f16_t*)(t.ws + m.x[src]);
  const f16_t* q = chain_at(t, m, op.a);
  const int r0 = w.tm * G::EDGE, c0 = w.tn * G::EDGE;
  const int rows = min(G::EDGE, m.rp - r0), cols = min(G::EDGE, m.cp - c0);
  Operand<f16_t> a, b;
  if (TALL) {
    a = {x + (int64_t)r0 * 2 * m.cp, 2 * m.cp, rows};
    b = {q + (int64_t)c0 * 2 * m.mp, 2 * m.mp, cols};
  } else {
    a = {q + (int64_t)r0 * 2 * m.mp, 2 * m.mp, rows};
    b = {x + 2 * c0, 2 * m.cp, cols};
  }
  typename G::Acc acc;
  G::product(smem, a, b, m.mp, acc);
  const int real_cols = m.cols;
  float lr = 0.f;
  if (OUT == 3) {
    const double ratio = out.scale_mode == OPTORCH_SCALE_ASPECT ? fmax(1., (double)m.rows / m.cols)
                         : out.scale_mode == OPTORCH_SCALE_RMS ? 0.04 * max(m.rows, m.cols) : 1.;
    lr = (float)(out.lr * sqrt(ratio));
  }
  G::out(smem, acc, rows, cols,
         [&](int, int r, int c, float (&v)[8], int) {
           r += r0; c += c0;
#pragma unroll
           for (int e = 0; e < 8; ++e) v[e] *= op.alpha;
           if (OUT == TO_PLANES) {
             store_planes((f16_t*)(t.ws + m.x[src ^ 1]) + (int64_t)r * 2 * m.cp, c, v);
             return;
           }
           const int n = min(8, real_cols - c);
           if (r >= m.rows || n <= 0) return;
           const int64_t at = m.offset + r * m.ld + c;
           if (OUT == OPTORCH_FP32) put8((float*)out.o + at, n, v);
           if (OUT == OPTORCH_BF16) put8((bf16_t*)out.o + at, n, v);
           if (OUT == OPTORCH_FP16) put8((f16_t*)out.o + at, n, v);
           if (OUT == 3) {
             float w0[8];
             get8((const float*)out.w + at, n, w0);
#pragma unroll
             for (int e = 0; e < 8; ++e) v[e] = __fmaf_rn(-lr, v[e], w0[e] * out.keep);
             put8(out.w + at, n, v);
             if (out.w16) {
               if (out.w16_bf16) put8((bf16_t*)out.w16 + at, n, v);
               else put8((f16_t*)out.w16 + at, n, v);
             }
           }
         },
         [](int, int, float (&)[8], int) {}, false);
}

template <class K> void allow_lds(K k, size_t lds) {
  if (lds > 65536) (void)hipFuncSetAttribute((const void*)k, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
}

template <int W, bool TALL> void run_gram(hipStream_t st, const OrthoTables& t, const OrthoWork* w, int n, const OrthoLaunch& l) {
  const size_t lds = Tile<f16_t, 2, W, TALL, TALL>::LDS;
  allow_lds(gram_kernel<W, TALL>, lds);
  OSEQ_LAUNCH((gram_kernel<W, TALL>), dim3(n), dim3(256), lds, st, t, w, l.src, l.op[0]);
}
template <bool TALL> void run_gram_of(int w, hipStream_t st, const OrthoTables& t, const OrthoWork* ws, int n, const OrthoLaunch& l) {
  if (!n) return;
  if (w == 128) run_gram<128, TALL>(st, t, ws, n, l);
  else if (w == 64) run_gram<64, TALL>(st, t, ws, n, l);
  else run_gram<32, TALL>(st, t, ws, n, l);
}
template <int W> void run_chain(hipStream_t st, const OrthoTables& t, const OrthoWork* w, int n, const OrthoLaunch& l) {
  const size_t lds = Tile<f16_t, 2, W, false, false>::LDS;
  allow_lds(chain_kernel<W>, lds);
  OSEQ_LAUNCH(chain_kernel<W>, dim3(n * l.ops), dim3(256), lds, st, t, w, n, l.op[0], l.op[1]);
}
template <int W, bool TALL, int OUT> void run_apply(hipStream_t st, const OrthoTables& t, const OrthoWork* w, int n, const OrthoLaunch& l, const Target& o) {
  const size_t lds = Tile<f16_t, 2, W, false, !TALL>::LDS;
  allow_lds(apply_kernel<W, TALL, OUT>, lds);
  OSEQ_LAUNCH((apply_kernel<W, TALL, OUT>), dim3(n), dim3(256), lds, st, t, w, l.src, l.op[0], o);
}
template <bool TALL, int OUT> void run_apply_w(int w, hipStream_t st, const OrthoTables& t, const OrthoWork* ws, int n, const OrthoLaunch& l, const Target& o) {
  if (w == 128) run_apply<128, TALL, OUT>(st, t, ws, n, l, o);
  else if (w == 64) run_apply<64, TALL, OUT>(st, t, ws, n, l, o);
  else run_apply<32, TALL, OUT>(st, t, ws, n, l, o);
}
template <bool TALL> void run_apply_of(int w, hipStream_t st, const OrthoTables& t, const OrthoWork* ws, int n, const OrthoLaunch& l, const OrthoRun& r, const Target& o) {
  if (!n) return;
  if (!l.last) run_apply_w<TALL, TO_PLANES>(w, st, t, ws, n, l, o);
  else if (r.muon) run_apply_w<TALL, 3>(w, st, t, ws, n, l, o);
  else if (r.o_precision == OPTORCH_FP32) run_apply_w<TALL, OPTORCH_FP32>(w, st, t, ws, n, l, o);
  else if (r.o_precision == OPTORCH_BF16) run_apply_w<TALL, OPTORCH_BF16>(w, st, t, ws, n, l, o);
  else run_apply_w<TALL, OPTORCH_FP16>(w, st, t, ws, n, l, o);
}

template <class G, bool MUON> void run_elements(hipStream_t st, const OrthoTables& t, const OrthoPlanHost& p, const Source& s, int32_t* skipped) {
  OSEQ_LAUNCH((norms_kernel<G, MUON>), dim3(t.nchunks), dim3(256), 0, st, t, s);
  OSEQ_LAUNCH(scales_kernel, dim3(t.nmat), dim3(64), 0, st, t, p.eps, (double)p.first_scale);
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
  for (const OrthoLaunch& l : p.launches) {
    if (l.kind == OL_GRAM) {
      run_gram_of<false>(p.w_gram, st, t, works + p.gram[0].off, p.gram[0].n, l);
      run_gram_of<true>(p.w_gram, st, t, works + p.gram[1].off, p.gram[1].n, l);
      if (!p.joins.empty()) {
        const int edge = 2 * p.w_gram, per = edge / 32;
        OSEQ_LAUNCH(gram_join_kernel, dim3((int)p.joins.size() * per * per), dim3(256), 0, st, t, (const OrthoJoin*)(ws + p.off_joins), edge, l.op[0]);
      }
    } else if (l.kind == OL_CHAIN) {
      const OrthoWork* w = works + p.chain.off;
      if (p.w_chain == 128) run_chain<128>(st, t, w, p.chain.n, l);
      else if (p.w_chain == 64) run_chain<64>(st, t, w, p.chain.n, l);
      else run_chain<32>(st, t, w, p.chain.n, l);
    } else {
      run_apply_of<false>(p.w_apply, st, t, works + p.apply[0].off, p.apply[0].n, l, r, o);
      run_apply_of<true>(p.w_apply, st, t, works + p.apply[1].off, p.apply[1].n, l, r, o);
    }
  }
}

}  // namespace oseq
