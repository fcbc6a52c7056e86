// Orthogonalised updates: the kernels of the plan made in ortho.cpp.  Every launch does its part for all matrices of the list; a
// block finds its matrix and tile in a table.
//   norms    sum of squares of each piece of a matrix, in 64 bits
//   scales   1 / max(norm, eps) per matrix, and whether all its elements are finite (with few pieces: part of the next)
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

// f(place in the flat vectors, n, row of X, column) for groups of eight neighbouring columns of a piece, n of them inside
// (0: none); a tall matrix' groups run along its own columns: row and column of the transposed group's first value
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

// sum of squares of a matrix from its pieces', by a block, and the scale of its first iterate
__device__ __forceinline__ double norm2_of(const OrthoTables& t, const OrthoMat& m, double (&part)[4]) {
  double sum = 0.;
  for (int i = threadIdx.x; i < m.chunks; i += 256) sum += t.partial[m.chunk0 + i];
#pragma unroll
  for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
  __syncthreads();
  return (part[0] + part[1]) + (part[2] + part[3]);
}
__device__ __forceinline__ double scale_of(double norm2, float eps, double times) {
  const double norm = sqrt(norm2);
  return times / (norm < (double)eps ? (double)eps : norm);  // (NaN stays NaN)
}

__global__ void __launch_bounds__(256) scales_kernel(OrthoTables t, float eps, double times) {
  __shared__ double part[4];
  const double sum = norm2_of(t, t.mats[blockIdx.x], part);
  if (threadIdx.x == 0) {
    t.scale[blockIdx.x] = scale_of(sum, eps, times);
    t.bad[blockIdx.x] = sum <= 1.7976931348623157e308 ? 0 : 1;
  }
}

// FEW pieces (FEW_CHUNKS) in all: every block makes its scale from the pieces' sums itself, which saves a launch
constexpr int FEW_CHUNKS = 256;
template <class G, bool MUON, bool FEW>
__global__ void __launch_bounds__(256) planes_kernel(OrthoTables t, Source s, int32_t* skipped, float eps, double times) {
  __shared__ float turn[128][65];  // a tall matrix' piece on its way to its transposed place
  __shared__ double part[4];
  const OrthoChunk c = t.chunks[blockIdx.x];
  const OrthoMat& m = t.mats[c.mat];
  bool skip = false;
  if (MUON) {
    bool any = false;
    if (FEW) any = (int)threadIdx.x < t.nchunks && !(t.partial[threadIdx.x] <= 1.7976931348623157e308);
    else for (int i = threadIdx.x; i < t.nmat; i += 256) any |= t.bad[i] != 0;
    skip = __syncthreads_or(any);
    if (blockIdx.x == 0 && threadIdx.x == 0) {
      t.skip[0] = skip;
      if (skipped) *skipped = skip;
    }
  }
  const double scale = FEW ? scale_of(norm2_of(t, m, part), eps, times) : t.scale[c.mat];
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

// ---- small matrices ----------------------------------------------------------------------------------------------------
// All the m x m products between two iterates of a matrix with m <= 128, by one block, a wavefront for each 32 x 32 tile of
// the lower triangle.  A (then C = P A, then the new A) and P stay in LDS, Q in memory.  A launch for each product takes
// 3.5 (m = 32) to 5 us (m = 128), most of it waiting for memory and the next launch; here a product takes 1.1 to 3.6, half
// of that the instructions that round and store a tile: update of matrices of 8 x 27, 8 x 72 and 10 x 8 71 -> 42 us with up
// to three steps between iterates (49 with two, as they are now), 100 x 512 orthogonalised 105 -> 96.
//
// LDS: rows as in memory, 512 bytes apart, the 16-byte piece i of row r at i ^ (r & 15), so that sixteen neighbouring rows
// touch all banks and an address is a lane's own part with a constant in exclusive or and a constant offset.
constexpr int SMALL_PITCH = 4 * ORTHO_SMALL;
constexpr int small_lds(int m) { return 2 * m * SMALL_PITCH; }
typedef Op<f16_t>::V V8;
typedef Vec<f16_t, 4> V4;

__global__ void __launch_bounds__(640) small_chain_kernel(OrthoTables t, OrthoOps ops) {
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  const OrthoMat& mat = t.mats[blockIdx.x];
  constexpr int pitch = SMALL_PITCH;
  const int m = mat.m, nt = m / 32;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int ti = 0;
  while ((ti + 1) * (ti + 2) / 2 <= wave) ++ti;
  const int tj = wave - ti * (ti + 1) / 2, r0 = ti * 32, c0 = tj * 32, l = lane & 31, h = lane >> 5;
  const bool mine = ti < nt;
  const uint32_t area[2] = {0u, (uint32_t)(m * pitch)};
  auto fold = [](int r) { return (uint32_t)(r & 15); };
  // whole matrices between memory and LDS
  const int per = m / 4, inverse = (1 << 18) / per + 1;  // (exact up to i = 4096)
  auto piece_at = [&](int i) {
    const int r = (i * inverse) >> 18;
    return (uint32_t)(r * pitch) + (((uint32_t)(i - r * per) ^ fold(r)) << 4);
  };
  auto copy_out = [&](uint32_t from, int buf) {
    f16_t* d = chain_at(t, mat, buf);
    for (int i = threadIdx.x; i < m * per; i += blockDim.x)
      *reinterpret_cast<Vec<f16_t, 8>*>(d + i * 8) = *reinterpret_cast<const Vec<f16_t, 8>*>(smem + from + piece_at(i));
  };
  {
    const f16_t* a = chain_at(t, mat, OB_A);
    for (int i = threadIdx.x; i < m * per; i += blockDim.x)
      *reinterpret_cast<Vec<f16_t, 8>*>(smem + piece_at(i)) = *reinterpret_cast<const Vec<f16_t, 8>*>(a + i * 8);
  }
  __syncthreads();
  // a lane's part of the addresses: operands of the tile's rows and columns; four neighbouring rows of its column,
  // transposed; its column
  const uint32_t row_at = (uint32_t)((r0 + l) * pitch) + (((uint32_t)h ^ fold(l)) << 4), col_at = (uint32_t)((c0 + l) * pitch) + (((uint32_t)h ^ fold(l)) << 4);
  const uint32_t four_at = (uint32_t)((c0 + l) * pitch) + (((uint32_t)(ti * 8) ^ fold(l)) << 4) + h * 8;
  const uint32_t one_at = (((uint32_t)(tj * 8 + (l >> 3)) ^ (uint32_t)(4 * h)) << 4) + (l & 7) * 2;
  // Addresses of a store are made again each time: kept over the loop they spill
  auto fresh = [](uint32_t v) { asm volatile("" : "+v"(v)); return v; };
  auto operand = [&](uint32_t at, int k, int g, int plane) {
    return *reinterpret_cast<const V8*>(smem + (at ^ (uint32_t)((k * 8 + plane * 4 + g * 2) << 4)));
  };
  // (A tile is stored transposed and, off the diagonal, as it is.  On the diagonal the operands change places, so that
  // there too a product is stored as it is: transposed, what rounding leaves of asymmetry made results of m = 32 four times
  // less exact.)
  auto products = [&](v16f& acc, const V8& ah, const V8& al, const V8& bh, const V8& bl) {
    acc = Op<f16_t>::mma(ah, bl, acc);
    acc = Op<f16_t>::mma(al, bh, acc);
    acc = Op<f16_t>::mma(ah, bh, acc);
  };
  V4 hi[4], lo[4];  // a finished tile: four neighbouring rows at a time
  auto finish = [&](const OrthoOp& op, const v16f& acc, bool poly) {
    const uint32_t from = fresh(four_at);
    each<4>([&](auto q) {
      float v[4], w[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = op.alpha * acc[q * 4 + e];
      if (poly) {  // (A is symmetric)
        load_f32<f16_t, 4>(reinterpret_cast<const f16_t*>(smem + (from ^ (q * 16u))), w);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = __fmaf_rn(op.beta, w[e], v[e]);
        load_f32<f16_t, 4>(reinterpret_cast<const f16_t*>(smem + (from ^ (q * 16u + 64u))), w);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = __fmaf_rn(op.beta, w[e], v[e]);
        if (ti == tj) {
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] += 8 * q + 4 * h + e == l ? op.diag : 0.f;
        }
      }
      hi[q] = round_vec<f16_t, 4>(v);
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = v[e] - (float)hi[q].v[e];
      lo[q] = round_vec<f16_t, 4>(w);
    });
  };
  auto to_lds = [&](uint32_t to) {
    const uint32_t four = fresh(to + four_at);
    each<4>([&](auto q) {
      *reinterpret_cast<V4*>(smem + (four ^ (q * 16u))) = hi[q];
      *reinterpret_cast<V4*>(smem + (four ^ (q * 16u + 64u))) = lo[q];
    });
    if (ti == tj) return;
    const uint32_t row = fresh(to + (uint32_t)((r0 + 4 * h) * pitch) + one_at);
    each<16>([&](auto i) {  // (row r0 + 8 q + 4 h + e is folded by 8 (q & 1) + 4 h + e)
      constexpr int q = i / 4, e = i % 4;
      *reinterpret_cast<f16_t*>(smem + (row ^ ((8u * (q & 1) + e) << 4)) + (8 * q + e) * pitch) = hi[q].v[e];
      *reinterpret_cast<f16_t*>(smem + (row ^ ((8u * (q & 1) + e + 4u) << 4)) + (8 * q + e) * pitch) = lo[q].v[e];
    });
  };
  auto to_memory = [&](int buf) {
    f16_t* d = chain_at(t, mat, buf);
    const int ld = 2 * m;
    f16_t* four = d + fresh((c0 + l) * ld + ti * 64 + 4 * h);
    each<4>([&](auto q) {
      *reinterpret_cast<V4*>(four + 8 * q) = hi[q];
      *reinterpret_cast<V4*>(four + 8 * q + 32) = lo[q];
    });
    if (ti == tj) return;
    f16_t* one = d + fresh((r0 + 4 * h) * ld + tj * 64 + l);
    each<16>([&](auto i) {
      constexpr int q = i / 4, e = i % 4;
      one[0] = hi[q].v[e];
      one[32] = lo[q].v[e];
      one += e == 3 ? 5 * ld : ld;
    });
  };
  for (int o = 0; o < ops.n; ++o) {
    const OrthoOp op = ops.op[o];
    v16f acc;
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[e] = 0.f;
    const bool to_q = op.dst == OB_Q0 || op.dst == OB_Q1, poly = op.extra >= 0;
    if (poly) {  // P from A; the first one is Q too
      if (mine) {
        for (int k = 0; k < nt; ++k)
          each<2>([&](auto g) {
            products(acc, operand(row_at, k, g, 0), operand(row_at, k, g, 1), operand(col_at, k, g, 0), operand(col_at, k, g, 1));
          });
        finish(op, acc, true);
        to_lds(area[1]);
      }
      __syncthreads();
      if (to_q) copy_out(area[1], op.dst);
    } else if (to_q) {  // Q <- P Q
      if (mine) {
        const f16_t* q = chain_at(t, mat, op.b) + (c0 + l) * (2 * m) + h * 8;
        V8 b[ORTHO_SMALL / 32][4];  // (all of them on their way at once)
        each<ORTHO_SMALL / 32>([&](auto k) {
          each<4>([&](auto i) { b[k][i] = *reinterpret_cast<const V8*>(q + min((int)k, nt - 1) * 64 + i * 16); });
        });
        each<ORTHO_SMALL / 32>([&](auto k) {
          if (k < nt)
            each<2>([&](auto g) {
              const V8 ph = operand(area[1] + row_at, k, g, 0), pl = operand(area[1] + row_at, k, g, 1);
              if (ti == tj) products(acc, b[k][g], b[k][g + 2], ph, pl);
              else products(acc, ph, pl, b[k][g], b[k][g + 2]);
            });
        });
        finish(op, acc, false);
      }
      if (o + 1 < ops.n) {
        if (mine) to_memory(op.dst);
        __syncthreads();
      } else {  // (A's place is free)
        if (mine) to_lds(area[0]);
        __syncthreads();
        copy_out(area[0], op.dst);
      }
    } else {  // C from P and A, the new A from C and P: they take A's place, which every wavefront has read
      const bool swap = (op.a == OB_C) == (ti != tj);
      const uint32_t a_at = row_at + area[swap ? 0 : 1], b_at = col_at + area[swap ? 1 : 0];
      if (mine) {
        for (int k = 0; k < nt; ++k)
          each<2>([&](auto g) { products(acc, operand(a_at, k, g, 0), operand(a_at, k, g, 1), operand(b_at, k, g, 0), operand(b_at, k, g, 1)); });
        finish(op, acc, false);
      }
      __syncthreads();
      if (mine) to_lds(area[0]);
      __syncthreads();
    }
  }
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

void run_small(hipStream_t st, const OrthoTables& t, int m, const OrthoOps& ops) {
  const int tiles = m / 32 * (m / 32 + 1) / 2, lds = small_lds(m);
  if (lds > 65536) (void)hipFuncSetAttribute((const void*)small_chain_kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  OSEQ_LAUNCH(small_chain_kernel, dim3(t.nmat), dim3(tiles * 64), lds, st, t, ops);
}

template <class G, bool MUON> void run_elements(hipStream_t st, const OrthoTables& t, const OrthoPlanHost& p, const Source& s, int32_t* skipped) {
  OSEQ_LAUNCH((norms_kernel<G, MUON>), dim3(t.nchunks), dim3(256), 0, st, t, s);
  const double times = p.first_scale;
  if (t.nchunks <= FEW_CHUNKS) {
    OSEQ_LAUNCH((planes_kernel<G, MUON, true>), dim3(t.nchunks), dim3(256), 0, st, t, s, skipped, p.eps, times);
  } else {
    OSEQ_LAUNCH(scales_kernel, dim3(t.nmat), dim3(256), 0, st, t, p.eps, times);
    OSEQ_LAUNCH((planes_kernel<G, MUON, false>), dim3(t.nchunks), dim3(256), 0, st, t, s, skipped, p.eps, times);
  }
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
  const int kind = !r.muon && r.o_precision == OPTORCH_BF16 ? OUT_BF16 : OUT_OTHER;
  const std::vector<OrthoLaunch>& launches = p.launches[kind];
  for (size_t i = 0; i < launches.size(); ++i) {
    const OrthoLaunch& c = launches[i];
    if (c.kind == OL_GRAM) {
      const OrthoWork* w = works + p.gram.work0;
      if (p.gram.w == 128) run(gram_kernel<128>, p.gram.n, lds_of<128>(), st, t, w, c.src, c.op[0]);
      else if (p.gram.w == 64) run(gram_kernel<64>, p.gram.n, lds_of<64>(), st, t, w, c.src, c.op[0]);
      else run(gram_kernel<32>, p.gram.n, lds_of<32>(), st, t, w, c.src, c.op[0]);
      join(p.gram, c);
    } else if (c.kind == OL_CHAIN && p.most_m <= ORTHO_SMALL) {
      OrthoOps ops = {};
      for (; launches[i].kind == OL_CHAIN; ++i)  // (an apply follows)
        for (int k = 0; k < launches[i].ops; ++k) ops.op[ops.n++] = launches[i].op[k];
      --i;
      run_small(st, t, p.most_m, ops);
    } else if (c.kind == OL_CHAIN) {
      const OrthoList& l = p.chain;
      const OrthoWork* w = works + l.work0;
      if (l.w == 128) run(chain_kernel<128>, l.n * c.ops, lds_of<128>(), st, t, w, l.n, l.slots, c.op[0], c.op[1]);
      else if (l.w == 64) run(chain_kernel<64>, l.n * c.ops, lds_of<64>(), st, t, w, l.n, l.slots, c.op[0], c.op[1]);
      else run(chain_kernel<32>, l.n * c.ops, lds_of<32>(), st, t, w, l.n, l.slots, c.op[0], c.op[1]);
      join(l, c);
    } else {
      const OrthoList& l = c.last ? p.last[r.muon] : p.apply;
      const OrthoWork* w = works + l.work0;
      if (!c.last) run_apply<TO_PLANES>(st, t, l, w, c, o);
      else if (r.muon) run_apply<3>(st, t, l, w, c, o);
      else if (r.o_precision == OPTORCH_FP32) run_apply<OPTORCH_FP32>(st, t, l, w, c, o);
      else if (r.o_precision == OPTORCH_BF16) run_apply<OPTORCH_BF16>(st, t, l, w, c, o);
      else run_apply<OPTORCH_FP16>(st, t, l, w, c, o);
    }
  }
}

}  // namespace oseq
