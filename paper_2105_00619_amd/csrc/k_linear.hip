// Linear layers: y = act(x w^T + bias) + residual with the pre-activation z kept, and their gradients
//   dz = dy * act'(z);   dx = dz w,   dw = dz^T x,   dbias = column sums of dz.
// The three products are one kernel body (mat_core.h) that reads an operand along or across the reduction, so nothing is
// transposed in memory.  fp32 values are three bf16 planes that hold all 24 bits; of the nine products of planes the six whose
// indices add up to at most two count (the others are below 2^-26 of the result).
#include <math.h>

#include "mat_core.h"
#include "matrix.h"

namespace oseq {

namespace {

using namespace mat;

constexpr float INV_SQRT2 = 0.70710678118654752f, INV_SQRT_2PI = 0.39894228040143268f;

template <int ACT> __device__ __forceinline__ float act(float z) {
  if (ACT == OPTORCH_ACT_RELU) return z > 0.f ? z : (z != z ? z : 0.f);
  if (ACT == OPTORCH_ACT_GELU) return 0.5f * z * erfcf(-z * INV_SQRT2);
  if (ACT == OPTORCH_ACT_SILU) return z / (1.f + expf(-z));
  return z;
}

template <int ACT> __device__ __forceinline__ float act_slope(float z) {
  if (ACT == OPTORCH_ACT_RELU) return z > 0.f ? 1.f : 0.f;
  if (ACT == OPTORCH_ACT_GELU) return 0.5f * erfcf(-z * INV_SQRT2) + z * expf(-0.5f * z * z) * INV_SQRT_2PI;
  if (ACT == OPTORCH_ACT_SILU) {
    const float s = 1.f / (1.f + expf(-z));
    return s * (1.f + z * (1.f - s));
  }
  return 1.f;
}

// Eight neighbouring values, n of them inside; `wide`: their addresses are 16-byte aligned whenever n is 8
template <class T> __device__ __forceinline__ void load8(const T* p, int n, bool wide, float (&v)[8]) {
  if (wide && n == 8) {
    load_f32<T, 8>(p, v);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < n ? to_f32(p[e]) : 0.f;
  }
}
template <class T> __device__ __forceinline__ void store8(T* p, int n, bool wide, const float (&v)[8]) {
  if (wide && n == 8) {
    store_f32<T, 8>(p, v);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) p[e] = from_f32<T>(v[e]);
  }
}

// ---- operands laid out anew --------------------------------------------------------------------------------------------
// A value as three bf16 planes: the value rounded, what that leaves, what the two leave.  Where rounding would leave the range of
// bf16 the first plane is cut off instead; a value that is not finite has it in the first plane alone.
__device__ __forceinline__ void planes_of(float x, bf16_t (&p)[3]) {
  p[0] = (bf16_t)x;
  p[1] = p[2] = (bf16_t)0.f;
  if (!(fabsf(x) <= 3.4028235e38f)) return;
  if (!(fabsf((float)p[0]) <= 3.4028235e38f)) p[0] = (bf16_t)copysignf(3.3895314e38f, x);
  x -= (float)p[0];
  p[1] = (bf16_t)x;
  p[2] = (bf16_t)(x - (float)p[1]);
}

// eight neighbouring columns from c on, laid out as the products want them (mat_core.h)
template <int PL, class T> __device__ __forceinline__ void store_planes8(T* row, int c, const float (&v)[8]) {
  T* p = row + place_of<PL>(c);
  if (PL == 1) {
    store_f32<T, 8>(p, v);
  } else {
    Vec<bf16_t, 8> q[3];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      bf16_t t[3];
      planes_of(v[e], t);
#pragma unroll
      for (int k = 0; k < 3; ++k) q[k].v[e] = t[k];
    }
#pragma unroll
    for (int k = 0; k < 3; ++k) *reinterpret_cast<Vec<bf16_t, 8>*>(p + k * 16) = q[k];
  }
}

// S: type in memory; T: type of the planes.  Columns are filled up to whole blocks (block_of) with zeros.
template <class S, class T, int PL>
__global__ void __launch_bounds__(256) pack_kernel(const S* __restrict__ src, int64_t ld, int64_t rows, int cols, bool wide, T* __restrict__ dst) {
  const int c8 = (cols + block_of(PL) - 1) / block_of(PL) * (block_of(PL) / 8);
  const int64_t n = rows * c8;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / c8;
    const int c = (int)(i - r * c8) * 8;
    float v[8];
    load8<S>(src + r * ld + c, min(8, cols - c), wide, v);
    store_planes8<PL, T>(dst + r * c8 * (8 * span_of(PL)), c, v);
  }
}

// dz and the sums of its columns over this block's rows.  Thirty-two threads take a row's 256 columns, eight rows at a time.
struct DzArgs {
  const void* dy; int64_t lddy; const void* z; int64_t ldz;
  int64_t rows; int cols, rows_per_block;
  bool wide_dy, wide_z, write;
  void* dz;       // laid out as the products want it
  float* sums;    // [row blocks][cols], or null
};
template <class S, class T, int PL, int ACT>
__global__ void __launch_bounds__(256) dz_kernel(DzArgs a) {
  __shared__ float part[8][256 + 8];
  const int cg = threadIdx.x & 31, rl = threadIdx.x >> 5, c = blockIdx.x * 256 + cg * 8;
  const int padded = (a.cols + block_of(PL) - 1) / block_of(PL) * block_of(PL);
  const int64_t r0 = (int64_t)blockIdx.y * a.rows_per_block, r1 = min(a.rows, r0 + a.rows_per_block);
  float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  const int n = min(8, a.cols - c);
  if (c < padded)
    for (int64_t r = r0 + rl; r < r1; r += 8) {
      float v[8], z[8];
      load8<S>((const S*)a.dy + r * a.lddy + c, n, a.wide_dy, v);
      if (ACT != OPTORCH_ACT_NONE) {
        load8<S>((const S*)a.z + r * a.ldz + c, n, a.wide_z, z);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= act_slope<ACT>(z[e]);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (e >= n) v[e] = 0.f;
        sum[e] += v[e];
      }
      if (a.write) store_planes8<PL, T>((T*)a.dz + r * padded * span_of(PL), c, v);
    }
  if (!a.sums) return;
#pragma unroll
  for (int e = 0; e < 8; ++e) part[rl][cg * 8 + e] = sum[e];
  __syncthreads();
  const int col = blockIdx.x * 256 + threadIdx.x;
  if (col < a.cols) {
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) s += part[k][threadIdx.x];
    a.sums[(int64_t)blockIdx.y * a.cols + col] = s;
  }
}

// dbias[c] = sum of the row blocks' sums: sixteen threads a column
__global__ void __launch_bounds__(256) dbias_kernel(const float* __restrict__ sums, int blocks, int cols, float* __restrict__ out) {
  __shared__ float part[16][17];
  const int cl = threadIdx.x & 15, t = threadIdx.x >> 4, c = blockIdx.x * 16 + cl;
  float s = 0.f;
  if (c < cols)
    for (int b = t; b < blocks; b += 16) s += sums[(int64_t)b * cols + c];
  part[t][cl] = s;
  __syncthreads();
  if (t == 0 && c < cols) {
    s = 0.f;
#pragma unroll
    for (int k = 0; k < 16; ++k) s += part[k][cl];
    out[c] = s;
  }
}

// ---- the products ------------------------------------------------------------------------------------------------------
struct ProductArgs {
  const void* a; int lda;  // the operands, mat_core.h
  const void* b; int ldb;
  int64_t M;
  int N, K;
  int tiles_m, tiles_n, parts, k_part;
  float* partial;     // parts > 1: [parts][M][up8(N)] sums
  // what becomes of a sum
  const float* bias;
  const void* residual; int64_t ldr;
  void* out; int64_t ldo;   // y, dx or dw
  void* z; int64_t ldz;     // or null
  bool wide_out, wide_z, wide_r;
};

// bias, activation and skip connection of eight neighbouring sums; ACT < 0: the sums alone
template <class O, int ACT>
__device__ __forceinline__ void finish(const ProductArgs& a, int64_t row, int col, float (&v)[8], int n) {
  if (ACT >= 0) {
    if (a.bias) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += e < n ? a.bias[col + e] : 0.f;
    }
    if (a.z) store8<O>((O*)a.z + row * a.ldz + col, n, a.wide_z, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = act<ACT>(v[e]);
    if (a.residual) {
      float r[8];
      load8<O>((const O*)a.residual + row * a.ldr + col, n, a.wide_r, r);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += r[e];
    }
  }
  store8<O>((O*)a.out + row * a.ldo + col, n, a.wide_out, v);
}

// The value at (r, k) of an operand of three planes
template <bool R> __device__ __forceinline__ float value_of(const bf16_t* p, int64_t ld, int64_t r, int64_t k) {
  p += R ? k * ld + place_of<3>(r) : r * ld + place_of<3>(k);
  const float hi = (float)p[0];
  return fabsf(hi) <= 3.4028235e38f ? (hi + (float)p[16]) + (float)p[32] : hi;
}

// An infinity among the operands makes sums of planes NaN (infinity times a plane of zero): such a sum is made again, one product
// after the other, so that infinities and NaNs come out as from fp32 arithmetic
template <bool AR, bool BR>
__device__ __forceinline__ float sum_again(const ProductArgs& a, int64_t m, int n, int k0, int k1) {
  float s = 0.f;
  for (int k = k0; k < k1; ++k)
    s = fmaf(value_of<AR>((const bf16_t*)a.a, a.lda, m, k), value_of<BR>((const bf16_t*)a.b, a.ldb, n, k), s);
  return s;
}

// O: type of the result; T: of the planes
template <class O, class T, int W, bool AR, bool BR, int ACT>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(W == 128 ? 1 : 2, W == 128 ? 1 : 8)))
product_kernel(ProductArgs a) {
  constexpr int PL = sizeof(O) == 4 ? 3 : 1;
  typedef Tile<T, PL, W, AR, BR> G;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  // neighbouring tiles on one XCD: each of the eight takes a run of them, eight rows of tiles at a time
  const int total = a.tiles_m * a.tiles_n * a.parts;
  const int per = (total + 7) / 8, id = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
  if ((int)(blockIdx.x >> 3) >= per || id >= total) return;
  const int tiles = a.tiles_m * a.tiles_n, part = id / tiles, t = id - part * tiles;
  const int band = t / (8 * a.tiles_n), rows_in = min(8, a.tiles_m - band * 8), u = t - band * 8 * a.tiles_n;
  const int tn = u / rows_in, tm = band * 8 + u - tn * rows_in;
  const int64_t m0 = (int64_t)tm * G::EDGE;
  const int n0 = tn * G::EDGE;
  const int rows = (int)min<int64_t>(G::EDGE, a.M - m0), cols = min(G::EDGE, a.N - n0);
  const int k0 = part * a.k_part, k1 = min(a.K, k0 + a.k_part);
  Operand<T> oa, ob;
  oa.base = (const T*)a.a + (AR ? (int64_t)k0 * a.lda + place_of<PL>(m0) : m0 * a.lda + place_of<PL>(k0));
  oa.ld = a.lda; oa.rows = rows;
  ob.base = (const T*)a.b + (BR ? (int64_t)k0 * a.ldb + place_of<PL>(n0) : (int64_t)n0 * a.ldb + place_of<PL>(k0));
  ob.ld = a.ldb; ob.rows = cols;
  typename G::Acc acc;
  G::product(smem, oa, ob, k1 - k0, acc);
  const int n8 = (a.N + 7) & ~7;
  auto emit = [&](int r, int c, float (&v)[8], int n) {
    if (a.parts > 1) store_f32<float, 8>(a.partial + ((int64_t)part * a.M + m0 + r) * n8 + n0 + c, v);
    else finish<O, ACT>(a, m0 + r, n0 + c, v, n);
  };
  uint32_t again = 0;  // fp32: which of this thread's values are to be summed again
  G::out(smem, acc, rows, cols,
         [&](int idx, int r, int c, float (&v)[8], int n) {
           if (sizeof(O) == 4) {
             bool bad = false;
#pragma unroll
             for (int e = 0; e < 8; ++e) bad |= e < n && !(fabsf(v[e]) <= 3.4028235e38f);
             if (bad) { again |= 1u << idx; return; }
           }
           emit(r, c, v, n);
         },
         [](int, int, float (&)[8], int) {}, false);
  if constexpr (sizeof(O) == 4) {
    while (again) {
      const int idx = __builtin_ctz(again);
      again &= again - 1;
      int r, c;
      G::place(idx, r, c);
      const int n = min(8, cols - c);
      float v[8];
      for (int e = 0; e < 8; ++e) v[e] = e < n ? sum_again<AR, BR>(a, m0 + r, n0 + c + e, k0, k1) : 0.f;
      emit(r, c, v, n);
    }
  }
}

// the parts' sums, added in order
template <class O, int ACT>
__global__ void __launch_bounds__(256) join_kernel(ProductArgs a) {
  const int c8 = (a.N + 7) / 8;
  const int64_t n = a.M * c8;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    float v[8];
    load_f32<float, 8>(a.partial + i * 8, v);
    for (int p = 1; p < a.parts; ++p) {
      float t[8];
      load_f32<float, 8>(a.partial + ((int64_t)p * n + i) * 8, t);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += t[e];
    }
    const int64_t r = i / c8;
    const int c = (int)(i - r * c8) * 8;
    finish<O, ACT>(a, r, c, v, min(8, a.N - c));
  }
}

template <class T> __global__ void __launch_bounds__(256) clear_kernel(T* p, int64_t rows, int cols, int64_t ld) {
  const int64_t n = rows * cols;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) p[i / cols * ld + i % cols] = from_f32<T>(0.f);
}

int grid_of(int64_t n) { return (int)std::max<int64_t>(1, std::min<int64_t>((n + 255) / 256, 4096)); }

template <class O, class T, int W, bool AR, bool BR, int ACT> void run_product_w(hipStream_t st, ProductArgs& a) {
  constexpr int PL = sizeof(O) == 4 ? 3 : 1;
  typedef Tile<T, PL, W, AR, BR> G;
  const int per = (a.tiles_m * a.tiles_n * a.parts + 7) / 8;
  auto k = product_kernel<O, T, W, AR, BR, ACT>;
  // (more LDS than a launch gets unasked; set again on every launch: which devices know it is not ours to remember)
  if (G::LDS > 65536) (void)hipFuncSetAttribute((const void*)k, hipFuncAttributeMaxDynamicSharedMemorySize, G::LDS);
  OSEQ_LAUNCH(k, dim3(per * 8), dim3(256), G::LDS, st, a);
  if (a.parts > 1) OSEQ_LAUNCH((join_kernel<O, ACT>), dim3(grid_of(a.M * ((a.N + 7) / 8))), dim3(256), 0, st, a);
}

template <class O, class T, bool AR, bool BR, int ACT> void run_product(hipStream_t st, ProductArgs& a, const ProductShape& s) {
  const int b = 2 * s.wave;
  a.tiles_m = ceil_div(a.M, b); a.tiles_n = ceil_div(a.N, b);
  a.k_part = (int)(((int64_t)ceil_div(a.K, 64) + s.parts - 1) / s.parts) * 64;
  a.parts = ceil_div(a.K, a.k_part);
  if (s.wave == 128) run_product_w<O, T, 128, AR, BR, ACT>(st, a);
  else if (s.wave == 64) run_product_w<O, T, 64, AR, BR, ACT>(st, a);
  else run_product_w<O, T, 32, AR, BR, ACT>(st, a);
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }
// whether groups of eight neighbouring columns of a matrix begin at 16-byte boundaries (fp32: 16 bytes of each half)
bool wide(const void* p, int64_t ld, int esize) { return aligned16(p) && ld * esize % 16 == 0; }
// whether a 16-bit matrix can be an operand as it lies
bool direct(const void* p, int64_t ld, int cols) { return aligned16(p) && ld % 8 == 0 && cols % 8 == 0; }

// Tiles and parts of a product: the largest tiles that still give the 256 CUs work, the reduction cut where even the small ones
// do not.
ProductShape shape_of(int64_t M, int64_t N, int64_t K) {
  auto tiles = [&](int w) { return (int64_t)ceil_div(M, 2 * w) * ceil_div(N, 2 * w); };
  const int64_t steps = (K + 63) / 64;
  if (tiles(128) >= 224) return {128, 1};
  if (tiles(64) >= 224) return {64, 1};
  const int w = tiles(32) > 512 ? 64 : 32;
  const int64_t t = tiles(w);
  int64_t parts = std::min<int64_t>(512 / t, steps / 4);
  parts = std::max<int64_t>(1, std::min<int64_t>(parts, 32));
  return {w, (int)parts};
}

template <class S, class T, int PL>
void pack(hipStream_t st, const void* src, int64_t ld, int64_t rows, int cols, void* dst) {
  OSEQ_LAUNCH((pack_kernel<S, T, PL>), dim3(grid_of(rows * ((cols + 7) / 8))), dim3(256), 0, st, (const S*)src, ld, rows, cols,
              wide(src, ld, sizeof(S)), (T*)dst);
}

template <class S, class T, int PL, int ACT> void run_dz(hipStream_t st, const optorch_linear_t& a, const LinearPlan& p) {
  char* ws = (char*)a.workspace;
  DzArgs d;
  d.dy = a.dy; d.lddy = a.lddy; d.z = a.z; d.ldz = a.ldz;
  d.rows = a.rows; d.cols = a.out_features;
  d.rows_per_block = ceil_div(a.rows, p.sum_blocks);
  d.wide_dy = wide(a.dy, a.lddy, sizeof(S)); d.wide_z = ACT != OPTORCH_ACT_NONE && wide(a.z, a.ldz, sizeof(S));
  d.write = p.make_dz;
  d.dz = ws + p.off_dz;
  d.sums = a.dbias ? (float*)(ws + p.off_sums) : nullptr;
  OSEQ_LAUNCH((dz_kernel<S, T, PL, ACT>), dim3(ceil_div(d.cols, 256), p.sum_blocks), dim3(256), 0, st, d);
  if (a.dbias)
    OSEQ_LAUNCH(dbias_kernel, dim3(ceil_div(d.cols, 16)), dim3(256), 0, st, (const float*)d.sums, p.sum_blocks, d.cols, a.dbias);
}

struct Where { const void* p; int ld; };
// places of a row of n columns laid out anew
template <int PL> int row_of(int n) { return (n + block_of(PL) - 1) / block_of(PL) * block_of(PL) * span_of(PL); }

template <class S, class T, int PL> void forward_of(const optorch_linear_t& a, const LinearPlan& p) {
  hipStream_t st = (hipStream_t)a.hip_stream;
  char* ws = (char*)a.workspace;
  const int row = row_of<PL>(a.in_features);
  Where x{a.x, (int)a.ldx}, w{a.w, (int)a.ldw};
  if (p.pack_x) { pack<S, T, PL>(st, a.x, a.ldx, a.rows, a.in_features, ws + p.off_x); x = {ws + p.off_x, row}; }
  if (p.pack_w) { pack<S, T, PL>(st, a.w, a.ldw, a.out_features, a.in_features, ws + p.off_w); w = {ws + p.off_w, row}; }
  ProductArgs g = {};
  g.a = x.p; g.lda = x.ld;
  g.b = w.p; g.ldb = w.ld;
  g.M = a.rows; g.N = a.out_features; g.K = (int)up8(a.in_features);  // (up to the zeros behind a row)
  g.partial = (float*)(ws + p.off_parts);
  g.bias = a.bias;
  g.residual = a.residual; g.ldr = a.ldr; g.wide_r = a.residual && wide(a.residual, a.ldr, sizeof(S));
  g.out = a.y; g.ldo = a.ldy; g.wide_out = wide(a.y, a.ldy, sizeof(S));
  g.z = a.z; g.ldz = a.ldz; g.wide_z = a.z && wide(a.z, a.ldz, sizeof(S));
  switch (a.activation) {
    case OPTORCH_ACT_NONE: run_product<S, T, false, false, OPTORCH_ACT_NONE>(st, g, p.y); break;
    case OPTORCH_ACT_RELU: run_product<S, T, false, false, OPTORCH_ACT_RELU>(st, g, p.y); break;
    case OPTORCH_ACT_GELU: run_product<S, T, false, false, OPTORCH_ACT_GELU>(st, g, p.y); break;
    default: run_product<S, T, false, false, OPTORCH_ACT_SILU>(st, g, p.y);
  }
}

template <class S, class T, int PL> void backward_of(const optorch_linear_t& a, const LinearPlan& p) {
  hipStream_t st = (hipStream_t)a.hip_stream;
  char* ws = (char*)a.workspace;
  const int row = row_of<PL>(a.in_features);
  if (p.make_dz || a.dbias) switch (a.activation) {
    case OPTORCH_ACT_NONE: run_dz<S, T, PL, OPTORCH_ACT_NONE>(st, a, p); break;
    case OPTORCH_ACT_RELU: run_dz<S, T, PL, OPTORCH_ACT_RELU>(st, a, p); break;
    case OPTORCH_ACT_GELU: run_dz<S, T, PL, OPTORCH_ACT_GELU>(st, a, p); break;
    default: run_dz<S, T, PL, OPTORCH_ACT_SILU>(st, a, p);
  }
  Where dz{a.dy, (int)a.lddy}, x{a.x, (int)a.ldx}, w{a.w, (int)a.ldw};
  if (p.make_dz) dz = {ws + p.off_dz, row_of<PL>(a.out_features)};
  if (p.pack_x) { pack<S, T, PL>(st, a.x, a.ldx, a.rows, a.in_features, ws + p.off_x); x = {ws + p.off_x, row}; }
  if (p.pack_w) { pack<S, T, PL>(st, a.w, a.ldw, a.out_features, a.in_features, ws + p.off_w); w = {ws + p.off_w, row}; }
  ProductArgs g = {};
  g.a = dz.p; g.lda = dz.ld;
  g.partial = (float*)(ws + p.off_parts);
  if (a.dx) {
    g.b = w.p; g.ldb = w.ld;
    g.M = a.rows; g.N = a.in_features; g.K = a.out_features;
    g.out = a.dx; g.ldo = a.lddx; g.wide_out = wide(a.dx, a.lddx, sizeof(S));
    run_product<S, T, false, true, -1>(st, g, p.dx);
  }
  if (a.dw) {
    g.b = x.p; g.ldb = x.ld;
    g.M = a.out_features; g.N = a.in_features; g.K = (int)a.rows;
    g.out = a.dw; g.ldo = a.lddw; g.wide_out = wide(a.dw, a.lddw, sizeof(S));
    run_product<S, T, true, true, -1>(st, g, p.dw);
  }
}

template <class S> void clear(const optorch_linear_t& a) {
  hipStream_t st = (hipStream_t)a.hip_stream;
  if (a.dw) OSEQ_LAUNCH(clear_kernel<S>, dim3(grid_of((int64_t)a.out_features * a.in_features)), dim3(256), 0, st, (S*)a.dw, (int64_t)a.out_features, a.in_features, a.lddw);
  if (a.dbias) OSEQ_LAUNCH(clear_kernel<float>, dim3(grid_of(a.out_features)), dim3(256), 0, st, a.dbias, (int64_t)1, a.out_features, (int64_t)a.out_features);
}

}  // namespace

LinearPlan plan_linear(const optorch_linear_t& a, bool backward) {
  LinearPlan p = {};
  const bool f32 = a.precision == OPTORCH_FP32;
  const uint64_t in_row = 2 * (uint64_t)(f32 ? row_of<3>(a.in_features) : row_of<1>(a.in_features));
  const uint64_t out_row = 2 * (uint64_t)(f32 ? row_of<3>(a.out_features) : row_of<1>(a.out_features));
  const bool need_x = !backward || a.dw, need_w = !backward || a.dx;
  p.pack_x = need_x && (f32 || !direct(a.x, a.ldx, a.in_features));
  p.pack_w = need_w && (f32 || !direct(a.w, a.ldw, a.in_features));
  p.make_dz = backward && (a.dx || a.dw) && (f32 || a.activation != OPTORCH_ACT_NONE || !direct(a.dy, a.lddy, a.out_features));
  uint64_t o = 0;
  auto take = [&](uint64_t n) { const uint64_t at = o; o = up256(o + n); return at; };
  if (p.pack_x) p.off_x = take((uint64_t)a.rows * in_row);
  if (p.pack_w) p.off_w = take((uint64_t)a.out_features * in_row);
  if (p.make_dz) p.off_dz = take((uint64_t)a.rows * out_row);
  uint64_t parts = 0;
  auto product = [&](ProductShape& s, int64_t M, int64_t N, int64_t K) {
    s = shape_of(M, N, K * (f32 ? 6 : 1));
    if (s.parts > 1) parts = std::max(parts, (uint64_t)s.parts * M * up8(N) * 4);
  };
  if (!backward) {
    product(p.y, a.rows, a.out_features, a.in_features);
  } else {
    // row blocks of the dz pass: enough of them for every CU, sums of at least 32 rows each
    const int64_t across = (a.out_features + 255) / 256;
    p.sum_blocks = (int)std::max<int64_t>(1, std::min<int64_t>((a.rows + 31) / 32, std::max<int64_t>(1, 2048 / across)));
    if (a.dbias) p.off_sums = take((uint64_t)p.sum_blocks * a.out_features * 4);
    if (a.dx) product(p.dx, a.rows, a.in_features, a.out_features);
    if (a.dw) product(p.dw, a.out_features, a.in_features, a.rows);
  }
  if (parts) p.off_parts = take(parts);
  p.bytes = o;
  return p;
}

void launch_linear_forward(const optorch_linear_t& a, const LinearPlan& p) {
  if (a.precision == OPTORCH_FP32) forward_of<float, bf16_t, 3>(a, p);
  else if (a.precision == OPTORCH_BF16) forward_of<bf16_t, bf16_t, 1>(a, p);
  else forward_of<f16_t, f16_t, 1>(a, p);
}

void launch_linear_backward(const optorch_linear_t& a, const LinearPlan& p) {
  if (a.rows == 0) {
    if (a.precision == OPTORCH_FP32) clear<float>(a);
    else if (a.precision == OPTORCH_BF16) clear<bf16_t>(a);
    else clear<f16_t>(a);
    return;
  }
  if (a.precision == OPTORCH_FP32) backward_of<float, bf16_t, 3>(a, p);
  else if (a.precision == OPTORCH_BF16) backward_of<bf16_t, bf16_t, 1>(a, p);
  else backward_of<f16_t, f16_t, 1>(a, p);
}

}  // namespace oseq
