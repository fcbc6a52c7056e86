// Layer norm over the rows of a matrix and its gradient:
//   y = h weight + bias,  h = (x - mean) rstd;
//   dx = rstd (u - mean(u) - h mean(u h)) + residual,  u = dy weight;  dweight = sum over rows of dy h,  dbias = that of dy.
// Both are bound by memory: a row is read once and stays in the registers of the threads that share it, eight values each, for all of its
// sums; blocks walk the rows, the next one on its way while the sums of this one are made, weight and bias in registers (read for every
// row they are four times a bf16 row: forward 74 us).  16384 x 4096 in bf16: forward 47 us (5.7 TB/s), backward with the skip
// connection's gradient 92 us and 6 to join the blocks' sums (5.5 TB/s); a kernel that only adds three such matrices takes 74 to 95.
#include "mat_layout.h"

namespace oseq {

namespace {

// Two sums over the G threads of a row (G a power of two; rows of more than a wavefront: `lds` holds two floats a wavefront, a
// place of its own for every other call)
template <int G> __device__ __forceinline__ void row_sums(float& a, float& b, float* lds) {
  a = lanes_sum<(G < 64 ? G : 64)>(a);
  b = lanes_sum<(G < 64 ? G : 64)>(b);
  if constexpr (G > 64) {
    constexpr int WAVES = G / 64;
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) { lds[2 * wave] = a; lds[2 * wave + 1] = b; }
    __syncthreads();
    a = b = 0.f;
    const float* p = lds + wave / WAVES * (2 * WAVES);
#pragma unroll
    for (int w = 0; w < WAVES; ++w) { a += p[2 * w]; b += p[2 * w + 1]; }
  }
}

constexpr int threads_of(int lanes) { return lanes < 256 ? 256 : lanes; }

// Eight neighbouring values as they were loaded, n of them inside, zeros beside them.  ONCE: past the caches, 16-bit values.  (As vectors
// of words: as an array of values the loads of 16384 x 4096 took 55 us forward, so 47.)
template <class S> struct Raw { Vec<S, 8> v; };
template <int BYTES> struct Loose16;
template <> struct Loose16<2> { typedef __attribute__((ext_vector_type(4), aligned(2))) uint32_t V; };
template <> struct Loose16<4> { typedef __attribute__((ext_vector_type(4), aligned(4))) uint32_t V; };
template <class S, bool ONCE> __device__ __forceinline__ void ask(const S* p, int n, Raw<S>& r) {
  typedef typename Loose16<sizeof(S)>::V V;
  if (n == 8) {
    V c[sizeof(S) / 2];
#pragma unroll
    for (int i = 0; i < (int)sizeof(S) / 2; ++i) {
      const V* q = reinterpret_cast<const V*>(p) + i;
      c[i] = ONCE ? __builtin_nontemporal_load(q) : *q;
    }
    __builtin_memcpy(&r, c, sizeof(r));
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) r.v.v[e] = e < n ? p[e] : from_f32<S>(0.f);
  }
}
template <class S> __device__ __forceinline__ void take(const Raw<S>& r, float (&v)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = to_f32(r.v.v[e]);
}

struct NormForward {
  const void* x; int64_t ldx;
  const float *weight, *bias;
  float eps;
  void* y; int64_t ldy;
  float *mean, *rstd;
  int64_t rows; int cols;
};

template <int N> __device__ __forceinline__ void vector_of(const float* p, int c, int n, float other, float (&v)[N]) {
  if (p) load8<float>(p + c, n, v);
#pragma unroll
  for (int e = 0; e < N; ++e) v[e] = p ? v[e] : other;
}

// Mean and variance from the deviations from a first mean: the mean that was rounded in its sum is off, and the deviations, which
// are exact, say by how much.  G threads have a row, 8 C values each, in pieces that lie side by side for neighbouring threads; a block walks its rows, weight and bias
// in registers, the next row on its way.
template <class S, int G, int C>
__global__ void __launch_bounds__(threads_of(G)) norm_forward_kernel(NormForward a) {
  constexpr int ROWS = threads_of(G) / G;
  __shared__ float lds[2][2 * 16];
  const int t = threadIdx.x % G, r = threadIdx.x / G;
  float w[C][8], b[C][8];
  int inside[C];
#pragma unroll
  for (int j = 0; j < C; ++j) {
    const int c = (j * G + t) * 8;
    inside[j] = min(8, max(0, a.cols - c));
    vector_of(a.weight, c, inside[j], 1.f, w[j]);
    vector_of(a.bias, c, inside[j], 0.f, b[j]);
  }
  const float n = 1.f / (float)a.cols;
  const bool whole = a.cols == G * C * 8;
  const int64_t step = (int64_t)gridDim.x * ROWS;
  Raw<S> next[C];
  auto fetch = [&](int64_t first) {
    const S* x = (const S*)a.x + min(first + r, a.rows - 1) * a.ldx;
#pragma unroll
    for (int j = 0; j < C; ++j) ask<S, false>(x + (j * G + t) * 8, inside[j], next[j]);
  };
  int64_t first = (int64_t)blockIdx.x * ROWS;
  if (first < a.rows) fetch(first);
  for (; first < a.rows; first += step) {
    float v[C][8];
    float sum = 0.f, square = 0.f;
#pragma unroll
    for (int j = 0; j < C; ++j) {
      take<S>(next[j], v[j]);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum += v[j][e];
    }
    if (first + step < a.rows) fetch(first + step);
    row_sums<G>(sum, square, lds[0]);
    const float mean = sum * n;
    sum = square = 0.f;
#pragma unroll
    for (int j = 0; j < C; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        v[j][e] -= mean;
        if (!whole) v[j][e] = e < inside[j] ? v[j][e] : 0.f;
        sum += v[j][e];
        square = __fmaf_rn(v[j][e], v[j][e], square);
      }
    row_sums<G>(sum, square, lds[1]);
    const float off = sum * n, rstd = 1.f / sqrtf(fmaxf(square * n - off * off, 0.f) + a.eps);
    const int64_t row = first + r;
    if (row >= a.rows) continue;
    if (t == 0 && a.mean) { a.mean[row] = mean + off; a.rstd[row] = rstd; }
#pragma unroll
    for (int j = 0; j < C; ++j) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[j][e] = __fmaf_rn((v[j][e] - off) * rstd, w[j][e], b[j][e]);
      if (inside[j] > 0) store8<S>((S*)a.y + row * a.ldy + (j * G + t) * 8, inside[j], v[j]);
    }
  }
}

// Rows of more than 16384 columns: a block each, which reads it for every sum (the second and third time from the caches)
template <class S>
__global__ void __launch_bounds__(1024) norm_forward_long_kernel(NormForward a) {
  __shared__ float lds[2][2 * 16];
  const int64_t row = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
  if (row >= a.rows) return;
  const S* x = (const S*)a.x + row * a.ldx;
  auto each8 = [&](auto f) {
    for (int c = threadIdx.x * 8; c < a.cols; c += 8192) {
      float v[8];
      load8<S>(x + c, min(8, a.cols - c), v);
      f(c, min(8, a.cols - c), v);
    }
  };
  float sum = 0.f, square = 0.f;
  each8([&](int, int, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) sum += v[e];
  });
  row_sums<1024>(sum, square, lds[0]);
  const float n = 1.f / (float)a.cols, first = sum * n;
  sum = square = 0.f;
  each8([&](int, int k, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float d = e < k ? v[e] - first : 0.f;
      sum += d;
      square = __fmaf_rn(d, d, square);
    }
  });
  row_sums<1024>(sum, square, lds[1]);
  const float off = sum * n, rstd = 1.f / sqrtf(fmaxf(square * n - off * off, 0.f) + a.eps);
  if (threadIdx.x == 0 && a.mean) { a.mean[row] = first + off; a.rstd[row] = rstd; }
  each8([&](int c, int k, float (&v)[8]) {
    float w[8], b[8];
    vector_of(a.weight, c, k, 1.f, w);
    vector_of(a.bias, c, k, 0.f, b);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = __fmaf_rn((v[e] - first - off) * rstd, w[e], b[e]);
    store8<S>((S*)a.y + row * a.ldy + c, k, v);
  });
}

struct NormBackward {
  const void* x; int64_t ldx; const void* dy; int64_t lddy;
  const void* residual; int64_t ldr;
  const float *weight, *mean, *rstd;
  void* dx; int64_t lddx;
  int64_t rows; int cols;
  float *dweight, *dbias;  // [blocks][cols] each, `apart` floats from block to block; or null
  int64_t apart;
};

// A block walks its rows, the next one's values on their way; a thread keeps the same columns of all of them, and their sums for dweight and dbias in
// registers.  dy is zero beside the matrix, so nothing else has to be left out.  Without SUMS it
// makes dx alone.
template <class S, int G, int C, bool SUMS, bool ONCE>
__global__ void __launch_bounds__(threads_of(G)) norm_backward_kernel(NormBackward a) {
  constexpr int ROWS = threads_of(G) / G;
  __shared__ float lds[2][2 * 16];
  __shared__ float part[ROWS > 1 && SUMS ? 2 : 1][ROWS > 1 && SUMS ? ROWS : 1][ROWS > 1 && SUMS ? G * 8 * C : 1];
  const int t = threadIdx.x % G, r = threadIdx.x / G;
  float w[C][8], dw[C][8], db[C][8];
  int inside[C];
#pragma unroll
  for (int j = 0; j < C; ++j) {
    const int c = (j * G + t) * 8;
    inside[j] = min(8, max(0, a.cols - c));
    vector_of(a.weight, c, inside[j], 1.f, w[j]);
#pragma unroll
    for (int e = 0; e < 8; ++e) dw[j][e] = db[j][e] = 0.f;
  }
  const float n = 1.f / (float)a.cols;
  const int64_t step = (int64_t)gridDim.x * ROWS;
  const bool add = a.residual && a.dx, stats = a.dx || a.dweight;
  Raw<S> nx[C] = {}, ny[C], nr[C];
  float mean = 0.f, rstd = 0.f;
  auto fetch = [&](int64_t first) {
    const int64_t row = min(first + r, a.rows - 1);
    const S *x = (const S*)a.x + row * a.ldx, *dy = (const S*)a.dy + row * a.lddy, *res = (const S*)a.residual + row * a.ldr;
#pragma unroll
    for (int j = 0; j < C; ++j) {
      const int c = (j * G + t) * 8;
      if (stats) ask<S, ONCE>(x + c, inside[j], nx[j]);
      ask<S, ONCE>(dy + c, first + r < a.rows ? inside[j] : 0, ny[j]);
      if (add) ask<S, ONCE>(res + c, inside[j], nr[j]);
    }
    if (stats) {
      mean = a.mean[row];
      rstd = a.rstd[row];
    }
  };
  int turn = 0;
  int64_t first = (int64_t)blockIdx.x * ROWS;
  if (first < a.rows) fetch(first);
  for (; first < a.rows; first += step, turn ^= 1) {
    const int64_t row = first + r;
    const bool real = row < a.rows;
    float h[C][8], u[C][8], su = 0.f, suh = 0.f;
    const float rs = rstd;
    Raw<S> res[C];
#pragma unroll
    for (int j = 0; j < C; ++j) {
      take<S>(nx[j], h[j]);
      take<S>(ny[j], u[j]);
      if (add) res[j] = nr[j];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        h[j][e] = (h[j][e] - mean) * rs;
        if (SUMS) {
          dw[j][e] = __fmaf_rn(u[j][e], h[j][e], dw[j][e]);
          db[j][e] += u[j][e];
        }
        u[j][e] *= w[j][e];
        su += u[j][e];
        suh = __fmaf_rn(u[j][e], h[j][e], suh);
      }
    }
    if (first + step < a.rows) fetch(first + step);
    if (!a.dx) continue;
    row_sums<G>(su, suh, lds[turn]);
    su *= n;
    suh *= n;
    if (!real) continue;
#pragma unroll
    for (int j = 0; j < C; ++j) {
      float more[8];
      if (add) take<S>(res[j], more);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        u[j][e] = __fmaf_rn(-h[j][e], suh, u[j][e] - su);
        u[j][e] = add ? __fmaf_rn(rs, u[j][e], more[e]) : rs * u[j][e];
      }
      if (inside[j] > 0) store8<S>((S*)a.dx + row * a.lddx + (j * G + t) * 8, inside[j], u[j]);
    }
  }
  if (!SUMS || (!a.dweight && !a.dbias)) return;
  float *dweight = a.dweight ? a.dweight + blockIdx.x * a.apart : nullptr, *dbias = a.dbias ? a.dbias + blockIdx.x * a.apart : nullptr;
  if constexpr (ROWS > 1 && SUMS) {
#pragma unroll
    for (int j = 0; j < C; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        part[0][r][(j * G + t) * 8 + e] = dw[j][e];
        part[1][r][(j * G + t) * 8 + e] = db[j][e];
      }
    __syncthreads();
    for (int c = threadIdx.x; c < a.cols; c += threads_of(G)) {
      float s = 0.f, b = 0.f;
#pragma unroll
      for (int q = 0; q < ROWS; ++q) { s += part[0][q][c]; b += part[1][q][c]; }
      if (dweight) dweight[c] = s;
      if (dbias) dbias[c] = b;
    }
  } else {
#pragma unroll
    for (int j = 0; j < C; ++j) {
      if (inside[j] <= 0) break;
      if (dweight) store8<float>(dweight + (j * G + t) * 8, inside[j], dw[j]);
      if (dbias) store8<float>(dbias + (j * G + t) * 8, inside[j], db[j]);
    }
  }
}

// Rows of more than 16384 columns: dx as above, a block for each row
template <class S>
__global__ void __launch_bounds__(1024) norm_dx_long_kernel(NormBackward a) {
  __shared__ float lds[2 * 16];
  const int64_t row = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
  if (row >= a.rows) return;
  const float mean = a.mean[row], rstd = a.rstd[row], n = 1.f / (float)a.cols;
  auto each8 = [&](auto f) {
    for (int c = threadIdx.x * 8; c < a.cols; c += 8192) {
      const int k = min(8, a.cols - c);
      float h[8], u[8], w[8];
      load8<S>((const S*)a.x + row * a.ldx + c, k, h);
      load8<S>((const S*)a.dy + row * a.lddy + c, k, u);
      vector_of(a.weight, c, k, 1.f, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        h[e] = e < k ? (h[e] - mean) * rstd : 0.f;
        u[e] = e < k ? u[e] * w[e] : 0.f;
      }
      f(c, k, h, u);
    }
  };
  float su = 0.f, suh = 0.f;
  each8([&](int, int, float (&h)[8], float (&u)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) { su += u[e]; suh = __fmaf_rn(u[e], h[e], suh); }
  });
  row_sums<1024>(su, suh, lds);
  su *= n;
  suh *= n;
  each8([&](int c, int k, float (&h)[8], float (&u)[8]) {
    float add[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (a.residual) load8<S>((const S*)a.residual + row * a.ldr + c, k, add);
#pragma unroll
    for (int e = 0; e < 8; ++e) u[e] = rstd * (u[e] - su - h[e] * suh) + add[e];
    store8<S>((S*)a.dx + row * a.lddx + c, k, u);
  });
}
// ... and the sums of a block's rows for 256 columns: 32 threads take a row's, eight rows at a time
template <class S>
__global__ void __launch_bounds__(256) norm_sums_long_kernel(NormBackward a, int64_t rows_per_block) {
  __shared__ float part[2][8][256 + 8];
  const int cg = threadIdx.x & 31, rl = threadIdx.x >> 5, c = blockIdx.x * 256 + cg * 8, k = min(8, max(0, a.cols - c));
  const int64_t r0 = (int64_t)blockIdx.y * rows_per_block, r1 = min(a.rows, r0 + rows_per_block);
  float dw[8], db[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) dw[e] = db[e] = 0.f;
  for (int64_t r = r0 + rl; r < r1; r += 8) {
    float x[8], d[8];
    load8<S>((const S*)a.dy + r * a.lddy + c, k, d);
    if (a.dweight) {
      load8<S>((const S*)a.x + r * a.ldx + c, k, x);
      const float mean = a.mean[r], rstd = a.rstd[r];
#pragma unroll
      for (int e = 0; e < 8; ++e) dw[e] = __fmaf_rn(d[e], (x[e] - mean) * rstd, dw[e]);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) db[e] += d[e];
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) { part[0][rl][cg * 8 + e] = dw[e]; part[1][rl][cg * 8 + e] = db[e]; }
  __syncthreads();
  const int col = blockIdx.x * 256 + threadIdx.x;
  if (col >= a.cols) return;
  float s = 0.f, b = 0.f;
#pragma unroll
  for (int q = 0; q < 8; ++q) { s += part[0][q][threadIdx.x]; b += part[1][q][threadIdx.x]; }
  if (a.dweight) a.dweight[blockIdx.y * a.apart + col] = s;
  if (a.dbias) a.dbias[blockIdx.y * a.apart + col] = b;
}

// The blocks' sums, added in a fixed order: 32 threads a column, dweight's columns before dbias'
__global__ void __launch_bounds__(1024) norm_join_kernel(const float* sums, int blocks, int cols, int64_t apart, float* dweight, float* dbias) {
  __shared__ float part[32][33];
  const int cl = threadIdx.x & 31, t = threadIdx.x >> 5;
  const int across = (cols + 31) / 32, which = dweight ? blockIdx.x / across : 1, c = (dweight ? blockIdx.x % across : blockIdx.x) * 32 + cl;
  float s = 0.f;
  if (c < cols) {
    const float* p = sums + (dweight && which ? cols : 0) + c;
    float q[4] = {0.f, 0.f, 0.f, 0.f};  // (four loads on their way)
    int b = t;
    for (; b + 96 < blocks; b += 128) {
#pragma unroll
      for (int e = 0; e < 4; ++e) q[e] += p[(b + 32 * e) * apart];
    }
    for (; b < blocks; b += 32) q[0] += p[b * apart];
    s = (q[0] + q[1]) + (q[2] + q[3]);
  }
  part[t][cl] = s;
  __syncthreads();
  if (t == 0 && c < cols) {
    s = 0.f;
#pragma unroll
    for (int k = 0; k < 32; ++k) s += part[k][cl];
    (which ? dbias : dweight)[c] = s;
  }
}

__global__ void __launch_bounds__(256) norm_clear_kernel(float* a, float* b, int n) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= n) return;
  if (a) a[i] = 0.f;
  if (b) b[i] = 0.f;
}

// Blocks of 256 threads (of more threads as many fewer)
constexpr int FORWARD_BLOCKS = 2048, BACKWARD_BLOCKS = 1024;
// Whether a gradient's matrices are read past the caches: where they are larger than the last of those holds (256 MB), which else still has them
// from whatever made them.  bf16, past the caches / through them: 16384 x 4096 91 / 102 us, 8192 x 8192 88 / 103; 65536 x 512 49 / 45, 7003 x 1777 34 / 28.
bool once(const optorch_layer_norm_t& a) { return a.rows * (int64_t)a.cols * 2 * (a.residual ? 4 : 3) > (384ll << 20); }

// The threads of a row, eight values each (or 16 of 1024 threads); 0 where it does not fit
int lanes_of(int cols) {
  int g = 8;
  while (g < 1024 && g * 8 < cols) g *= 2;
  return cols <= 16384 ? g : 0;
}
// f(threads of a row, eights of values that each has)
template <class F> void with_lanes(int cols, F&& f) {
  switch (lanes_of(cols)) {
    case 8: f(std::integral_constant<int, 8>{}, std::integral_constant<int, 1>{}); break;
    case 16: f(std::integral_constant<int, 16>{}, std::integral_constant<int, 1>{}); break;
    case 32: f(std::integral_constant<int, 32>{}, std::integral_constant<int, 1>{}); break;
    case 64: f(std::integral_constant<int, 64>{}, std::integral_constant<int, 1>{}); break;
    case 128: f(std::integral_constant<int, 128>{}, std::integral_constant<int, 1>{}); break;
    case 256: f(std::integral_constant<int, 256>{}, std::integral_constant<int, 1>{}); break;
    case 512: f(std::integral_constant<int, 512>{}, std::integral_constant<int, 1>{}); break;
    default:
      if (cols <= 8192) f(std::integral_constant<int, 1024>{}, std::integral_constant<int, 1>{});
      else f(std::integral_constant<int, 1024>{}, std::integral_constant<int, 2>{});
  }
}

template <class S> void forward_of(const optorch_layer_norm_t& a) {
  hipStream_t st = (hipStream_t)a.hip_stream;
  NormForward f = {a.x, a.ldx, a.weight, a.bias, a.eps, a.y, a.ldy, a.mean, a.rstd, a.rows, a.cols};
  if (!lanes_of(a.cols)) {
    OSEQ_LAUNCH(norm_forward_long_kernel<S>, grid_of_blocks(a.rows), dim3(1024), 0, st, f);
    return;
  }
  with_lanes(a.cols, [&](auto g, auto c) {
    constexpr int G = g, C = c;
    const dim3 grid(std::min(ceil_div(a.rows, threads_of(G) / G), FORWARD_BLOCKS * 256 / threads_of(G))), block(threads_of(G));
    OSEQ_LAUNCH((norm_forward_kernel<S, G, C>), grid, block, 0, st, f);
  });
}

template <class S> void backward_of(const optorch_layer_norm_t& a, const NormPlan& p) {
  hipStream_t st = (hipStream_t)a.hip_stream;
  const bool sums = a.dweight || a.dbias, join = sums && p.blocks > 1;
  float* ws = (float*)a.workspace;
  const int each = (a.dweight ? 1 : 0) + (a.dbias ? 1 : 0);
  NormBackward b = {a.x, a.ldx, a.dy, a.lddy, a.residual, a.ldr, a.weight, a.mean, a.rstd, a.dx, a.lddx, a.rows, a.cols, a.dweight, a.dbias, 0};
  if (join) {
    if (a.dweight) b.dweight = ws;
    if (a.dbias) b.dbias = ws + (a.dweight ? a.cols : 0);
    b.apart = (int64_t)each * a.cols;
  }
  const bool apart = !p.lanes || a.cols > 8192;  // the sums by a kernel of their own
  if (!p.lanes) {
    if (a.dx) OSEQ_LAUNCH(norm_dx_long_kernel<S>, grid_of_blocks(a.rows), dim3(1024), 0, st, b);
  } else if (a.dx || !apart) {
    with_lanes(a.cols, [&](auto g, auto c) {
      constexpr int G = g, C = c;
      const dim3 grid(apart ? (int)std::min<int64_t>(a.rows, 256) : p.blocks), block(threads_of(G));
      if constexpr (sizeof(S) == 2) {
        if (once(a)) {
          OSEQ_LAUNCH((norm_backward_kernel<S, G, C, C == 1, true>), grid, block, 0, st, b);
          return;
        }
      }
      OSEQ_LAUNCH((norm_backward_kernel<S, G, C, C == 1, false>), grid, block, 0, st, b);
    });
  }
  if (apart && sums) OSEQ_LAUNCH(norm_sums_long_kernel<S>, dim3(ceil_div(a.cols, 256), p.blocks), dim3(256), 0, st, b, (int64_t)ceil_div(a.rows, p.blocks));
  if (join)
    OSEQ_LAUNCH(norm_join_kernel, dim3(ceil_div(a.cols, 32) * each), dim3(1024), 0, st, (const float*)ws, p.blocks, (int)a.cols, b.apart, a.dweight, a.dbias);
}

}  // namespace

NormPlan plan_norm_backward(const optorch_layer_norm_t& a) {
  NormPlan p = {};
  p.lanes = lanes_of(a.cols);
  if (p.lanes && a.cols <= 8192) {
    const int threads = threads_of(p.lanes), rows = threads / p.lanes;
    p.blocks = (int)std::min<int64_t>((a.rows + rows - 1) / rows, BACKWARD_BLOCKS * 256 / threads);
  } else {
    p.blocks = (int)std::max<int64_t>(1, std::min<int64_t>((a.rows + 31) / 32, 2048 / ((a.cols + 255) / 256)));
  }
  const int each = (a.dweight ? 1 : 0) + (a.dbias ? 1 : 0);
  p.bytes = p.blocks > 1 && each ? up256((uint64_t)p.blocks * each * a.cols * 4) : 0;
  return p;
}

void launch_norm_forward(const optorch_layer_norm_t& a) {
  if (a.precision == OPTORCH_FP32) forward_of<float>(a);
  else if (a.precision == OPTORCH_BF16) forward_of<bf16_t>(a);
  else forward_of<f16_t>(a);
}

void launch_norm_backward(const optorch_layer_norm_t& a, const NormPlan& p) {
  if (a.rows == 0) {
    if (a.dweight || a.dbias) OSEQ_LAUNCH(norm_clear_kernel, dim3(ceil_div(a.cols, 256)), dim3(256), 0, (hipStream_t)a.hip_stream, a.dweight, a.dbias, (int)a.cols);
    return;
  }
  if (a.precision == OPTORCH_FP32) backward_of<float>(a, p);
  else if (a.precision == OPTORCH_BF16) backward_of<bf16_t>(a, p);
  else backward_of<f16_t>(a, p);
}

}  // namespace oseq
