// Layer norm over the rows of a matrix and its gradient:
//   y = h weight + bias,  h = (x - mean) rstd;
//   dx = rstd (u - mean(u) - h mean(u h)) + residual,  u = dy weight;  dweight = sum over rows of dy h,  dbias = that of dy.
// Both are bound by memory: a row is read once and stays in the registers of the threads that share it (16 values each) for all of its
// sums.
#include "mat_layout.h"

namespace oseq {

namespace {

// Sums over the G threads of a row (G a power of two; rows of more than a wavefront: `lds` holds two floats a wavefront, a
// place of its own for every other sum)
template <int G> __device__ __forceinline__ void row_sums(float& a, float& b, float* lds) {
#pragma unroll
  for (int o = (G < 64 ? G : 64) / 2; o > 0; o >>= 1) {
    a += __shfl_xor(a, o);
    b += __shfl_xor(b, o);
  }
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
constexpr int CHUNKS = 2;           // groups of eight values that a thread has of a row
constexpr int MOST_LANES = 1024;    // 16384 columns; longer rows are read once for every sum

struct NormForward {
  const void* x; int64_t ldx;
  const float *weight, *bias;
  float eps;
  void* y; int64_t ldy;
  float *mean, *rstd;
  int64_t rows; int cols;
};

__device__ __forceinline__ void vector8(const float* p, int c, int n, float other, float (&v)[8]) {
  if (p) load8<float>(p + c, n, v);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = p ? v[e] : other;
}

// Mean and variance from the deviations from a first mean: the mean that was rounded in its sum is off, and the deviations, which
// are exact, say by how much.
template <class S, int G>
__global__ void __launch_bounds__(threads_of(G)) norm_forward_kernel(NormForward a) {
  constexpr int ROWS = threads_of(G) / G;
  __shared__ float lds[2][2 * 16];
  const int t = threadIdx.x % G;
  const int64_t wanted = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * ROWS + threadIdx.x / G, row = min(wanted, a.rows - 1);
  const S* x = (const S*)a.x + row * a.ldx;
  float v[CHUNKS][8];
  float sum = 0.f, other = 0.f;
#pragma unroll
  for (int j = 0; j < CHUNKS; ++j) {
    const int c = (j * G + t) * 8;
    load8<S>(x + c, min(8, max(0, a.cols - c)), v[j]);
  }
#pragma unroll
  for (int j = 0; j < CHUNKS; ++j)
#pragma unroll
    for (int e = 0; e < 8; ++e) sum += v[j][e];
  row_sums<G>(sum, other, lds[0]);
  const float n = 1.f / (float)a.cols, first = sum * n;
  float square = 0.f;
  sum = 0.f;
#pragma unroll
  for (int j = 0; j < CHUNKS; ++j)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      v[j][e] = (j * G + t) * 8 + e < a.cols ? v[j][e] - first : 0.f;
      sum += v[j][e];
      square = __fmaf_rn(v[j][e], v[j][e], square);
    }
  row_sums<G>(sum, square, lds[1]);
  const float off = sum * n, rstd = 1.f / sqrtf(fmaxf(square * n - off * off, 0.f) + a.eps);
  if (wanted >= a.rows) return;
  if (t == 0 && a.mean) { a.mean[row] = first + off; a.rstd[row] = rstd; }
  S* y = (S*)a.y + row * a.ldy;
#pragma unroll
  for (int j = 0; j < CHUNKS; ++j) {
    const int c = (j * G + t) * 8, k = min(8, a.cols - c);
    if (k <= 0) break;
    float w[8], b[8];
    vector8(a.weight, c, k, 1.f, w);
    vector8(a.bias, c, k, 0.f, b);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[j][e] = __fmaf_rn((v[j][e] - off) * rstd, w[e], b[e]);
    store8<S>(y + c, k, v[j]);
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
    vector8(a.weight, c, k, 1.f, w);
    vector8(a.bias, c, k, 0.f, b);
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

// A block walks its rows; a thread keeps the same columns of all of them, and their sums for dweight and dbias in registers.
template <class S, int G>
__global__ void __launch_bounds__(threads_of(G)) norm_backward_kernel(NormBackward a) {
  constexpr int ROWS = threads_of(G) / G;
  __shared__ float lds[2][2 * 16];
  __shared__ float part[ROWS > 1 ? 2 : 1][ROWS > 1 ? ROWS : 1][ROWS > 1 ? G * 8 * CHUNKS : 1];
  const int t = threadIdx.x % G, r = threadIdx.x / G;
  const bool sums = a.dweight || a.dbias;
  float w[CHUNKS][8], dw[CHUNKS][8], db[CHUNKS][8];
#pragma unroll
  for (int j = 0; j < CHUNKS; ++j) {
    const int c = (j * G + t) * 8;
    vector8(a.weight, c, min(8, max(0, a.cols - c)), 1.f, w[j]);
#pragma unroll
    for (int e = 0; e < 8; ++e) dw[j][e] = db[j][e] = 0.f;
  }
  const float n = 1.f / (float)a.cols;
  int turn = 0;
  for (int64_t first = (int64_t)blockIdx.x * ROWS; first < a.rows; first += (int64_t)gridDim.x * ROWS, turn ^= 1) {
    const int64_t row = min(first + r, a.rows - 1);
    const bool real = first + r < a.rows;
    float h[CHUNKS][8], u[CHUNKS][8], add[CHUNKS][8];
#pragma unroll
    for (int j = 0; j < CHUNKS; ++j) {
      const int c = (j * G + t) * 8, k = min(8, max(0, a.cols - c));
      load8<S>((const S*)a.x + row * a.ldx + c, k, h[j]);
      load8<S>((const S*)a.dy + row * a.lddy + c, k, u[j]);
      if (a.residual && a.dx) load8<S>((const S*)a.residual + row * a.ldr + c, k, add[j]);
    }
    const float mean = a.mean[row], rstd = a.rstd[row];
    float su = 0.f, suh = 0.f;
#pragma unroll
    for (int j = 0; j < CHUNKS; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const bool in = (j * G + t) * 8 + e < a.cols;
        h[j][e] = in ? (h[j][e] - mean) * rstd : 0.f;
        if (real && in) {
          dw[j][e] = __fmaf_rn(u[j][e], h[j][e], dw[j][e]);
          db[j][e] += u[j][e];
        }
        u[j][e] = in ? u[j][e] * w[j][e] : 0.f;
        su += u[j][e];
        suh = __fmaf_rn(u[j][e], h[j][e], suh);
      }
    if (!a.dx) continue;
    row_sums<G>(su, suh, lds[turn]);
    su *= n;
    suh *= n;
    if (!real) continue;
#pragma unroll
    for (int j = 0; j < CHUNKS; ++j) {
      const int c = (j * G + t) * 8, k = min(8, a.cols - c);
      if (k <= 0) break;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        u[j][e] = rstd * (u[j][e] - su - h[j][e] * suh);
        if (a.residual) u[j][e] += add[j][e];
      }
      store8<S>((S*)a.dx + row * a.lddx + c, k, u[j]);
    }
  }
  if (!sums) return;
  float *dweight = a.dweight ? a.dweight + blockIdx.x * a.apart : nullptr, *dbias = a.dbias ? a.dbias + blockIdx.x * a.apart : nullptr;
  if constexpr (ROWS > 1) {
#pragma unroll
    for (int j = 0; j < CHUNKS; ++j)
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
    for (int j = 0; j < CHUNKS; ++j) {
      const int c = (j * G + t) * 8, k = min(8, a.cols - c);
      if (k <= 0) break;
      if (dweight) store8<float>(dweight + c, k, dw[j]);
      if (dbias) store8<float>(dbias + c, k, db[j]);
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
      vector8(a.weight, c, k, 1.f, w);
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
    load8<S>((const S*)a.x + r * a.ldx + c, k, x);
    load8<S>((const S*)a.dy + r * a.lddy + c, k, d);
    const float mean = a.mean[r], rstd = a.rstd[r];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      dw[e] = __fmaf_rn(d[e], (x[e] - mean) * rstd, dw[e]);
      db[e] += d[e];
    }
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

// The blocks' sums, added in a fixed order: sixteen threads a column, dweight's columns before dbias'
__global__ void __launch_bounds__(256) norm_join_kernel(const float* sums, int blocks, int cols, int64_t apart, float* dweight, float* dbias) {
  __shared__ float part[16][17];
  const int cl = threadIdx.x & 15, t = threadIdx.x >> 4;
  const int across = (cols + 15) / 16, which = dweight ? blockIdx.x / across : 1, c = (dweight ? blockIdx.x % across : blockIdx.x) * 16 + cl;
  float s = 0.f;
  if (c < cols) {
    const float* p = sums + (dweight && which ? cols : 0) + c;
    float q[4] = {0.f, 0.f, 0.f, 0.f};  // (four loads on their way)
    int b = t;
    for (; b + 48 < blocks; b += 64) {
#pragma unroll
      for (int e = 0; e < 4; ++e) q[e] += p[(b + 16 * e) * apart];
    }
    for (; b < blocks; b += 16) q[0] += p[b * apart];
    s = (q[0] + q[1]) + (q[2] + q[3]);
  }
  part[t][cl] = s;
  __syncthreads();
  if (t == 0 && c < cols) {
    s = 0.f;
#pragma unroll
    for (int k = 0; k < 16; ++k) s += part[k][cl];
    (which ? dbias : dweight)[c] = s;
  }
}

__global__ void __launch_bounds__(256) norm_clear_kernel(float* a, float* b, int n) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= n) return;
  if (a) a[i] = 0.f;
  if (b) b[i] = 0.f;
}

// threads of a row, 0 where it does not fit
int lanes_of(int cols) {
  int g = 8;
  while (g <= MOST_LANES && g * 8 * CHUNKS < cols) g *= 2;
  return g <= MOST_LANES ? g : 0;
}

template <class S> void forward_of(const optorch_layer_norm_t& a) {
  hipStream_t st = (hipStream_t)a.hip_stream;
  NormForward f = {a.x, a.ldx, a.weight, a.bias, a.eps, a.y, a.ldy, a.mean, a.rstd, a.rows, a.cols};
  auto run = [&](auto g) {
    constexpr int G = g;
    OSEQ_LAUNCH((norm_forward_kernel<S, G>), grid_of_blocks(ceil_div(a.rows, threads_of(G) / G)), dim3(threads_of(G)), 0, st, f);
  };
  switch (lanes_of(a.cols)) {
    case 8: run(std::integral_constant<int, 8>{}); break;
    case 16: run(std::integral_constant<int, 16>{}); break;
    case 32: run(std::integral_constant<int, 32>{}); break;
    case 64: run(std::integral_constant<int, 64>{}); break;
    case 128: run(std::integral_constant<int, 128>{}); break;
    case 256: run(std::integral_constant<int, 256>{}); break;
    case 512: run(std::integral_constant<int, 512>{}); break;
    case 1024: run(std::integral_constant<int, 1024>{}); break;
    default: OSEQ_LAUNCH(norm_forward_long_kernel<S>, grid_of_blocks(a.rows), dim3(1024), 0, st, f);
  }
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
  auto run = [&](auto g) {
    constexpr int G = g;
    OSEQ_LAUNCH((norm_backward_kernel<S, G>), dim3(p.blocks), dim3(threads_of(G)), 0, st, b);
  };
  switch (p.lanes) {
    case 8: run(std::integral_constant<int, 8>{}); break;
    case 16: run(std::integral_constant<int, 16>{}); break;
    case 32: run(std::integral_constant<int, 32>{}); break;
    case 64: run(std::integral_constant<int, 64>{}); break;
    case 128: run(std::integral_constant<int, 128>{}); break;
    case 256: run(std::integral_constant<int, 256>{}); break;
    case 512: run(std::integral_constant<int, 512>{}); break;
    case 1024: run(std::integral_constant<int, 1024>{}); break;
    default:
      if (a.dx) OSEQ_LAUNCH(norm_dx_long_kernel<S>, grid_of_blocks(a.rows), dim3(1024), 0, st, b);
      if (sums) OSEQ_LAUNCH(norm_sums_long_kernel<S>, dim3(ceil_div(a.cols, 256), p.blocks), dim3(256), 0, st, b, (int64_t)ceil_div(a.rows, p.blocks));
  }
  if (join)
    OSEQ_LAUNCH(norm_join_kernel, dim3(ceil_div(a.cols, 16) * each), dim3(256), 0, st, (const float*)ws, p.blocks, (int)a.cols, b.apart, a.dweight, a.dbias);
}

}  // namespace

NormPlan plan_norm_backward(const optorch_layer_norm_t& a) {
  NormPlan p = {};
  p.lanes = lanes_of(a.cols);
  p.rows_at_once = p.lanes ? threads_of(p.lanes) / p.lanes : 1;
  if (p.lanes) p.blocks = (int)std::min<int64_t>((a.rows + p.rows_at_once - 1) / p.rows_at_once, 512);
  else p.blocks = (int)std::max<int64_t>(1, std::min<int64_t>((a.rows + 31) / 32, 2048 / ((a.cols + 255) / 256)));
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
