// Layer norm over the rows of a matrix and its gradient:
//   y = h weight + bias,  h = (x - mean) rstd;
//   dx = rstd (u - mean(u) - h mean(u h)) + residual,  u = dy weight;  dweight = sum over rows of dy h,  dbias = that of dy.
// Both are bound by memory: a row is read once and stays in the registers of the threads that share it, eight values each, for all of its
// sums; blocks walk the rows, the next one on its way while the sums of this one are made, weight and bias in registers (read for every
// row they are four times a bf16 row: forward 74 us).  16384 x 4096 in bf16: forward 45 us (5.9 TB/s), backward with the skip
// connection's gradient 89 us and 4 to join the blocks' sums (5.7 TB/s); a kernel that only adds three such matrices takes 74 to 95.
#include "mat_layout.h"

namespace oseq {

namespace {

// Two sums over the threads of a row: G lanes (a power of two up to 64), or with G = 0 the whole block of up to MAX threads.  `lds` holds two
// floats a wavefront, a place of its own for every other call, zeros for wavefronts that the block does not have (row_sums_begin): all are
// read at once, where a loop over those that there are waits for each (15249 x 2304 in bf16 backward 72 us, so 60).
template <int MAX> struct RowSums { float2 part[2][MAX / 64]; };
template <int G, int MAX> __device__ __forceinline__ void row_sums_begin(RowSums<MAX>& lds) {
  const int i = threadIdx.x % (MAX / 64), waves = blockDim.x >> 6;
  if (G == 0 && threadIdx.x < 2 * (MAX / 64) && i >= waves) lds.part[threadIdx.x / (MAX / 64)][i] = make_float2(0.f, 0.f);
}
template <int G, int MAX> __device__ __forceinline__ void row_sums(float& a, float& b, RowSums<MAX>& lds, int turn) {
  a = lanes_sum<(G ? G : 64)>(a);
  b = lanes_sum<(G ? G : 64)>(b);
  if constexpr (G == 0) {
    if ((threadIdx.x & 63) == 0) lds.part[turn][threadIdx.x >> 6] = make_float2(a, b);
    // (not __syncthreads, which waits for the next row's loads and the last one's stores)
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    a = b = 0.f;
#pragma unroll
    for (int w = 0; w < MAX / 64; ++w) {
      const float2 t = lds.part[turn][w];
      a += t.x;
      b += t.y;
    }
  }
}

// A thread's eight neighbouring values of a row of `cols`: from column `at` on, the first `skip` of them another thread's (the last threads have
// the row's last eight; all eight skipped: nothing of the row).  So no load depends on a branch: one that does waits for the loads before it, and
// rows that do not end with a wavefront took half as long again (15249 x 2304 backward 103 us, 2560 columns 74).
struct Piece { int at, skip; };
__device__ __forceinline__ Piece piece_of(int column, int cols) {
  const int at = max(0, min(column, cols - 8));
  return {at, min(8, column - at)};
}
// ... as they were loaded; rows of fewer than eight values end with zeros.  ONCE: past the caches, 16-bit values.  (As vectors of words: as an
// array of values the loads of 16384 x 4096 took 55 us forward, so 47.)
template <class S> struct Raw { Vec<S, 8> v; };
template <int BYTES> struct Loose16;
template <> struct Loose16<2> { typedef __attribute__((ext_vector_type(4), aligned(2))) uint32_t V; };
template <> struct Loose16<4> { typedef __attribute__((ext_vector_type(4), aligned(4))) uint32_t V; };
// SHORT: there may be fewer than eight columns.
template <class S, bool ONCE, bool SHORT> __device__ __forceinline__ void ask(const S* row, const Piece& p, int cols, Raw<S>& r) {
  typedef typename Loose16<sizeof(S)>::V V;
  if (!SHORT || cols >= 8) {
    V c[sizeof(S) / 2];
#pragma unroll
    for (int i = 0; i < (int)sizeof(S) / 2; ++i) {
      const V* q = reinterpret_cast<const V*>(row + p.at) + i;
      c[i] = ONCE ? __builtin_nontemporal_load(q) : *q;
    }
    __builtin_memcpy(&r, c, sizeof(r));
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) r.v.v[e] = e < cols ? row[e] : from_f32<S>(0.f);
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

// Whether any thread of the wavefront has less than eight values of its own; the others' wavefronts need no selects (as many as half of what
// else a forward pass has to do)
__device__ __forceinline__ bool any_cut(bool cut) { return __ballot(cut) != 0; }
// what is not the thread's own, or not there: zero
__device__ __forceinline__ void own(const Piece& p, int cols, float (&v)[8]) {
  asm volatile("");  // (a branch, not selects)
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = e >= p.skip && e < cols ? v[e] : 0.f;
}
template <bool SHORT, class T> __device__ __forceinline__ void put(T* row, const Piece& p, int cols, const float (&v)[8]) {
  if (p.skip == 0 && (!SHORT || cols >= 8)) {
    store8<T>(row + p.at, 8, v);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e >= p.skip && e < cols) row[p.at + e] = from_f32<T>(v[e]);
    asm volatile("");  // (or the two ways share their last stores, and the other one is no longer of 16 bytes)
  }
}

// (a NaN stays one, which fmaxf makes a zero of: rstd of a row that is not finite)
__device__ __forceinline__ float not_below_zero(float v) { return v < 0.f ? 0.f : v; }

template <int N> __device__ __forceinline__ void vector_of(const float* p, int c, int n, float other, float (&v)[N]) {
  if (p) load8<float>(p + c, n, v);
#pragma unroll
  for (int e = 0; e < N; ++e) v[e] = p ? v[e] : other;
}

// Mean and variance from the deviations from a first mean: the mean that was rounded in its sum is off, and the deviations, which
// are exact, say by how much.  G threads have a row (0: a block of up to MAX threads), 8 C values each, in pieces that lie side by side for
// neighbouring threads; a block walks its rows, weight and bias
// in registers, the next row on its way.
template <class S, int G, int MAX, int C>
__global__ void __launch_bounds__(MAX) norm_forward_kernel(NormForward a) {
  constexpr int ROWS = G ? MAX / G : 1;
  __shared__ RowSums<MAX> lds;
  row_sums_begin<G, MAX>(lds);
  const int lanes = G ? G : blockDim.x, t = G ? threadIdx.x % lanes : threadIdx.x, r = G ? threadIdx.x / lanes : 0;
  float w[C][8], b[C][8];
  Piece piece[C];
#pragma unroll
  for (int j = 0; j < C; ++j) {
    piece[j] = piece_of((j * lanes + t) * 8, a.cols);
    vector_of(a.weight, piece[j].at, min(8, a.cols), 1.f, w[j]);
    vector_of(a.bias, piece[j].at, min(8, a.cols), 0.f, b[j]);
  }
  const float n = 1.f / (float)a.cols;
  bool cut = a.cols < 8;
#pragma unroll
  for (int j = 0; j < C; ++j) cut |= piece[j].skip > 0;
  cut = any_cut(cut);
  const int64_t step = (int64_t)gridDim.x * ROWS;
  Raw<S> next[C];
  auto fetch = [&](int64_t first) {
    const S* x = (const S*)a.x + min(first + r, a.rows - 1) * a.ldx;
#pragma unroll
    for (int j = 0; j < C; ++j) ask<S, false, G == 8>(x, piece[j], a.cols, next[j]);
  };
  int64_t first = (int64_t)blockIdx.x * ROWS;
  if (first < a.rows) fetch(first);
  for (; first < a.rows; first += step) {
    float v[C][8];
    float sum = 0.f, square = 0.f;
#pragma unroll
    for (int j = 0; j < C; ++j) {
      take<S>(next[j], v[j]);
      if (cut) own(piece[j], a.cols, v[j]);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum += v[j][e];
    }
    if (first + step < a.rows) fetch(first + step);
    asm volatile("" ::: "memory");  // (the loads go out here)
    row_sums<G, MAX>(sum, square, lds, 0);
    const float mean = sum * n;
    sum = square = 0.f;
#pragma unroll
    for (int j = 0; j < C; ++j) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[j][e] -= mean;
      if (cut) own(piece[j], a.cols, v[j]);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        sum += v[j][e];
        square = __fmaf_rn(v[j][e], v[j][e], square);
      }
    }
    row_sums<G, MAX>(sum, square, lds, 1);
    const float off = sum * n, rstd = 1.f / sqrtf(not_below_zero(square * n - off * off) + a.eps);
    const int64_t row = first + r;
    if (row >= a.rows) continue;
    if (t == 0 && a.mean) { a.mean[row] = mean + off; a.rstd[row] = rstd; }
#pragma unroll
    for (int j = 0; j < C; ++j) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[j][e] = __fmaf_rn((v[j][e] - off) * rstd, w[j][e], b[j][e]);
      put<G == 8>((S*)a.y + row * a.ldy, piece[j], a.cols, v[j]);
    }
  }
}

// Rows of more than 16384 columns: a block each, which reads it for every sum (the second and third time from the caches)
template <class S>
__global__ void __launch_bounds__(1024) norm_forward_long_kernel(NormForward a) {
  __shared__ RowSums<1024> lds;
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
  row_sums<0, 1024>(sum, square, lds, 0);
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
  row_sums<0, 1024>(sum, square, lds, 1);
  const float off = sum * n, rstd = 1.f / sqrtf(not_below_zero(square * n - off * off) + a.eps);
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
// registers.  dy is taken for zero where a value is not the thread's own, so nothing else has to be left out.  Without SUMS it
// makes dx alone.
template <class S, int G, int MAX, int C, bool SUMS, bool ONCE>
__global__ void __launch_bounds__(MAX) norm_backward_kernel(NormBackward a) {
  constexpr int ROWS = G ? MAX / G : 1;
  __shared__ RowSums<MAX> lds;
  row_sums_begin<G, MAX>(lds);
  __shared__ float part[ROWS > 1 && SUMS ? 2 : 1][ROWS > 1 && SUMS ? ROWS : 1][ROWS > 1 && SUMS ? G * 8 * C : 1];
  const int lanes = G ? G : blockDim.x, t = G ? threadIdx.x % lanes : threadIdx.x, r = G ? threadIdx.x / lanes : 0;
  float w[C][8], dw[C][8], db[C][8];
  Piece piece[C];
#pragma unroll
  for (int j = 0; j < C; ++j) {
    piece[j] = piece_of((j * lanes + t) * 8, a.cols);
    vector_of(a.weight, piece[j].at, min(8, a.cols), 1.f, w[j]);
#pragma unroll
    for (int e = 0; e < 8; ++e) dw[j][e] = db[j][e] = 0.f;
  }
  const float n = 1.f / (float)a.cols;
  bool cut = a.cols < 8;
#pragma unroll
  for (int j = 0; j < C; ++j) cut |= piece[j].skip > 0;
  cut = any_cut(cut);
  const int64_t step = (int64_t)gridDim.x * ROWS;
  const bool add = a.residual && a.dx, stats = a.dx || a.dweight;
  Raw<S> nx[C] = {}, ny[C], nr[C];
  float mean = 0.f, rstd = 0.f;
  auto fetch = [&](int64_t first) {
    const int64_t row = min(first + r, a.rows - 1);
    const S *x = (const S*)a.x + row * a.ldx, *dy = (const S*)a.dy + row * a.lddy, *res = (const S*)a.residual + row * a.ldr;
#pragma unroll
    for (int j = 0; j < C; ++j) {
      if (stats) ask<S, ONCE, G == 8>(x, piece[j], a.cols, nx[j]);
      ask<S, ONCE, G == 8>(dy, piece[j], a.cols, ny[j]);
      if (add) ask<S, ONCE, G == 8>(res, piece[j], a.cols, nr[j]);
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
    const bool all = !cut && first + ROWS <= a.rows;
    Raw<S> res[C];
#pragma unroll
    for (int j = 0; j < C; ++j) {
      take<S>(nx[j], h[j]);
      take<S>(ny[j], u[j]);
      if (!all) own(real ? piece[j] : Piece{0, 8}, a.cols, u[j]);
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
    asm volatile("" ::: "memory");  // (the loads go out here)
    if (!a.dx) continue;
    row_sums<G, MAX>(su, suh, lds, turn);
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
      put<G == 8>((S*)a.dx + row * a.lddx, piece[j], a.cols, u[j]);
    }
  }
  if (!SUMS || (!a.dweight && !a.dbias)) return;
  float *dweight = a.dweight ? a.dweight + blockIdx.x * a.apart : nullptr, *dbias = a.dbias ? a.dbias + blockIdx.x * a.apart : nullptr;
  if constexpr (ROWS > 1 && SUMS) {
#pragma unroll
    for (int j = 0; j < C; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (e >= piece[j].skip) {
          part[0][r][piece[j].at + e] = dw[j][e];
          part[1][r][piece[j].at + e] = db[j][e];
        }
      }
    __syncthreads();
    for (int c = threadIdx.x; c < a.cols; c += MAX) {
      float s = 0.f, b = 0.f;
#pragma unroll
      for (int q = 0; q < ROWS; ++q) { s += part[0][q][c]; b += part[1][q][c]; }
      if (dweight) dweight[c] = s;
      if (dbias) dbias[c] = b;
    }
  } else {
#pragma unroll
    for (int j = 0; j < C; ++j) {
      if (dweight) put<G == 8>(dweight, piece[j], a.cols, dw[j]);
      if (dbias) put<G == 8>(dbias, piece[j], a.cols, db[j]);
    }
  }
}

// Rows of more than 16384 columns: dx as above, a block for each row
template <class S>
__global__ void __launch_bounds__(1024) norm_dx_long_kernel(NormBackward a) {
  __shared__ RowSums<1024> lds;
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
  row_sums<0, 1024>(su, suh, lds, 0);
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

// Blocks that walk the rows: as many as are on the card together, by their registers 32 wavefronts on a CU forward and 16 backward (a few
// more take as long again: 15249 x 2348 backward in 819 blocks of five wavefronts 154 us).
constexpr int FORWARD_WAVES = 32, BACKWARD_WAVES = 16;
int blocks_of(int threads, int waves) { return 256 * std::max(1, waves / (threads / 64)); }
// Whether a gradient's matrices are read past the caches: where they are larger than the last of those holds (256 MB), which else still has them
// from whatever made them.  bf16, past the caches / through them: 16384 x 4096 91 / 102 us, 8192 x 8192 88 / 103; 65536 x 512 49 / 45, 7003 x 1777 34 / 28.
bool once(const optorch_layer_norm_t& a) { return a.rows * (int64_t)a.cols * 2 * (a.residual ? 4 : 3) > (384ll << 20); }

// The threads of a row: a power of two of lanes up to 64 (512 columns), as many wavefronts as it takes up to 8192 columns, eight values each, or
// 16 of 1024 threads; 0: rows longer than that.  (Powers of two there too: 15249 x 2348 in bf16 backward 114 us, so 60.)
int lanes_of(int cols) {
  if (cols > 16384) return 0;
  if (cols > 8192) return 1024;
  if (cols > 512) return ceil_div(cols, 512) * 64;
  int g = 8;
  while (g * 8 < cols) g *= 2;
  return g;
}
int threads_of(int lanes) { return std::max(lanes, lanes > 64 ? 0 : 256); }
// f(lanes of a row or 0, most threads of a block, eights of values that each has)
template <class F> void with_lanes(int cols, F&& f) {
  const int lanes = lanes_of(cols);
  auto go = [&](auto g, auto most, auto c) { f(g, most, c); };
  typedef std::integral_constant<int, 0> Block;
  typedef std::integral_constant<int, 1> One;
  typedef std::integral_constant<int, 256> T256;
  if (lanes == 8) go(std::integral_constant<int, 8>{}, T256{}, One{});
  else if (lanes == 16) go(std::integral_constant<int, 16>{}, T256{}, One{});
  else if (lanes == 32) go(std::integral_constant<int, 32>{}, T256{}, One{});
  else if (lanes == 64) go(std::integral_constant<int, 64>{}, T256{}, One{});
  else if (lanes <= 256) go(Block{}, T256{}, One{});
  else if (lanes <= 512) go(Block{}, std::integral_constant<int, 512>{}, One{});
  else if (cols <= 8192) go(Block{}, std::integral_constant<int, 1024>{}, One{});
  else go(Block{}, std::integral_constant<int, 1024>{}, std::integral_constant<int, 2>{});
}

template <class S> void forward_of(const optorch_layer_norm_t& a) {
  hipStream_t st = (hipStream_t)a.hip_stream;
  NormForward f = {a.x, a.ldx, a.weight, a.bias, a.eps, a.y, a.ldy, a.mean, a.rstd, a.rows, a.cols};
  if (!lanes_of(a.cols)) {
    OSEQ_LAUNCH(norm_forward_long_kernel<S>, grid_of_blocks(a.rows), dim3(1024), 0, st, f);
    return;
  }
  const int lanes = lanes_of(a.cols), threads = threads_of(lanes);
  const dim3 grid((unsigned)std::min<int64_t>((a.rows + threads / lanes - 1) / (threads / lanes), blocks_of(threads, FORWARD_WAVES))), block(threads);
  with_lanes(a.cols, [&](auto g, auto most, auto c) { OSEQ_LAUNCH((norm_forward_kernel<S, g, most, c>), grid, block, 0, st, f); });
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
    const dim3 grid(apart ? (unsigned)std::min<int64_t>(a.rows, 256) : p.blocks), block(threads_of(p.lanes));
    with_lanes(a.cols, [&](auto g, auto most, auto c) {
      constexpr int G = g, MAX = most, C = c;
      if constexpr (sizeof(S) == 2) {
        if (once(a)) {
          OSEQ_LAUNCH((norm_backward_kernel<S, G, MAX, C, C == 1, true>), grid, block, 0, st, b);
          return;
        }
      }
      OSEQ_LAUNCH((norm_backward_kernel<S, G, MAX, C, C == 1, false>), grid, block, 0, st, b);
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
    p.blocks = (int)std::min<int64_t>((a.rows + rows - 1) / rows, blocks_of(threads, BACKWARD_WAVES));
    if (p.blocks <= 4) p.blocks = 1;  // (four turns of one block: no second launch to join them)
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
