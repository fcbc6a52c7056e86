// Linear layers: y = act(x w^T + bias) + residual with the pre-activation z kept, and their gradients
//   dz = dy * act'(z);   dx = dz w,   dw = dz^T x,   dbias = column sums of dz.
// The three products are one kernel body (mat_core.h) that reads an operand along or across the reduction, so nothing is
// transposed in memory.  fp32 values are three bf16 planes that hold all 24 bits; of the nine products of planes the six whose
// indices add up to at most two count (the others are below 2^-26 of the result).
#include <math.h>

#include "mat_layout.h"
#include "matrix.h"
#include "parts.h"

namespace oseq {

namespace {

using namespace mat;

// Phi(z), the normal distribution function, and e = exp(-z^2 / 2), which the density has too:
//   Phi(-x) = e t q(t),  t = 1 / (1 + p x),  x >= 0,
// with q fitted to erfcx(x / sqrt 2) / (2 t) for the least relative error on x = 0 .. 14 (reweighted least squares), so
// that the tail of GELU, where Phi is small, has the same bits as the rest.  FULL (fp32 and all gradients): off by 2e-8, by
// rounding 4e-7 at most and 1e-7 in the mean, x^2 log2(e) / 2 held in two floats as its error is that of e; 16 bits: 4e-6.
// (0.5 (1 + erf) in fp32 is 3e-5 off at z = -3.5.)  Layers of 8192 x 64 -> 8192, whose time is that of their outputs: 65 us
// without an activation, 92 with this in bf16; 125 and 177 in fp32.
template <bool FULL> __device__ __forceinline__ float normal_cdf(float z, float& e) {
  float x = fabsf(z);
  x = x > 32.f ? 32.f : x;  // (where e is 0; a NaN stays one)
  const float d = __fmaf_rn(FULL ? 0.345f : 0.3075f, x, 1.f);
  float t = __builtin_amdgcn_rcpf(d), q;
  const float s = x * x, h = s * -0.72134752f;
  e = __builtin_amdgcn_exp2f(h);
  if (FULL) {
    t = __fmaf_rn(t, __fmaf_rn(-d, t, 1.f), t);
    float l = __fmaf_rn(s, -0.72134752f, -h);
    l = __fmaf_rn(s, -9.62981517e-09f, l);
    l = __fmaf_rn(__fmaf_rn(x, x, -s), -0.72134752f, l);
    e = __fmaf_rn(e, l * 0.69314718f, e);
    q = __fmaf_rn(-0.0283822138f, t, 0.145283043f);
    q = __fmaf_rn(q, t, -0.271174967f);
    q = __fmaf_rn(q, t, 0.187198505f);
    q = __fmaf_rn(q, t, -0.0376027152f);
    q = __fmaf_rn(q, t, 0.111799955f);
    q = __fmaf_rn(q, t, 0.117238209f);
    q = __fmaf_rn(q, t, 0.138020888f);
    q = __fmaf_rn(q, t, 0.137619287f);
  } else {
    q = __fmaf_rn(-0.0755350366f, t, 0.19118157f);
    q = __fmaf_rn(q, t, 0.00591032254f);
    q = __fmaf_rn(q, t, 0.136933118f);
    q = __fmaf_rn(q, t, 0.118578926f);
    q = __fmaf_rn(q, t, 0.122930586f);
  }
  q = q * t * e;  // Phi(-|z|)
  return z < 0.f ? q : 1.f - q;
}
__device__ __forceinline__ float logistic(float z) {
  return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * -1.4426950408889634f));
}

template <int ACT, bool FULL> __device__ __forceinline__ float act(float z) {
  if (ACT == OPTORCH_ACT_RELU) return z > 0.f ? z : (z != z ? z : 0.f);
  if (ACT == OPTORCH_ACT_GELU) { float e; return z * normal_cdf<FULL>(z, e); }
  if (ACT == OPTORCH_ACT_SILU) return z * logistic(z);
  return z;
}

// act'(z) dy, of full precision for any type, since dbias is fp32.  What ReLU masks is 0, infinities and NaNs too.
template <int ACT> __device__ __forceinline__ float act_gradient(float z, float dy) {
  if (ACT == OPTORCH_ACT_RELU) return z > 0.f ? dy : 0.f;
  if (ACT == OPTORCH_ACT_GELU) {
    float e;
    const float c = normal_cdf<true>(z, e);
    return dy * __fmaf_rn(z * 0.39894228040143268f, e, c);
  }
  if (ACT == OPTORCH_ACT_SILU) {
    const float s = logistic(z);
    return dy * (s * (1.f + z * (1.f - s)));
  }
  return dy;
}

// ---- operands laid out anew --------------------------------------------------------------------------------------------
// S: type in memory; T: type of the planes.  Columns are filled up to whole blocks (block_of) with zeros.
struct Pack { const void* src; int64_t ld, rows; int cols; void* dst; int blocks; };
// x and w in one launch, w's blocks behind x's
template <class S, class T, int PL>
__global__ void __launch_bounds__(256) pack_kernel(Pack x, Pack w) {
  const bool second = (int)blockIdx.x >= x.blocks;
  const Pack p = second ? w : x;
  const int c8 = (p.cols + block_of(PL) - 1) / block_of(PL) * (block_of(PL) / 8);
  const int64_t n = p.rows * c8;
  for (int64_t i = (int64_t)(blockIdx.x - (second ? x.blocks : 0)) * 256 + threadIdx.x; i < n; i += (int64_t)p.blocks * 256) {
    const int64_t r = i / c8;
    const int c = (int)(i - r * c8) * 8;
    float v[8];
    load8<S>((const S*)p.src + r * p.ld + c, min(8, p.cols - c), v);
    store_planes8<PL, T>((T*)p.dst + r * c8 * (8 * span_of(PL)), c, v);
  }
}

// A value of dz in two 16-bit planes, the value rounded and what that leaves; one that is not finite has it in the first alone.
//   bf16  v = hi + lo.  Where rounding would leave the range of the type, hi is the largest value.
//   fp16  v = 2 (hi + lo / 2048): a dy near 65504 times a slope of up to 1.13 stays inside the range, and lo is as far above
//         fp16's smallest values as hi is.  (Unscaled, a dz of 1e-4 kept no more bits in two planes than in one.)
template <class T> constexpr float two_planes_scale() { return __is_same(T, f16_t) ? 2.f : 1.f; }
template <class T> __device__ __forceinline__ void two_planes8(const float (&v)[8], Vec<T, 8>& hi, Vec<T, 8>& lo) {
  constexpr float SCALE = two_planes_scale<T>();
  float h[8], l[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) h[e] = v[e] * (1.f / SCALE);
  hi = round_vec<T, 8>(h);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if (__is_same(T, bf16_t) && finite(v[e]) && !finite((float)hi.v[e])) hi.v[e] = from_f32<T>(copysignf(3.3895314e38f, v[e]));
    l[e] = finite(v[e]) ? (h[e] - (float)hi.v[e]) * (__is_same(T, f16_t) ? 2048.f : 1.f) : 0.f;
  }
  lo = round_vec<T, 8>(l);
}

// dz and the sums of its columns over this block's rows.  Thirty-two threads take a row's 256 columns, eight rows at a time.
struct DzArgs {
  const void* dy; int64_t lddy; const void* z; int64_t ldz;
  int64_t rows; int cols, rows_per_block;
  bool write;
  void* dz;       // laid out as the products want it
  int64_t second; // where the second plane is, in values (slopes_of_two)
  float* sums;    // [row blocks][cols], or null
};
// 16 bits: whether dz has more of them than dy
constexpr bool slopes_of_two(int precision, int act) {
  return precision != OPTORCH_FP32 && (act == OPTORCH_ACT_GELU || act == OPTORCH_ACT_SILU);
}
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
      load8<S>((const S*)a.dy + r * a.lddy + c, n, v);
      if (ACT != OPTORCH_ACT_NONE) {
        load8<S>((const S*)a.z + r * a.ldz + c, n, z);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = act_gradient<ACT>(z[e], v[e]);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (e >= n) v[e] = 0.f;
        sum[e] += v[e];
      }
      if (a.write) {
        T* row = (T*)a.dz + r * padded * span_of(PL);
        if constexpr (PL == 1 && slopes_of_two(OPTORCH_BF16, ACT)) {
          Vec<T, 8> hi, lo;
          two_planes8<T>(v, hi, lo);
          *reinterpret_cast<Vec<T, 8>*>(row + c) = hi;
          *reinterpret_cast<Vec<T, 8>*>(row + a.second + c) = lo;
        } else {
          store_planes8<PL, T>(row, c, v);
        }
      }
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

// ---- the products ------------------------------------------------------------------------------------------------------
struct ProductArgs {
  const void* a; int lda;  // the operands, mat_core.h
  int64_t second;          // TWICE: from a to its second plane
  const void* b; int ldb;
  int64_t M;
  int N, K;
  int tiles_m, tiles_n, parts;
  Parts cut;          // of K, in `parts`
  float* partial;     // parts > 1: [parts][M][up8(N)] sums
  // what becomes of a sum
  const float* bias;
  const void* residual; int64_t ldr;
  void* out; int64_t ldo;   // y, dx or dw
  void* z; int64_t ldz;     // or null
};

// the skip connection of neighbouring outputs
template <class O, int V> struct Skip { float v[V]; };
template <class O, int ACT, int V> __device__ __forceinline__ Skip<O, V> skip_of(const ProductArgs& a, int64_t row, int col, int n) {
  Skip<O, V> s = {};
  if (ACT >= 0 && a.residual) load8<O>((const O*)a.residual + row * a.ldr + col, n, s.v);
  return s;
}

template <int ACT, int V> __device__ __forceinline__ void bias_of(const ProductArgs& a, int col, int n, float (&b)[V]) {
#pragma unroll
  for (int e = 0; e < V; ++e) b[e] = ACT >= 0 && a.bias && e < n ? a.bias[col + e] : 0.f;
}

// bias, activation and skip connection of neighbouring sums; ACT < 0: the sums alone
template <class O, int ACT, int V>
__device__ __forceinline__ void finish(const ProductArgs& a, int64_t row, int col, float (&v)[V], int n, const float (&bias)[V], const Skip<O, V>& skip) {
  if (ACT >= 0) {
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] += bias[e];
    if (a.z) store8<O>((O*)a.z + row * a.ldz + col, n, v);
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = act<ACT, sizeof(O) == 4>(v[e]);
    if (a.residual) {
#pragma unroll
      for (int e = 0; e < V; ++e) v[e] += skip.v[e];
    }
  }
  store8<O>((O*)a.out + row * a.ldo + col, n, v);
}

// O: type of the result; T: of the planes
template <class O, class T, int W, bool AR, bool BR, int ACT, bool TWICE>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(W == 128 ? 1 : 2, W == 128 ? 1 : 8)))
product_kernel(ProductArgs a) {
  constexpr int PL = sizeof(O) == 4 ? 3 : 1;
  constexpr bool PLANES = PL > 1 || TWICE;
  typedef Tile<T, PL, W, AR, BR, TWICE> G;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  // neighbouring tiles on one XCD: each of the eight takes a run of them, eight rows of tiles at a time
  const int total = a.tiles_m * a.tiles_n * a.parts;
  const uint32_t block = blockIdx.y * gridDim.x + blockIdx.x;
  const int per = (total + 7) / 8, id = (block & 7) * per + (block >> 3);
  if ((int)(block >> 3) >= per || id >= total) return;
  const int tiles = a.tiles_m * a.tiles_n, part = id / tiles, t = id - part * tiles;
  const int band = t / (8 * a.tiles_n), rows_in = min(8, a.tiles_m - band * 8), u = t - band * 8 * a.tiles_n;
  const int tn = u / rows_in, tm = band * 8 + u - tn * rows_in;
  const int64_t m0 = (int64_t)tm * G::EDGE;
  const int n0 = tn * G::EDGE;
  const int rows = (int)min<int64_t>(G::EDGE, a.M - m0), cols = min(G::EDGE, a.N - n0);
  const int k0 = a.cut.first(part), k1 = a.cut.end(part);
  Operand<T> oa, ob;
  oa.base = (const T*)a.a + (AR ? (int64_t)k0 * a.lda + place_of<PL>(m0) : m0 * a.lda + place_of<PL>(k0));
  oa.ld = a.lda; oa.rows = rows;
  const Operand<T> first = oa;
  if (TWICE) { oa.base += a.second; oa.second = -a.second; }  // (what rounding left of the first plane, then that)
  ob.base = (const T*)a.b + (BR ? (int64_t)k0 * a.ldb + place_of<PL>(n0) : (int64_t)n0 * a.ldb + place_of<PL>(k0));
  ob.ld = a.ldb; ob.rows = cols;
  // A thread's outputs are of the same eight columns throughout.  (With the bias read for every eight outputs, each read
  // waited for, 4096 x 4096 x 4096 took 140 us, without a bias 112.)
  float bias[8];
  int br, bc;
  G::place(0, br, bc);
  if (a.parts == 1) bias_of<ACT>(a, n0 + bc, cols - bc, bias);
  const int n8 = (a.N + 7) & ~7;
  auto ask = [&](int r, int c, int n) { return a.parts > 1 ? Skip<O, 8>{} : skip_of<O, ACT, 8>(a, m0 + r, n0 + c, n); };
  auto emit = [&](int r, int c, float (&v)[8], int n, const Skip<O, 8>& skip) {
    if (a.parts > 1) store_f32<float, 8>(a.partial + ((int64_t)part * a.M + m0 + r) * n8 + n0 + c, v);
    else finish<O, ACT>(a, m0 + r, n0 + c, v, n, bias, skip);
  };
  constexpr bool LONG = ACT >= OPTORCH_ACT_GELU;
  typename G::Acc acc;
  uint32_t wait = 0;  // planes: which groups have a sum that is not finite
  auto scaled = [](float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] *= TWICE ? two_planes_scale<T>() : 1.f;
  };
  G::product(smem, oa, ob, k1 - k0, acc);
  G::template out<false, LONG>(smem, acc, rows, cols, ask, [&](int idx, int r, int c, float (&v)[8], int n, const Skip<O, 8>& skip) {
    scaled(v);
    if (PLANES) {
      bool bad = false;
#pragma unroll
      for (int e = 0; e < 8; ++e) bad |= e < n && !finite(v[e]);
      if (bad) { wait |= 1u << idx; return; }
    }
    emit(r, c, v, n, skip);
  });
  if constexpr (PLANES) {
    // An infinity among the operands makes sums of planes NaN (infinity times a plane of zero).  The groups that wait: the
    // tile is made of the first planes alone, which says what these sums are, and once more for the others of a group.  So
    // a tile that holds any costs three.
    if (!G::any_of(smem, wait != 0)) return;
    __syncthreads();
    Classes<G::GROUPS> classes = {};
    G::template product<true>(smem, first, ob, k1 - k0, acc);
    G::template out<false, false>(smem, acc, rows, cols, [](int, int, int) { return 0; }, [&](int idx, int, int, float (&v)[8], int, int) {
      if (wait >> idx & 1) classes.set(idx, v);
    });
    __syncthreads();  // (the rows on their way out lie where the next slots go)
    G::product(smem, oa, ob, k1 - k0, acc);
    G::template out<false, true>(smem, acc, rows, cols, [](int, int, int) { return 0; }, [&](int idx, int r, int c, float (&v)[8], int n, int) {
      if (!(wait >> idx & 1)) return;
      scaled(v);
      classes.apply(idx, v);
      emit(r, c, v, n, ask(r, c, n));
    });
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
    float bias[8];
    bias_of<ACT>(a, c, a.N - c, bias);
    finish<O, ACT>(a, r, c, v, min(8, a.N - c), bias, skip_of<O, ACT, 8>(a, r, c, min(8, a.N - c)));
  }
}

// ---- few rows ----------------------------------------------------------------------------------------------------------
// Up to 64 samples: the weights are what is read, once, straight into the operands of 16 x 16 MFMAs.  A block has 16
// outputs of all samples, its wavefronts (4 to 16) share the reduction and add up through LDS.  Few outputs: the same with
// the two operands in each other's place.  1 x 4096 -> 16384 in bf16, 134 MB: 27 us (4.9 TB/s, a copy's rate); as tiles of
// 64 x 64 with the reduction in four parts 38.
struct SkinnyArgs {
  ProductArgs p;       // a: x, b: w as they lie in memory; tiles and parts unused
  int k_wave;          // what a wavefront takes of the reduction, a multiple of 32
};

// S: type in memory; T: of the planes; MB: blocks of 16 samples, of a block's 16 outputs.  NARROW: MB blocks of 16 outputs,
// of a block's 16 samples.
template <class S, class T, int MB, Loads L, bool NARROW, int ACT>
__global__ void __launch_bounds__(1024) skinny_kernel(SkinnyArgs g) {
  constexpr int PL = sizeof(S) == 4 ? 3 : 1, U = PL == 3 ? (MB == 4 ? 1 : 2) : L == SINGLE ? 1 : MB == 4 || L == ODD ? 4 : 8;
  typedef typename Op<T>::V V;
  extern __shared__ float red[];  // [wavefront][MB][256]
  const ProductArgs& a = g.p;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  const int64_t first = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 16;
  if (first >= (NARROW ? a.M : (int64_t)a.N)) return;
  const int r16 = lane & 15, kc = (lane >> 4) * 8;
  const int k0 = wave * g.k_wave, k1 = min(a.K, k0 + g.k_wave);
  // one: the operand of which a block has 16 rows (w, NARROW: x), many: the other one
  const S* one = NARROW ? (const S*)a.a + min(first + r16, a.M - 1) * a.lda : (const S*)a.b + min(first + r16, (int64_t)a.N - 1) * a.ldb;
  const S* many[MB];
#pragma unroll
  for (int m = 0; m < MB; ++m)
    many[m] = NARROW ? (const S*)a.b + (int64_t)min(m * 16 + r16, a.N - 1) * a.ldb : (const S*)a.a + min<int64_t>(m * 16 + r16, a.M - 1) * a.lda;
  // fp32: the products of the first planes apart from the others: where they are not finite, they are the sum (Tile::product)
  v4f acc[MB], rest[PL == 3 ? MB : 1];
#pragma unroll
  for (int m = 0; m < MB; ++m) {
    acc[m] = v4f{0.f, 0.f, 0.f, 0.f};
    if constexpr (PL == 3) rest[m] = acc[m];
  }
  for (int k = k0; k < k1; k += 32 * U) {
    Raw8<S> ro[U], rm[U][MB];
#pragma unroll
    for (int u = 0; u < U; ++u) ro[u] = raw8<S, L>(one, k + u * 32 + kc, k1);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int m = 0; m < MB; ++m) rm[u][m] = raw8<S, L>(many[m], k + u * 32 + kc, k1);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      V po[PL], pm[PL];
      planes8<S, T>(ro[u], po);
#pragma unroll
      for (int m = 0; m < MB; ++m) {
        planes8<S, T>(rm[u][m], pm);
#pragma unroll
        for (int i = PL - 1; i >= 0; --i)
#pragma unroll
          for (int j = PL - 1 - i; j >= 0; --j) {
            v4f& sum = i + j ? rest[PL == 3 ? m : 0] : acc[m];
            sum = NARROW ? mma16(pm[i], po[j], sum) : mma16(po[i], pm[j], sum);
          }
      }
    }
  }
#pragma unroll
  for (int m = 0; m < MB; ++m) {
    if constexpr (PL == 3) {
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[m][e] += finite(acc[m][e]) ? rest[m][e] : 0.f;
    }
    *reinterpret_cast<v4f*>(red + ((wave * MB + m) * 64 + lane) * 4) = acc[m];
  }
  __syncthreads();
  // a thread has four neighbouring outputs of a sample
  for (int i = threadIdx.x; i < MB * 64; i += blockDim.x) {
    const int64_t row = (NARROW ? first : (i >> 6) * 16) + (i & 15);
    const int col = (NARROW ? (i >> 6) * 16 : (int)first) + ((i & 63) >> 4) * 4, n = min(4, a.N - col);
    if (row >= a.M || n <= 0) continue;
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    for (int q = 0; q < waves; ++q) {
      const v4f t = *reinterpret_cast<const v4f*>(red + (q * MB * 64 + i) * 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += t[e];
    }
    float bias[4];
    bias_of<ACT>(a, col, n, bias);
    finish<S, ACT>(a, row, col, v, n, bias, skip_of<S, ACT, 4>(a, row, col, n));
  }
}

template <class T> __global__ void __launch_bounds__(256) clear_kernel(T* p, int64_t rows, int cols, int64_t ld) {
  const int64_t n = rows * cols;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) p[i / cols * ld + i % cols] = from_f32<T>(0.f);
}

template <class O, class T, int W, bool AR, bool BR, int ACT, bool TWICE> void run_product_w(hipStream_t st, ProductArgs& a) {
  constexpr int PL = sizeof(O) == 4 ? 3 : 1;
  typedef Tile<T, PL, W, AR, BR, TWICE> G;
  const int per = (a.tiles_m * a.tiles_n * a.parts + 7) / 8;
  auto k = product_kernel<O, T, W, AR, BR, ACT, TWICE>;
  // (more LDS than a launch gets unasked; set again on every launch: which devices know it is not ours to remember)
  if (G::LDS > 65536) (void)hipFuncSetAttribute((const void*)k, hipFuncAttributeMaxDynamicSharedMemorySize, G::LDS);
  OSEQ_LAUNCH(k, grid_of_blocks((int64_t)per * 8), dim3(256), G::LDS, st, a);
  if (a.parts > 1) OSEQ_LAUNCH((join_kernel<O, ACT>), dim3(grid_of(a.M * ((a.N + 7) / 8))), dim3(256), 0, st, a);
}

template <class O, class T, bool AR, bool BR, int ACT, bool TWICE = false> void run_product(hipStream_t st, ProductArgs& a, const ProductShape& s) {
  const int b = 2 * s.wave;
  a.tiles_m = ceil_div(a.M, b); a.tiles_n = ceil_div(a.N, b);
  a.cut = parts_of(a.K, s.parts);
  a.parts = a.cut.count;
  if (s.wave == 128) run_product_w<O, T, 128, AR, BR, ACT, TWICE>(st, a);
  else if (s.wave == 64) run_product_w<O, T, 64, AR, BR, ACT, TWICE>(st, a);
  else run_product_w<O, T, 32, AR, BR, ACT, TWICE>(st, a);
}

template <class S, class T, int PL, int ACT> void run_dz(hipStream_t st, const optorch_linear_t& a, const LinearPlan& p) {
  char* ws = (char*)a.workspace;
  DzArgs d;
  d.dy = a.dy; d.lddy = a.lddy; d.z = a.z; d.ldz = a.ldz;
  d.rows = a.rows; d.cols = a.out_features;
  d.rows_per_block = ceil_div(a.rows, p.sum_blocks);
  d.write = p.make_dz;
  d.dz = ws + p.off_dz;
  d.second = p.dz_second;
  d.sums = a.dbias ? (float*)(ws + p.off_sums) : nullptr;
  OSEQ_LAUNCH((dz_kernel<S, T, PL, ACT>), dim3(ceil_div(d.cols, 256), p.sum_blocks), dim3(256), 0, st, d);
  if (a.dbias)
    OSEQ_LAUNCH(dbias_kernel, dim3(ceil_div(d.cols, 16)), dim3(256), 0, st, (const float*)d.sums, p.sum_blocks, d.cols, a.dbias);
}

constexpr int SKINNY_ROWS = 64, NARROW_ROWS = 512;

template <class S, class T, int MB, Loads L, bool NARROW, int ACT> void run_skinny_of(hipStream_t st, ProductArgs& p) {
  SkinnyArgs g;
  g.p = p;
  // wavefronts of at least 256 values of k each, what they ask for at once; more of them where there are few blocks
  const int blocks = ceil_div(NARROW ? p.M : (int64_t)p.N, 16), most = blocks >= 1024 ? 4 : blocks >= 256 ? 8 : 16;
  int waves = 4;
  while (waves < most && waves * 512 <= p.K) waves *= 2;
  g.k_wave = (ceil_div(p.K, waves) + 31) & ~31;
  OSEQ_LAUNCH((skinny_kernel<S, T, MB, L, NARROW, ACT>), grid_of_blocks(blocks), dim3(waves * 64), (size_t)waves * MB * 1024, st, g);
}
template <class S, class T, Loads L, bool NARROW, int ACT> void run_skinny_by(hipStream_t st, ProductArgs& p) {
  const int64_t rows = NARROW ? p.N : p.M;  // of the operand that every block reads
  if (rows <= 16) run_skinny_of<S, T, 1, L, NARROW, ACT>(st, p);
  else if (rows <= 32) run_skinny_of<S, T, 2, L, NARROW, ACT>(st, p);
  else run_skinny_of<S, T, 4, L, NARROW, ACT>(st, p);
}
template <class S, class T, bool NARROW, int ACT> void run_skinny(hipStream_t st, ProductArgs& p) {
  const bool odd = sizeof(S) == 2 && (p.K % 2 || p.lda % 2 || p.ldb % 2 || (uintptr_t)p.a % 4 || (uintptr_t)p.b % 4);
  if (p.K < 8) return run_skinny_by<S, T, SINGLE, NARROW, ACT>(st, p);
  if constexpr (sizeof(S) == 2) {
    if (odd) return run_skinny_by<S, T, ODD, NARROW, ACT>(st, p);
  }
  run_skinny_by<S, T, WIDE, NARROW, ACT>(st, p);
}

struct Where { const void* p; int ld; };
// x and w as operands: as they lie, or laid out anew
template <class S, class T, int PL> void operands(const optorch_linear_t& a, const LinearPlan& p, Where& x, Where& w) {
  char* ws = (char*)a.workspace;
  const int row = row_of<PL>(a.in_features);
  x = {a.x, (int)a.ldx};
  w = {a.w, (int)a.ldw};
  Pack px = {}, pw = {};
  auto anew = [&](Where& o, Pack& q, const void* src, int64_t ld, int64_t rows, uint64_t off) {
    o = {ws + off, row};
    q = {src, ld, rows, a.in_features, ws + off, grid_of(rows * ((a.in_features + 7) / 8))};
  };
  if (p.pack_x) anew(x, px, a.x, a.ldx, a.rows, p.off_x);
  if (p.pack_w) anew(w, pw, a.w, a.ldw, a.out_features, p.off_w);
  if (px.blocks + pw.blocks) OSEQ_LAUNCH((pack_kernel<S, T, PL>), dim3(px.blocks + pw.blocks), dim3(256), 0, (hipStream_t)a.hip_stream, px, pw);
}

template <class S, class T, int PL> void forward_of(const optorch_linear_t& a, const LinearPlan& p) {
  hipStream_t st = (hipStream_t)a.hip_stream;
  char* ws = (char*)a.workspace;
  Where x, w;
  operands<S, T, PL>(a, p, x, w);
  ProductArgs g = {};
  g.a = x.p; g.lda = x.ld;
  g.b = w.p; g.ldb = w.ld;
  g.M = a.rows; g.N = a.out_features; g.K = (int)up8(a.in_features);  // (up to the zeros behind a row)
  g.partial = (float*)(ws + p.off_parts);
  g.bias = a.bias;
  g.residual = a.residual; g.ldr = a.ldr;
  g.out = a.y; g.ldo = a.ldy;
  g.z = a.z; g.ldz = a.ldz;
  if (p.straight) {
    g.K = a.in_features;
    auto run = [&](auto act) {
      if (a.rows > SKINNY_ROWS) run_skinny<S, T, true, act>(st, g); else run_skinny<S, T, false, act>(st, g);
    };
    switch (a.activation) {
      case OPTORCH_ACT_NONE: run(std::integral_constant<int, OPTORCH_ACT_NONE>{}); break;
      case OPTORCH_ACT_RELU: run(std::integral_constant<int, OPTORCH_ACT_RELU>{}); break;
      case OPTORCH_ACT_GELU: run(std::integral_constant<int, OPTORCH_ACT_GELU>{}); break;
      default: run(std::integral_constant<int, OPTORCH_ACT_SILU>{});
    }
    return;
  }
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
  if (p.make_dz || a.dbias) switch (a.activation) {
    case OPTORCH_ACT_NONE: run_dz<S, T, PL, OPTORCH_ACT_NONE>(st, a, p); break;
    case OPTORCH_ACT_RELU: run_dz<S, T, PL, OPTORCH_ACT_RELU>(st, a, p); break;
    case OPTORCH_ACT_GELU: run_dz<S, T, PL, OPTORCH_ACT_GELU>(st, a, p); break;
    default: run_dz<S, T, PL, OPTORCH_ACT_SILU>(st, a, p);
  }
  Where dz{a.dy, (int)a.lddy}, x, w;
  if (p.make_dz) dz = {ws + p.off_dz, row_of<PL>(a.out_features)};
  operands<S, T, PL>(a, p, x, w);
  ProductArgs g = {};
  g.a = dz.p; g.lda = dz.ld; g.second = p.dz_second;
  g.partial = (float*)(ws + p.off_parts);
  constexpr bool CAN = PL == 1;  // (two planes of dz: 16 bits only)
  if (a.dx) {
    g.b = w.p; g.ldb = w.ld;
    g.M = a.rows; g.N = a.in_features; g.K = a.out_features;
    g.out = a.dx; g.ldo = a.lddx;
    if (CAN && p.dz_second) run_product<S, T, false, true, -1, CAN>(st, g, p.dx);
    else run_product<S, T, false, true, -1>(st, g, p.dx);
  }
  if (a.dw) {
    g.b = x.p; g.ldb = x.ld;
    g.M = a.out_features; g.N = a.in_features; g.K = (int)a.rows;
    g.out = a.dw; g.ldo = a.lddw;
    if (CAN && p.dz_second) run_product<S, T, true, true, -1, CAN>(st, g, p.dw);
    else run_product<S, T, true, true, -1>(st, g, p.dw);
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
  const bool anew_x = f32 || !direct(a.x, a.ldx, a.in_features), anew_w = f32 || !direct(a.w, a.ldw, a.in_features);
  // Few samples, or few outputs and samples that would be laid out anew.  As tiles / straight from memory, in us: fp32 9705
  // x 2688 -> 37 120 / 60; bf16 off its alignment 20000 x 333 -> 10 18 / 8, 4000 x 1001 -> 64 16 / 10, but 40000 x 77 -> 40
  // 12 / 22 and 9705 x 2687 -> 37 33 / 50: in 16 bits by the operations of the second way.
  const double straight = (double)a.rows * std::max(a.in_features, 128) * ((a.out_features + 15) & ~15);
  p.straight = !backward && (a.rows <= SKINNY_ROWS || (a.rows >= NARROW_ROWS && a.out_features <= SKINNY_ROWS && anew_x && (f32 || straight < 3e8)));
  const bool need_x = backward ? a.dw != nullptr : !p.straight, need_w = backward ? a.dx != nullptr : !p.straight;
  p.pack_x = need_x && anew_x;
  p.pack_w = need_w && anew_w;
  p.make_dz = backward && (a.dx || a.dw) && (f32 || a.activation != OPTORCH_ACT_NONE || !direct(a.dy, a.lddy, a.out_features));
  uint64_t o = 0;
  auto take = [&](uint64_t n) { const uint64_t at = o; o = up256(o + n); return at; };
  if (p.pack_x) p.off_x = take((uint64_t)a.rows * in_row);
  if (p.pack_w) p.off_w = take((uint64_t)a.out_features * in_row);
  // dz of 16-bit layers: rounded once it adds as much as the results' own rounding (dx and dw in bf16 2.3e-3 off, so
  // 1.7e-3), and in fp16 a large dy times a slope above 1 is infinite.  So it has two planes, and the products twice as
  // much to do (8192 x 2048 -> 8192 in bf16: 508 us with one, so 975).  ReLU and no activation leave the bits of dy.
  const bool two = p.make_dz && slopes_of_two(a.precision, a.activation);
  if (p.make_dz) p.off_dz = take((uint64_t)a.rows * out_row * (two ? 2 : 1));
  if (two) p.dz_second = (int64_t)a.rows * (int64_t)(out_row / 2);
  uint64_t parts = 0;
  auto product = [&](ProductShape& s, int64_t M, int64_t N, int64_t K) {
    s = shape_of(M, N, K, f32);
    if (s.parts > 1) parts = std::max(parts, (uint64_t)s.parts * M * up8(N) * 4);
  };
  if (p.straight) {
    // (no workspace)
  } else if (!backward) {
    product(p.y, a.rows, a.out_features, a.in_features);
  } else {
    // row blocks of the dz pass: four blocks for every CU, sums of at least 32 rows each
    const int64_t across = (a.out_features + 255) / 256;
    p.sum_blocks = (int)std::max<int64_t>(1, std::min<int64_t>((a.rows + 31) / 32, std::max<int64_t>(1, 1024 / across)));
    if (a.dbias) p.off_sums = take((uint64_t)p.sum_blocks * a.out_features * 4);
    if (a.dx) product(p.dx, a.rows, a.in_features, (int64_t)a.out_features * (two ? 2 : 1));
    if (a.dw) product(p.dw, a.out_features, a.in_features, a.rows * (two ? 2 : 1));
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
