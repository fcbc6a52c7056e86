// The two products of the gradient of a loss over many classes, for a piece of the classes:
//   dx += ds w (summed in fp32 over the pieces, then times each row's factor),   dw = ds^T x' times one factor,
// with x' the rows of x times their powers of two.  ds is read along the reduction for dx and across it for dw (mat_core.h).  In 16 bits it has
// two planes: each product is made with the second one first and then with the first (TWICE); of few rows the second plane is rows behind
// the first one's (copies), so that the weights are read once.
#include "mat_layout.h"
#include "parts.h"

namespace oseq {

namespace {

struct Grad {
  const void* a; int lda;
  int64_t second;     // from a to its second plane, or 0
  const void* b; int ldb;
  int64_t M;
  int N, K;
  int tiles_m, tiles_n, parts;
  int copies;         // rows of the result that are added up, M / copies apart
  Parts cut;          // of K, in `parts`
  float* partial;     // with more than one of either: [parts][M][up8(N)] sums
  float* acc;         // dx: [M][up8(N)], the sums of the pieces before this one, unless `start`; the sums with it, unless `end`
  bool start, end;
  const float4* info; // dx: the rows' factors
  const float* scale; // dw: the factor
  float unscale;      // and what either is multiplied by besides
  void* out; int64_t ldo;
};

struct Before { float v[8]; };
// the sums of the pieces before this one
template <bool DW> __device__ __forceinline__ Before before_of(const Grad& g, int64_t row, int col) {
  Before b = {};
  if (!DW && !g.start) load_f32<float, 8>(g.acc + row * ((g.N + 7) & ~7) + col, b.v);
  return b;
}
// what becomes of eight neighbouring sums, n of them inside
template <class O, bool DW> __device__ __forceinline__ void finish(const Grad& g, int64_t row, int col, float (&v)[8], int n, const Before& before) {
  if (!DW && !g.start) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += before.v[e];
  }
  if (!DW && !g.end) {
    store_f32<float, 8>(g.acc + row * ((g.N + 7) & ~7) + col, v);
    return;
  }
  const float4 known = DW ? make_float4(0.f, 0.f, 1.f, *g.scale) : g.info[row];
  const float f = known.w * g.unscale;
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = known.z == 0.f ? 0.f : v[e] * f;  // (a row that is left out: weights that are not finite say nothing of it)
  O* out = (O*)g.out + row * g.ldo + col;
  if (n == 8) {
    store8<O>(out, 8, v);
  } else {
    store8<O>(out, n, v);
    asm volatile("");  // (or the two ways share their last stores, and the other one is no longer of 16 bytes)
  }
}

// One block's tile of a product.  O: type of the result; T: of the planes; TWICE: ds has a second plane
template <class O, class T, int W, bool DW, bool TWICE>
__device__ __forceinline__ void tile(const Grad& a, uint32_t block, unsigned char* smem) {
  constexpr int PL = sizeof(O) == 4 ? 3 : 1;
  constexpr bool PLANES = PL > 1 || TWICE;
  typedef Tile<T, PL, W, DW, true, TWICE> G;
  // neighbouring tiles on one XCD: each of the eight takes a run of them, eight rows of tiles at a time
  const int total = a.tiles_m * a.tiles_n * a.parts;
  const int per = (total + 7) / 8, id = (block & 7) * per + (block >> 3);
  if ((int)(block >> 3) >= per || id >= total) return;
  const int tiles = a.tiles_m * a.tiles_n, part = id / tiles, t = id - part * tiles;
  const int band = t / (8 * a.tiles_n), rows_in = min(8, a.tiles_m - band * 8), u = t - band * 8 * a.tiles_n;
  const int tn = u / rows_in, tm = band * 8 + u - tn * rows_in;
  const int64_t m0 = (int64_t)tm * G::EDGE;
  const int n0 = tn * G::EDGE;
  const int rows = (int)min<int64_t>(G::EDGE, a.M - m0), cols = min(G::EDGE, a.N - n0);
  const int k0 = a.cut.first(part), k1 = a.cut.end(part);
  const Operand<T> first = {(const T*)a.a + (DW ? (int64_t)k0 * a.lda + place_of<PL>(m0) : m0 * a.lda + place_of<PL>(k0)), a.lda, rows};
  Operand<T> oa = first;
  if (TWICE) { oa.base += a.second; oa.second = -a.second; }  // (what rounding left of the first plane, then that)
  const Operand<T> ob = {(const T*)a.b + (int64_t)k0 * a.ldb + place_of<PL>(n0), a.ldb, cols};
  const int n8 = (a.N + 7) & ~7;
  auto ask = [&](int r, int c, int) { return a.parts * a.copies > 1 ? Before{} : before_of<DW>(a, m0 + r, n0 + c); };
  auto emit = [&](int r, int c, float (&v)[8], int n, const Before& before) {
    if (a.parts * a.copies > 1) store_f32<float, 8>(a.partial + ((int64_t)part * a.M + m0 + r) * n8 + n0 + c, v);
    else finish<O, DW>(a, m0 + r, n0 + c, v, n, before);
  };
  typename G::Acc acc;
  uint32_t wait = 0;  // planes: which groups have a sum that is not finite
  G::product(smem, oa, ob, k1 - k0, acc);
  G::template out<false, false>(smem, acc, rows, cols, ask, [&](int idx, int r, int c, float (&v)[8], int n, const Before& before) {
    if (PLANES) {
      bool bad = false;
#pragma unroll
      for (int e = 0; e < 8; ++e) bad |= e < n && !finite(v[e]);
      if (bad) { wait |= 1u << idx; return; }
    }
    emit(r, c, v, n, before);
  });
  if constexpr (PLANES) {
    // what the first planes alone say of such sums, and the others of their groups once more (as the layers' products do)
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
      classes.apply(idx, v);
      emit(r, c, v, n, ask(r, c, n));
    });
  }
}

template <class O, class T, int W, bool DW, bool TWICE>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(W == 128 ? 1 : 2, W == 128 ? 1 : 8))) grad_kernel(Grad a) {
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  tile<O, T, W, DW, TWICE>(a, blockIdx.y * gridDim.x + blockIdx.x, smem);
}

// the parts' sums and the copies', added in order: block `block` of `blocks`
template <class O, class T, bool DW> __device__ __forceinline__ void join_parts(const Grad& a, int block, int blocks) {
  const int c8 = (a.N + 7) / 8;
  const int64_t n = a.M / a.copies * c8;
  for (int64_t i = (int64_t)block * 256 + threadIdx.x; i < n; i += (int64_t)blocks * 256) {
    const int64_t r = i / c8;
    const int c = (int)(i - r * c8) * 8;
    const Before before = before_of<DW>(a, r, c);
    float v[8];
    load_f32<float, 8>(a.partial + i * 8, v);
    for (int p = 1; p < a.parts * a.copies; ++p) {
      const float f = a.copies > 1 && p % 2 ? Tile<T, sizeof(O) == 4 ? 3 : 1, 32, DW, true>::BETWEEN : 1.f;  // (the second plane)
      float t[8];
      load_f32<float, 8>(a.partial + ((int64_t)p * n + i) * 8, t);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = __fmaf_rn(t[e], f, v[e]);
    }
    finish<O, DW>(a, r, c, v, min(8, a.N - c), before);
  }
}
template <class O, class T, bool DW> __global__ void __launch_bounds__(256) grad_join_kernel(Grad a) { join_parts<O, T, DW>(a, blockIdx.x, gridDim.x); }

// Both products and the sums for dbias in one launch, where neither product fills the card: they read the same ds and nothing of each other.
// 128 x 512 -> 1000 in bf16: 11.5 us of kernels as two launches, 7.6 as one.
struct Both {
  Grad dw, dx;
  uint32_t dw_blocks, dx_blocks;   // of the products; then those of dbias
  const float* bias_sums; int bias_rows; float* dbias;
  int dw_joins, dx_joins;          // blocks that add up parts
};
template <class O, class T, int W, bool TWICE>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 8))) both_kernel(Both b) {
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  const uint32_t block = blockIdx.x;
  if (block < b.dw_blocks) tile<O, T, W, true, TWICE>(b.dw, block, smem);
  else if (block < b.dw_blocks + b.dx_blocks) tile<O, T, W, false, TWICE>(b.dx, block - b.dw_blocks, smem);
  else column_sums(b.bias_sums, b.bias_rows, (int)b.dw.M, b.dbias, block - b.dw_blocks - b.dx_blocks, reinterpret_cast<float(*)[17]>(smem));
}
template <class O, class T> __global__ void __launch_bounds__(256) both_join_kernel(Both b) {
  if ((int)blockIdx.x < b.dw_joins) join_parts<O, T, true>(b.dw, blockIdx.x, b.dw_joins);
  else join_parts<O, T, false>(b.dx, blockIdx.x - b.dw_joins, b.dx_joins);
}

template <class O, class T, int W, bool DW, bool TWICE> void run_w(hipStream_t st, Grad& a) {
  typedef Tile<T, sizeof(O) == 4 ? 3 : 1, W, DW, true, TWICE> G;
  a.tiles_m = ceil_div(a.M, 2 * W);
  a.tiles_n = ceil_div(a.N, 2 * W);
  const int per = (a.tiles_m * a.tiles_n * a.parts + 7) / 8;
  auto k = grad_kernel<O, T, W, DW, TWICE>;
  // (more LDS than a launch gets unasked; set again on every launch: which devices know it is not ours to remember)
  if (G::LDS > 65536) (void)hipFuncSetAttribute((const void*)k, hipFuncAttributeMaxDynamicSharedMemorySize, G::LDS);
  OSEQ_LAUNCH(k, grid_of_blocks((int64_t)per * 8), dim3(256), G::LDS, st, a);
  if (a.parts * a.copies > 1) OSEQ_LAUNCH((grad_join_kernel<O, T, DW>), dim3(grid_of(a.M / a.copies * ((a.N + 7) / 8))), dim3(256), 0, st, a);
}
template <class O, class T, bool DW, bool TWICE> void run_as(hipStream_t st, Grad& a, const ProductShape& s) {
  a.cut = parts_of(a.K, s.parts);
  a.parts = a.cut.count;
  if (s.wave == 128) run_w<O, T, 128, DW, TWICE>(st, a);
  else if (s.wave == 64) run_w<O, T, 64, DW, TWICE>(st, a);
  else run_w<O, T, 32, DW, TWICE>(st, a);
}
template <class O, class T, bool DW> void run(hipStream_t st, Grad& a, const ProductShape& s) {
  constexpr bool CAN = sizeof(O) == 2;  // (two planes of ds: 16 bits only)
  if (CAN && a.second) run_as<O, T, DW, CAN>(st, a, s); else run_as<O, T, DW, false>(st, a, s);
}

template <class O, class T, int W, bool TWICE> void run_both_as(hipStream_t st, Both& b) {
  constexpr int PL = sizeof(O) == 4 ? 3 : 1, LDS = Tile<T, PL, W, true, true>::LDS;
  static_assert(LDS == Tile<T, PL, W, false, true>::LDS, "both products' slots are alike");
  auto blocks = [](Grad& g) {
    g.tiles_m = ceil_div(g.M, 2 * W);
    g.tiles_n = ceil_div(g.N, 2 * W);
    return (uint32_t)((g.tiles_m * g.tiles_n * g.parts + 7) / 8 * 8);
  };
  auto joins = [](const Grad& g) { return g.parts * g.copies > 1 ? grid_of(g.M / g.copies * ((g.N + 7) / 8)) : 0; };
  b.dw_blocks = blocks(b.dw);
  b.dx_blocks = blocks(b.dx);
  auto k = both_kernel<O, T, W, TWICE>;
  if (LDS > 65536) (void)hipFuncSetAttribute((const void*)k, hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
  OSEQ_LAUNCH(k, dim3(b.dw_blocks + b.dx_blocks + (b.dbias ? ceil_div(b.dw.M, 16) : 0)), dim3(256), LDS, st, b);
  b.dw_joins = joins(b.dw);
  b.dx_joins = joins(b.dx);
  if (b.dw_joins + b.dx_joins) OSEQ_LAUNCH((both_join_kernel<O, T>), dim3(b.dw_joins + b.dx_joins), dim3(256), 0, st, b);
}

template <class O, class T, int W> void run_both(hipStream_t st, Both& b) {
  constexpr bool CAN = sizeof(O) == 2;
  if (CAN && b.dx.second) run_both_as<O, T, W, CAN>(st, b); else run_both_as<O, T, W, false>(st, b);
}

template <class O, class T> void piece_of(const optorch_softmax_loss_t& a, const LossPiece& p) {
  hipStream_t st = (hipStream_t)a.hip_stream;
  Both b = {};
  Grad g = {};
  g.a = p.ds; g.lda = (int)p.ds_row; g.second = p.second;
  g.info = (const float4*)p.info;
  g.scale = p.scale;
  g.unscale = 1.f / loss_scale_of(a.precision);
  if (a.dx) {
    g.b = p.w; g.ldb = p.ldw;
    g.M = a.rows * p.copies; g.N = a.in_features; g.K = p.count;
    g.copies = p.copies;
    g.partial = p.parts;
    g.acc = p.acc; g.start = p.start; g.end = p.end;
    g.out = a.dx; g.ldo = a.lddx;
    b.dx = g;
    if (!p.both) run<O, T, false>(st, g, p.dx);
  }
  if (a.dw) {
    g.b = p.xs; g.ldb = p.ldxs;
    g.M = p.count; g.N = a.in_features; g.K = (int)(a.rows * p.copies);
    g.copies = 1;
    g.partial = p.both ? p.parts + p.dx_parts : p.parts;
    g.out = (O*)a.dw + p.first * a.lddw; g.ldo = a.lddw;
    b.dw = g;
    if (!p.both) run<O, T, true>(st, g, p.dw);
  }
  if (p.both) {
    for (Grad* q : {&b.dx, &b.dw}) {
      q->cut = parts_of(q->K, q == &b.dx ? p.dx.parts : p.dw.parts);
      q->parts = q->cut.count;
    }
    b.bias_sums = p.bias_sums; b.bias_rows = p.bias_rows; b.dbias = a.dbias ? a.dbias + p.first : nullptr;
    if (p.dx.wave == 64) run_both<O, T, 64>(st, b); else run_both<O, T, 32>(st, b);
  } else if (a.dbias) {
    OSEQ_LAUNCH(dbias_kernel, dim3(ceil_div(p.count, 16)), dim3(256), 0, st, p.bias_sums, p.bias_rows, p.count, a.dbias + p.first);
  }
}

}  // namespace

void launch_loss_piece(const optorch_softmax_loss_t& a, const LossPiece& p) {
  if (a.precision == OPTORCH_FP32) piece_of<float, bf16_t>(a, p);
  else if (a.precision == OPTORCH_BF16) piece_of<bf16_t, bf16_t>(a, p);
  else piece_of<f16_t, f16_t>(a, p);
}

}  // namespace oseq
