// What the kernels on matrix products share besides the products themselves (mat_core.h): values at any address, values as planes, sums
// that are not finite, and the choice of tiles.
#pragma once
#include <math.h>

#include <algorithm>

#include "mat_core.h"
#include "matrix.h"

namespace oseq {

namespace {

using namespace mat;

// Eight (or four) neighbouring values, n of them inside, at any address (the memory system takes accesses off their
// alignment; value by value 20011 rows of 514 took 34 us, so 20)
template <class T, int V> struct Loose { T v[V]; } __attribute__((packed, aligned(alignof(T))));
template <class T, int V> __device__ __forceinline__ void load8(const T* p, int n, float (&v)[V]) {
  if (n == V) {
    const Loose<T, V> t = *reinterpret_cast<const Loose<T, V>*>(p);
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = to_f32(t.v[e]);
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = e < n ? to_f32(p[e]) : 0.f;
  }
}
template <class T, int V> __device__ __forceinline__ void store8(T* p, int n, const float (&v)[V]) {
  if (n == V) {
    *reinterpret_cast<Loose<T, V>*>(p) = __builtin_bit_cast(Loose<T, V>, round_vec<T, V>(v));
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e)
      if (e < n) p[e] = from_f32<T>(v[e]);
  }
}

__device__ __forceinline__ bool finite(float v) { return fabsf(v) <= 3.4028235e38f; }

// The sum over groups of G neighbouring lanes (G a power of two up to 64), the same bits in each of them: exchanges inside a row of 16 lanes
// and between rows by the vector unit itself (through LDS, as shuffles, a wavefront's sum takes six times as long).
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
template <int CTRL> __device__ __forceinline__ float add_moved(float v) {
  return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, false));
}
template <int G> __device__ __forceinline__ float lanes_sum(float v) {
  if (G >= 2) v = add_moved<0xB1>(v);   // quad_perm 1, 0, 3, 2
  if (G >= 4) v = add_moved<0x4E>(v);   // quad_perm 2, 3, 0, 1
  if (G >= 8) v = add_moved<0x141>(v);  // half a row mirrored
  if (G >= 16) v = add_moved<0x140>(v); // a row mirrored
  if (G >= 32) {
    const u32x2 r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(r.x) + __uint_as_float(r.y);
  }
  if (G >= 64) {
    const u32x2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(r.x) + __uint_as_float(r.y);
  }
  return v;
}

// A value as three bf16 planes: the value rounded, what that leaves, what the two leave.  Where rounding would leave the
// range of bf16 the first two are cut off instead, so that they do not add up to more than the value; a value that is not
// finite has it in the first plane alone.
__device__ __forceinline__ float cut_off(float x) { return __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, x) & 0xffff0000u); }
__device__ __forceinline__ void planes_of(float x, bf16_t (&p)[3]) {
  p[0] = (bf16_t)x;
  p[1] = p[2] = (bf16_t)0.f;
  if (!finite(x)) return;
  const bool large = !finite((float)p[0]);
  if (large) p[0] = (bf16_t)cut_off(x);
  x -= (float)p[0];
  p[1] = (bf16_t)(large ? cut_off(x) : x);
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

// ---- operands of 16 x 16 MFMAs straight from memory
typedef __attribute__((ext_vector_type(4))) float v4f;
__device__ __forceinline__ v4f mma16(Op<bf16_t>::V a, Op<bf16_t>::V b, v4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ v4f mma16(Op<f16_t>::V a, Op<f16_t>::V b, v4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

// Eight values of a row as loaded, those that the eight places from k on have before `end`.  Not SINGLE (at least eight
// values before `end`): at the end they are the row's last eight, those that an earlier group has taken as zeros: the same
// ones in either operand. ODD: 16-bit values off the boundaries of 32 bits, from the 32-bit words that hold them (16-byte
// loads at such addresses: 9705 x 2687 -> 37 in bf16 92 us, so 49).
enum Loads { WIDE, ODD, SINGLE };
template <class S> struct Raw8 { Chunk c[sizeof(S) / 2]; };
template <class S, Loads L> __device__ __forceinline__ Raw8<S> raw8(const S* row, int k, int end) {
  Raw8<S> r;
  if (L != SINGLE) {
    const S* p = row + min(k, end - 8);
    if constexpr (L == ODD) {
      const uint32_t half = (uint32_t)(uintptr_t)p & 2u;
      const uint32_t* q = reinterpret_cast<const uint32_t*>(reinterpret_cast<const char*>(p) - half);
      struct Words { uint32_t v[4]; } const w = *reinterpret_cast<const Words*>(q);
      const uint32_t last = q[half ? 4 : 3];
#pragma unroll
      for (int i = 0; i < 4; ++i) r.c[0][i] = __builtin_amdgcn_alignbit(i < 3 ? w.v[i + 1] : last, w.v[i], half * 8);
    } else {
      r = __builtin_bit_cast(Raw8<S>, *reinterpret_cast<const Loose<S, 8>*>(p));
    }
    if (k + 8 > end) {
      Vec<S, 8> v = __builtin_bit_cast(Vec<S, 8>, r);
#pragma unroll
      for (int e = 0; e < 8; ++e) v.v[e] = end - 8 + e < k ? from_f32<S>(0.f) : v.v[e];
      r = __builtin_bit_cast(Raw8<S>, v);
    }
  } else {
    Vec<S, 8> v;
#pragma unroll
    for (int e = 0; e < 8; ++e) v.v[e] = k + e < end ? row[k + e] : from_f32<S>(0.f);
    r = __builtin_bit_cast(Raw8<S>, v);
  }
  return r;
}
// ... as MFMA operands, values as planes_of has them: with its cases only where there is a value beyond the largest bf16 (a
// NaN makes all of its planes NaN here; what counts is the first)
template <class S, class T> __device__ __forceinline__ void planes8(const Raw8<S>& r, typename Op<T>::V (&p)[sizeof(S) == 4 ? 3 : 1]) {
  if constexpr (sizeof(S) == 2) {
    p[0] = __builtin_bit_cast(typename Op<T>::V, r.c[0]);
  } else {
    const Vec<float, 8> v = __builtin_bit_cast(Vec<float, 8>, r);
    float x[8], most = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      x[e] = v.v[e];
      most = fmaxf(most, fabsf(x[e]));
    }
    if (__builtin_expect(most > 3.3895314e38f, 0)) {
      Vec<bf16_t, 8> q[3];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        bf16_t t[3];
        planes_of(x[e], t);
#pragma unroll
        for (int k = 0; k < 3; ++k) q[k].v[e] = t[k];
      }
#pragma unroll
      for (int k = 0; k < 3; ++k) p[k] = __builtin_bit_cast(typename Op<T>::V, q[k]);
      return;
    }
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      const Vec<bf16_t, 8> q = round_vec<bf16_t, 8>(x);
      p[k] = __builtin_bit_cast(typename Op<T>::V, q);
      if (k < 2) {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] -= (float)q.v[e];
      }
    }
  }
}

// out[c] = sum of the row blocks' sums: sixteen threads a column, sixteen columns a block; part: LDS, 16 x 17
__device__ __forceinline__ void column_sums(const float* __restrict__ sums, int blocks, int cols, float* __restrict__ out, int block, float (*part)[17]) {
  const int cl = threadIdx.x & 15, t = threadIdx.x >> 4, c = block * 16 + cl;
  float s = 0.f;
  if (c < cols) {
    float q[4] = {0.f, 0.f, 0.f, 0.f};  // (four loads on their way)
    int b = t;
    for (; b + 48 < blocks; b += 64) {
#pragma unroll
      for (int e = 0; e < 4; ++e) q[e] += sums[(int64_t)(b + 16 * e) * cols + c];
    }
    for (; b < blocks; b += 16) q[0] += sums[(int64_t)b * cols + c];
    s = (q[0] + q[1]) + (q[2] + q[3]);
  }
  part[t][cl] = s;
  __syncthreads();
  if (t == 0 && c < cols) {
    s = 0.f;
#pragma unroll
    for (int k = 0; k < 16; ++k) s += part[k][cl];
    out[c] = s;
  }
}
__global__ void __launch_bounds__(256) dbias_kernel(const float* __restrict__ sums, int blocks, int cols, float* __restrict__ out) {
  __shared__ float part[16][17];
  column_sums(sums, blocks, cols, out, blockIdx.x, part);
}

// What sums that are not finite have to become, two bits a value (1: NaN, 2: infinity, 3: -infinity, 0: as summed), eight
// values a group
template <int GROUPS> struct Classes {
  uint32_t bits[(GROUPS + 1) / 2];
  // (the group is a constant but where the epilogue is a loop: then a select for each word)
  __device__ __forceinline__ void set(int group, const float (&v)[8]) {
    uint32_t c = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) c |= (finite(v[e]) ? 0u : v[e] != v[e] ? 1u : v[e] > 0.f ? 2u : 3u) << (2 * e);
#pragma unroll
    for (int i = 0; i < (GROUPS + 1) / 2; ++i)
      if (i == group / 2) bits[i] |= c << (group % 2 * 16);
  }
  __device__ __forceinline__ void apply(int group, float (&v)[8]) const {
    uint32_t c = 0;
#pragma unroll
    for (int i = 0; i < (GROUPS + 1) / 2; ++i)
      if (i == group / 2) c = bits[i] >> (group % 2 * 16);
#pragma unroll
    for (int e = 0; e < 8; ++e, c >>= 2)
      if (c & 3) v[e] = (c & 3) == 1 ? __builtin_nanf("") : (c & 3) == 2 ? __builtin_inff() : -__builtin_inff();
  }
};

// A launch has fewer than 2^32 threads along x: blocks of at most 1024 threads (a multiple of eight where they go to XCDs
// in turn), further rows of them along y
dim3 grid_of_blocks(int64_t blocks) {
  constexpr int64_t MOST = 1 << 21;
  return dim3((unsigned)std::min(blocks, MOST), (unsigned)((blocks + MOST - 1) / MOST));
}

int grid_of(int64_t n) { return (int)std::max<int64_t>(1, std::min<int64_t>((n + 255) / 256, 4096)); }

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }
// whether a 16-bit matrix can be an operand as it lies
bool direct(const void* p, int64_t ld, int cols) { return aligned16(p) && ld % 8 == 0 && cols % 8 == 0; }

// Tiles and parts of a product, by what it would take in us: tile steps (64 places of two operands), a block's beginning
// and end, the join of parts (a launch, reading them, and the epilogue's memory by itself).  Two blocks of 128 x 128 or
// three of 64 x 64 share a CU, which makes their steps a fifth shorter.  Fitted to 12 products of 67 MFLOP to 69 GFLOP,
// bf16 and fp32, with all tiles and 1 to 32 parts: the choice is within 10 % of the best of them.  (By filling the CUs
// alone, 1024 x 1024 x 1024 in bf16 took 14.3 us in two parts, 8.3 in one, and 432 x 13952 x 2968 79 us as 64 x 64 tiles,
// 56 as 128 x 128 in four parts; in fp32 636 and 383.)
ProductShape shape_of(int64_t M, int64_t N, int64_t K, bool f32, int64_t most_parts = 32, int only = 0) {
  constexpr int CUS = 256;
  ProductShape best = {32, 1, 0.f};
  double least = 1e300;
  const int64_t steps = f32 ? (K + 15) / 16 : (K + 63) / 64, most = std::max<int64_t>(1, std::min<int64_t>(most_parts, std::min(steps / 4, (K + 63) / 64)));
  for (int w : {128, 64, 32}) {
    if (only && w != only) continue;
    const int64_t tiles = (int64_t)ceil_div(M, 2 * w) * ceil_div(N, 2 * w);
    const double step = w == 128 ? (f32 ? 2.0 : 1.65) : w == 64 ? (f32 ? 0.65 : 0.6) : 0.3;
    const double ends = w == 128 ? 8.0 : w == 64 ? 4.0 : 3.5;
    const int share = w == 128 ? 1 : w == 64 ? 2 : 3;
    for (int64_t parts = 1; parts <= most && (parts == 1 || parts * tiles <= 4 * CUS); ++parts) {
      const int64_t each = (steps + parts - 1) / parts;
      const double load = (double)(tiles * parts) / CUS, up = std::ceil(load);
      const double busy = up <= 1 || share == 1 ? std::max(1., up) : 0.82 * 0.5 * (load + up);  // blocks a CU makes, as if one by one
      double us = std::max(1., busy) * each * step + ends * std::ceil(up / share);
      if (parts > 1) us += 3.0 + 0.3 * parts + (double)M * N * (4 * parts + (f32 ? 12 : 6)) / 6e6;
      if (us < least) { least = us; best = {w, (int)parts, (float)us}; }
    }
  }
  return best;
}

// places of a row of n columns laid out anew
template <int PL> int row_of(int n) { return (n + block_of(PL) - 1) / block_of(PL) * block_of(PL) * span_of(PL); }

}  // namespace

}  // namespace oseq
