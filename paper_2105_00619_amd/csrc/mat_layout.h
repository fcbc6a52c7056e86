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

// dbias[c] = sum of the row blocks' sums: sixteen threads a column
__global__ void __launch_bounds__(256) dbias_kernel(const float* __restrict__ sums, int blocks, int cols, float* __restrict__ out) {
  __shared__ float part[16][17];
  const int cl = threadIdx.x & 15, t = threadIdx.x >> 4, c = blockIdx.x * 16 + cl;
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
ProductShape shape_of(int64_t M, int64_t N, int64_t K, bool f32, int64_t most_parts = 32) {
  constexpr int CUS = 256;
  ProductShape best = {32, 1};
  double least = 1e300;
  const int64_t steps = f32 ? (K + 15) / 16 : (K + 63) / 64, most = std::max<int64_t>(1, std::min<int64_t>(most_parts, std::min(steps / 4, (K + 63) / 64)));
  for (int w : {128, 64, 32}) {
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
      if (us < least) { least = us; best = {w, (int)parts}; }
    }
  }
  return best;
}

// places of a row of n columns laid out anew
template <int PL> int row_of(int n) { return (n + block_of(PL) - 1) / block_of(PL) * block_of(PL) * span_of(PL); }

}  // namespace

}  // namespace oseq
