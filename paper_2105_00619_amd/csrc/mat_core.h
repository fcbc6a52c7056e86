// Matrix products on the 16-bit matrix cores: C[m][n] = sum over k of A(m, k) * B(n, k), one tile of C per block.
//
// Either operand lies in memory along the reduction ("K": element (r, k) at r * ld + k) or across it ("R": at k * ld + r), so
// one kernel body serves a layer (K, K), its data gradient (K, R) and its weight gradient (R, R).  A product may be a sum of
// several products of planes (fp32 values as two or three 16-bit planes): the planes of a pair are one longer reduction.
//
// Four wavefronts in two rows and two columns, each with WM x WN of the block's 2 WM x 2 WN; 64 values of k a stage, two stages in
// LDS, filled by loads that write LDS themselves.  A stage is loaded while the one before it is used.  With 128 x 128 a wavefront
// reads 32 KB from LDS for 64 MFMAs of 32 cycles, four of them 1024 of the 2048 cycles of a stage and the stage's writes 512; with
// 64 x 64 it would be 1024 of 512 + 512: tiles that large pay as soon as there is one for every CU.
//
// LDS, K: rows of 128 bytes, the 16-byte piece c of row r at c ^ (r & 7), so that the eight lanes a cycle serves (consecutive
// rows, one piece) touch all banks once.  R: rows of one k, 32-byte units u of 16 values at u ^ f(k): the transposing read takes
// four consecutive k of two units at once.  The loads write LDS in lane order, so each lane fetches the piece that belongs there.
#pragma once
#include "dev_common.h"

namespace oseq {
namespace mat {

typedef __attribute__((ext_vector_type(16))) float v16f;
typedef __attribute__((ext_vector_type(4))) int v4i;

template <class T> struct Op;
template <> struct Op<bf16_t> {
  typedef __attribute__((ext_vector_type(8))) __bf16 V;
  __device__ static __forceinline__ v16f mma(V a, V b, v16f c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
template <> struct Op<f16_t> {
  typedef __attribute__((ext_vector_type(8))) _Float16 V;
  __device__ static __forceinline__ v16f mma(V a, V b, v16f c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};

// One operand of a tile: `base` is its element (first row of the tile, k = 0) in plane 0, `rows` how many of the tile's rows
// exist (at least 1; R: in memory there are as many as the next multiple of 8).  ld is a multiple of 8 and base 16-byte aligned.
// K: the reduction's length is a multiple of 8.
template <class T> struct Operand {
  const T* base;
  int64_t plane;  // elements from one plane to the next
  int ld, rows;
};

// The planes that are multiplied, in the order given: product s takes plane a(s) of A and b(s) of B
struct Planes {
  uint32_t a = 0, b = 0;  // two bits each
  int n = 1;
  __host__ __device__ void add(int i, int j) { a |= (uint32_t)i << (2 * n); b |= (uint32_t)j << (2 * n); ++n; }
  // values in `planes` planes: every product whose planes' indices add up to less than `planes`, the small ones first
  __host__ __device__ static Planes of(int planes) {
    Planes p;
    if (planes == 1) return p;
    p.n = 0;
    for (int s = planes - 1; s >= 0; --s)
      for (int i = 0; i <= s; ++i) p.add(i, s - i);
    return p;
  }
};

constexpr int BK = 64;
constexpr uint32_t OUTSIDE = 0x80000000u;  // a buffer offset beyond every buffer: reads as zero

__device__ __forceinline__ v4i buffer_of(const void* p) {
  const uint64_t a = (uint64_t)p;
  v4i r;
  r[0] = __builtin_amdgcn_readfirstlane((int)(uint32_t)a);
  r[1] = __builtin_amdgcn_readfirstlane((int)((a >> 32) & 0xffffu));
  r[2] = (int)OUTSIDE;
  r[3] = 0x00020000;
  return r;
}

// 16 bytes per lane from memory to LDS, to lds + 16 * lane
__device__ __forceinline__ void load_to_lds(const v4i& buf, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds), "v"(off), "s"(buf));
}

// The loads of one operand: B rows of a tile, 64 of k
template <class T, int B, bool R>
struct Stage {
  static constexpr int BYTES = B * BK * 2, NLD = BYTES / 4096;  // loads per thread
  static constexpr int KROWS = R ? 512 / B : 0;                 // R: rows of k that a wavefront's load covers
  static constexpr int UNITS = B / 16;
  __device__ static __forceinline__ int fold(int k) { return UNITS >= 8 ? (k & 3) * 2 : UNITS >= 4 ? (k & 1) * 2 : 0; }

  uint32_t off[NLD];
  int kfirst;  // the k of this thread's piece within a stage (R: of its first load)
  const T* next;
  int64_t step;

  __device__ __forceinline__ void init(const Operand<T>& o, int wave, int lane) {
#pragma unroll
    for (int i = 0; i < NLD; ++i) {
      const int j = wave * NLD + i;
      if (R) {
        const int k = j * KROWS + lane / (B / 8), slot = lane % (B / 8);
        int r = ((slot >> 1) ^ fold(k)) * 16 + (slot & 1) * 8;
        r = min(r, (o.rows - 1) & ~7);
        off[i] = ((uint32_t)k * (uint32_t)o.ld + (uint32_t)r) * 2u;
        if (i == 0) kfirst = k;
      } else {
        const int r = min(j * 8 + (lane >> 3), o.rows - 1), c = (lane & 7) ^ (lane >> 3);
        off[i] = ((uint32_t)r * (uint32_t)o.ld + (uint32_t)c * 8u) * 2u;
        kfirst = c * 8;
      }
    }
    step = R ? (int64_t)BK * o.ld : BK;
  }
  // `left` values of k exist from the stage's first on
  __device__ __forceinline__ void load(int i, const v4i& buf, int left, uint32_t lds, int wave) const {
    const uint32_t out = (R ? kfirst + i * KROWS : kfirst) < left ? 0u : OUTSIDE;
    load_to_lds(buf, off[i] | out, lds + (uint32_t)(wave * NLD + i) * 1024u);
  }
  // the MFMA operand of rows [32 * block, + 32) of the wavefront's rows from `first` on, k in [16 * ks, + 16)
  typedef typename Op<T>::V V;
  __device__ static __forceinline__ V read(const unsigned char* st, int row, int ks, int lane) {
    if (R) {
      const int g = lane >> 4, i16 = lane & 15;
      const int k = ks * 16 + (g >> 1) * 8 + (i16 >> 2);
      const int unit = (row >> 4) + (g & 1);
      const unsigned char* p = st + k * (B * 2) + ((unit ^ fold(k)) * 32 + (i16 & 3) * 8);
      return lds_tr_read8<V>(reinterpret_cast<const T*>(p), reinterpret_cast<const T*>(p + 4 * (B * 2)));
    }
    const int r = row + (lane & 31), c = (ks * 2 + (lane >> 5)) ^ (r & 7);
    return *reinterpret_cast<const V*>(st + r * 128 + c * 16);
  }
};

template <class T, int WM, int WN, bool AR, bool BR>
struct Tile {
  static constexpr int BM = 2 * WM, BN = 2 * WN, MI = WM / 32, NI = WN / 32;
  typedef Stage<T, BM, AR> SA;
  typedef Stage<T, BN, BR> SB;
  static constexpr int STAGE = SA::BYTES + SB::BYTES, LDS = 2 * STAGE;
  static constexpr int EPITCH = WN + 4;  // floats of a row on its way out
  static_assert(4 * 32 * EPITCH * 4 <= LDS, "the epilogue's rows do not fit");
  typedef typename Op<T>::V V;
  typedef v16f Acc[MI][NI];

  // the sum over k in [0, K) of every plane pair
  __device__ static __forceinline__ void product(unsigned char* smem, const Operand<T>& a, const Operand<T>& b, const Planes& pl, int K,
                                                 Acc& acc) {
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave >> 1, wn = wave & 1;
    SA sa; SB sb;
    sa.init(a, wave, lane);
    sb.init(b, wave, lane);
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem;
    const int per = (K + BK - 1) / BK, total = per * pl.n;
    int s = 0, left = K;  // of the next stage to load
    const T* pa = a.base + (int64_t)(pl.a & 3) * a.plane;
    const T* pb = b.base + (int64_t)(pl.b & 3) * b.plane;
    v4i ba, bb;
    auto begin = [&]() { ba = buffer_of(pa); bb = buffer_of(pb); };
    auto advance = [&]() {
      left -= BK;
      pa += sa.step; pb += sb.step;
      if (left <= 0) {
        ++s;
        left = K;
        pa = a.base + (int64_t)((pl.a >> (2 * s)) & 3) * a.plane;
        pb = b.base + (int64_t)((pl.b >> (2 * s)) & 3) * b.plane;
      }
    };
    auto load_piece = [&](int i, uint32_t lds) {
      if (i < SA::NLD) sa.load(i, ba, left, lds, wave);
      else sb.load(i - SA::NLD, bb, left, lds + SA::BYTES, wave);
    };
    constexpr int NLD = SA::NLD + SB::NLD;
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NI; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;

    begin();
#pragma unroll
    for (int i = 0; i < NLD; ++i) load_piece(i, lds0);
    advance();
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (total > 1) {
      begin();
#pragma unroll
      for (int i = 0; i < NLD; ++i) load_piece(i, lds0 + STAGE);
      advance();
    }
    V fa[2][MI], fb[2][NI];
    const unsigned char* cur = smem;
    auto read = [&](int buf, const unsigned char* st, int ks) {
#pragma unroll
      for (int i = 0; i < MI; ++i) fa[buf][i] = SA::read(st, wm * WM + i * 32, ks, lane);
#pragma unroll
      for (int j = 0; j < NI; ++j) fb[buf][j] = SB::read(st + SA::BYTES, wn * WN + j * 32, ks, lane);
    };
    read(0, cur, 0);
    for (int t = 0; t < total; ++t) {
      const unsigned char* other = smem + (cur == smem ? STAGE : 0);
      const uint32_t cur_lds = lds0 + (cur == smem ? 0 : STAGE);
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) {
        const int buf = ks & 1;
        if (ks < 3) {
          read(buf ^ 1, cur, ks + 1);
        } else {
          // every read of this stage is done and the next stage has arrived: the barrier hands both over
          asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
          __builtin_amdgcn_s_barrier();
          asm volatile("" ::: "memory");
          if (t + 2 < total) {
            begin();
#pragma unroll
            for (int i = 0; i < NLD; ++i) load_piece(i, cur_lds);
            advance();
          }
          if (t + 1 < total) read(buf ^ 1, other, 0);
        }
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
          for (int j = 0; j < NI; ++j) acc[i][j] = Op<T>::mma(fa[buf][i], fb[buf][j], acc[i][j]);
      }
      cur = other;
    }
  }

  // the place in the tile of a thread's eight values number `idx` on their way out
  static constexpr int LPR = WN / 8, RPP = 64 / LPR, PASSES = 32 / RPP;  // lanes per row, rows per pass
  __device__ static __forceinline__ void place(int idx, int& r, int& c) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    r = (wave >> 1) * WM + idx / PASSES * 32 + idx % PASSES * RPP + lane / LPR;
    c = (wave & 1) * WN + lane % LPR * 8;
  }

  // f(idx, row, column, values, n) for eight neighbouring columns at a time, n of them inside: row < rows, column < cols, both from
  // the tile's corner.  A wavefront takes 32 rows at a time through its own part of LDS, so that memory sees whole rows.
  // ft, where given: the same for the transposed tile, f(column, row, ...) with eight neighbouring rows.
  template <class F, class FT>
  __device__ static __forceinline__ void out(unsigned char* smem, const Acc& acc, int rows, int cols, F&& f, FT&& ft, bool transposed) {
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave >> 1, wn = wave & 1;
    float* area = reinterpret_cast<float*>(smem) + wave * (32 * EPITCH);
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      const int r0 = wm * WM + i * 32, c0 = wn * WN;
#pragma unroll
      for (int j = 0; j < NI; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) area[(8 * (e >> 2) + 4 * (lane >> 5) + (e & 3)) * EPITCH + j * 32 + (lane & 31)] = acc[i][j][e];
      asm volatile("" ::: "memory");
#pragma unroll 1
      for (int p = 0; p < PASSES; ++p) {
        const int r = p * RPP + lane / LPR, c = (lane % LPR) * 8;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = area[r * EPITCH + c + e];
        if (r0 + r < rows && c0 + c < cols) f(i * PASSES + p, r0 + r, c0 + c, v, min(8, cols - c0 - c));
      }
      if (transposed) {
#pragma unroll 1
        for (int p = 0; p < WN / 16; ++p) {
          const int c = p * 16 + (lane & 15), r = (lane >> 4) * 8;
          float v[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = area[(r + e) * EPITCH + c];
          if (r0 + r < rows && c0 + c < cols) ft(c0 + c, r0 + r, v, min(8, rows - r0 - r));
        }
      }
      asm volatile("" ::: "memory");
    }
  }
};

}  // namespace mat
}  // namespace oseq
