// Matrix products on the 16-bit matrix cores: C[m][n] = sum over k of A(m, k) * B(n, k), one tile of C per block.
//
// Either operand lies in memory along the reduction ("K": rows of k) or across it ("R": rows of one k each), so one kernel body
// serves a layer (K, K), its data gradient (K, R) and its weight gradient (R, R).
//
// Values of more bits than 16 are two or three 16-bit planes, and their products the sum of several products of planes (the
// largest ones; mat::Steps).  The planes of neighbouring columns lie together, so that what is loaded once serves all products:
//   one plane      columns as they are
//   two planes     32 columns of plane 0, the same 32 of plane 1; ...
//   three planes   16 columns of plane 0, of plane 1, of plane 2, 16 unused; ...
// "Places" below are positions in a row so laid out.  64 places of an operand along k are a slot: four groups of 16, each
// group one plane of 16 values of k.  (Planes apart in memory, one product of planes after the other, take half as many
// loads again with two planes and twice as many with three; that is what a product of an operand of two planes with one of
// 16 bits does, TWICE below.)
//
// Four wavefronts in two rows and two columns, each with W x W of the block's 2 W x 2 W.  Slots are a ring in LDS, A and B
// in turn, filled by loads that write LDS themselves.  While the products of two slots are made, the loads of the two that
// were used up before go out, evenly.  A tile step of 256 x 256 takes 1.6 to 1.7 us with one plane and 2.1 to 2.2 with two
// (its MFMAs alone 0.95 and 1.55), one of 128 x 128 0.6 with either, one of 64 x 64 0.3; with the loads going through
// registers and stores to LDS 10 % more.
//
// LDS, K: rows of 128 bytes, the 16-byte piece c of row r at c ^ (r / 2 & 7), so that sixteen consecutive rows, one piece
// of each, touch all 64 banks once (c ^ (r & 7), right for 32 banks, cost half as many cycles again).  R: rows of one k,
// 32-byte units u of 16 values at u ^ fold(k): the transposing read takes four consecutive k of two blocks of rows at once.
// The loads write LDS in lane order, so each lane fetches the piece that belongs there.
#pragma once
#include <utility>

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

// Places that a column takes, columns that are laid out together, and where plane p of column c is
constexpr int span_of(int planes) { return planes == 3 ? 4 : planes; }
constexpr int block_of(int planes) { return planes == 1 ? 8 : planes == 2 ? 32 : 16; }
template <int PL> __host__ __device__ constexpr int64_t place_of(int64_t c, int p = 0) {
  return PL == 1 ? c : PL == 2 ? (c >> 5) * 64 + p * 32 + (c & 31) : (c >> 4) * 64 + p * 16 + (c & 15);
}

// One operand of a tile: `base` is its first place (first row of the tile, k = 0), ld the places from one row of memory to
// the next (a multiple of 8; base 16-byte aligned), `rows` how many of the tile's rows exist (at least 1).  Memory holds
// whole blocks of columns (block_of; one plane: of eight).  TWICE: places from here to the second plane, a matrix like this
// one (or 0: the same once more).
template <class T> struct Operand {
  const T* base;
  int ld, rows;
  int64_t second = 0;
};

constexpr int SLOT_K = 64;                 // places of a slot along k (R: values of k and their planes)
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

// The loads and reads of one operand: B rows of a tile.  TWICE: the reduction once, and once more with the second plane.
template <class T, int PL, int B, bool R, bool TWICE = false>
struct Feed {
  static constexpr int BYTES = B * SLOT_K * 2, NLD = BYTES / 4096;  // of a slot; loads per thread
  static constexpr int SPAN = span_of(PL);
  static constexpr int PITCH = B * SPAN;          // R: places of a row of k
  static constexpr int KROWS = R ? 512 / PITCH : 0;  // R: rows of k that a wavefront's load covers (or 0: half a row)
  static constexpr int KS = R ? SLOT_K / SPAN : SLOT_K;  // what a slot takes of the reduction: values of k (R) or places
  static constexpr int UNITS = PITCH / 16;
  __device__ static __forceinline__ int fold(int k) { return PL == 3 ? (k & 3) : UNITS >= 8 ? (k & 3) * 2 : UNITS >= 4 ? (k & 1) * 2 : 0; }

  uint32_t off[NLD];
  int kfirst;  // the k (or place) of this thread's piece within a slot, in its first load
  const T* next;
  int64_t step;
  v4i buf;
  int left;  // of the reduction from the next slot on; what lies beyond is filled with zeros
  const T* again;  // TWICE: where the second plane begins, and how long it is
  int whole;

  __device__ __forceinline__ void init(const Operand<T>& o, int K, int wave, int lane) {
#pragma unroll
    for (int i = 0; i < NLD; ++i) {
      const int j = wave * NLD + i;
      if (R) {
        const int e = j * 512 + lane * 8, k = e / PITCH, slot = (e % PITCH) / 8;
        const int unit = (slot >> 1) ^ fold(k);
        const int v = min(unit * 16 + (slot & 1) * 8, ((o.rows * SPAN - 1) | (PL == 1 ? 7 : 63)) - 7);
        off[i] = ((uint32_t)k * (uint32_t)o.ld + (uint32_t)v) * 2u | (PL == 3 && unit % 4 == 3 ? OUTSIDE : 0u);
        if (i == 0) kfirst = k;
      } else {
        const int r = j * 8 + (lane >> 3), c = (lane & 7) ^ ((r >> 1) & 7);
        off[i] = ((uint32_t)min(r, o.rows - 1) * (uint32_t)o.ld + (uint32_t)c * 8u) * 2u | (PL == 3 && c >= 6 ? OUTSIDE : 0u);
        if (i == 0) kfirst = c * 8;
      }
    }
    next = o.base;
    buf = buffer_of(next);
    step = R ? (int64_t)KS * o.ld : KS;
    left = K;
    if (TWICE) { again = o.base + o.second; whole = K; }
  }
  __device__ __forceinline__ void load(int i, uint32_t lds, int wave) const {
    uint32_t o = off[i];
    if (PL == 1) {  // (planes are laid out to whole slots along k)
      const int k = R ? kfirst + i * 512 / PITCH : kfirst ^ ((i & 1) * 32);  // (K: a load further, eight rows, the piece's bit 2 changes)
      o |= k < left ? 0u : OUTSIDE;
    } else if (R) {
      const int k = kfirst + i * 512 / PITCH;
      o |= k < left ? 0u : OUTSIDE;
    } else {
      o |= left > 0 ? 0u : OUTSIDE;
    }
    load_to_lds(buf, o, lds + (uint32_t)(wave * NLD + i) * 1024u);
  }
  __device__ __forceinline__ void advance() {
    left -= KS;
    next += step;
    if (TWICE && left <= 0) { next = again; left = whole; }
    buf = buffer_of(next);
  }
  // the MFMA operand of group g, rows [row, row + 32) of the tile
  typedef typename Op<T>::V V;
  __device__ static __forceinline__ V read(const unsigned char* st, int row, int g, int lane) {
    if (R) {
      const int kk = PL == 1 ? g : PL == 2 ? (g & 1) : 0, plane = PL == 1 ? 0 : PL == 2 ? (g >> 1) : g;
      const int q = lane >> 4, i16 = lane & 15;
      const int k = kk * 16 + (q >> 1) * 8 + (i16 >> 2);
      const int b = (row >> 4) + (q & 1);  // block of 16 rows
      const int unit = PL == 1 ? b : PL == 2 ? (b >> 1) * 4 + plane * 2 + (b & 1) : b * 4 + plane;
      const unsigned char* p = st + k * (PITCH * 2) + ((unit ^ fold(k)) * 32 + (i16 & 3) * 8);
      return lds_tr_read8<V>(reinterpret_cast<const T*>(p), reinterpret_cast<const T*>(p + 4 * (PITCH * 2)));
    }
    const int r = row + (lane & 31), c = (g * 2 + (lane >> 5)) ^ ((r >> 1) & 7);
    return *reinterpret_cast<const V*>(st + r * 128 + c * 16);
  }
};

// The products of two slots: step s multiplies group a(s) of A with group b(s) of B.  Every group is read into registers
// once; `reads` says which ones step s reads behind its MFMAs (bits 0-3: groups of A, 4-7: of B), from the steps HAND on
// those of the next two slots: a group is read again one step after its last use or later, and a step or more before its
// next one.  At HAND every group of the two slots has been read, and they change hands.
template <int PL> struct Steps;
template <> struct Steps<1> {
  static constexpr int N = 4, HAND = 2, FIRST = 0x77;
  static constexpr int a(int s) { return s; }
  static constexpr int b(int s) { return s; }
  static constexpr int reads(int s) { return s == 0 ? 0x88 : s == 1 ? 0 : s == 2 ? 0x11 : 0x66; }
};
template <> struct Steps<2> {  // (0: hi of k 0-15, 1: hi of 16-31, 2, 3: lo)  hi lo + lo hi + hi hi of each
  static constexpr int N = 6, HAND = 3, FIRST = 0x55;
  static constexpr int a(int s) { return s == 0 ? 0 : s == 1 ? 2 : s == 2 ? 0 : s == 3 ? 1 : s == 4 ? 3 : 1; }
  static constexpr int b(int s) { return s == 0 ? 2 : s == 1 ? 0 : s == 2 ? 0 : s == 3 ? 3 : s == 4 ? 1 : 1; }
  static constexpr int reads(int s) { return s == 0 ? 0x82 : s == 1 ? 0x28 : s == 3 ? 0x41 : s == 4 ? 0x14 : 0; }
};
template <> struct Steps<3> {  // every product of planes whose indices add up to at most two
  static constexpr int N = 6, HAND = 3, FIRST = 0x22;
  static constexpr int a(int s) { return s == 0 ? 1 : s == 1 ? 1 : s == 5 ? 2 : 0; }
  static constexpr int b(int s) { return s == 0 ? 1 : s == 1 ? 0 : s == 2 ? 1 : s == 3 ? 0 : s == 4 ? 2 : 0; }
  static constexpr int reads(int s) { return s == 0 ? 0x55 : s == 3 ? 0x22 : 0; }
};

// f(0), f(1), ... f(N - 1), each with its number as a constant (the compiler gives up on unrolling what is below)
template <class F, int... I> __device__ __forceinline__ void each_of(F&& f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, class F> __device__ __forceinline__ void each(F&& f) { each_of(f, std::make_integer_sequence<int, N>{}); }
// the group of the read number `i` of a step that reads the groups of `set`, mi blocks of rows each
constexpr int group_of(int set, int i, int mi) {
  for (int g = 0; g < 8; ++g)
    if (set >> g & 1) {
      if (i < mi) return g;
      i -= mi;
    }
  return 0;
}

constexpr int ring_slots(int w) { return w == 128 ? 5 : w == 64 ? 5 : 6; }

template <class T, int PL, int W, bool AR, bool BR, bool TWICE = false>
struct Tile {
  static_assert(!TWICE || PL == 1, "planes apart in memory are 16-bit operands");
  static constexpr int RING = ring_slots(W), EDGE = 2 * W, MI = W / 32;
  typedef Feed<T, PL, EDGE, AR, TWICE> FA;
  typedef Feed<T, PL, EDGE, BR, TWICE> FB;
  typedef Steps<PL> S;
  static constexpr int SLOT = FA::BYTES, LDS = RING * SLOT;
  static constexpr int EPITCH = W + 4;  // floats of a row on its way out
  static_assert(4 * 32 * EPITCH * 4 + 16 <= LDS, "the epilogue's rows and a word for each wavefront do not fit");
  typedef typename Op<T>::V V;
  typedef v16f Acc[MI][MI];
  // TWICE: what the first plane's sum is multiplied by before the second plane's is added (fp16: the first plane is held larger by as
  // much, or it would be lost below the type's smallest values)
  static constexpr float BETWEEN = __is_same(T, f16_t) ? 1.f / 2048.f : 1.f;

  // The sum over k in [0, K).  LEADING: of the first planes' products alone, which are what an infinity or a NaN makes of a
  // sum (infinity times a later plane, which may be zero or of the other sign, is not).
  template <bool LEADING = false>
  __device__ static __forceinline__ void product(unsigned char* smem, const Operand<T>& a, const Operand<T>& b, int K, Acc& acc) {
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave >> 1, wn = wave & 1;
    FA fda;
    FB fdb;
    // what a slot takes: values of k where the operand lies across it, places where along
    const int once = PL == 1 ? (K + SLOT_K - 1) / SLOT_K : (K + block_of(PL) - 1) / block_of(PL);  // slots
    const int kv = PL == 1 ? K : AR && BR ? 0 : once * SLOT_K;  // (along: at most the places of a row)
    fda.init(a, AR ? K : kv, wave, lane);
    fdb.init(b, BR ? K : kv, wave, lane);
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem;
    const int total = TWICE && !LEADING ? 2 * once : once;
    constexpr int NLD = FA::NLD, MFMAS = MI * MI, PLACES = S::N * MFMAS;
    // Load n of the sequence A, B, A, B, ... goes to slot n mod RING; from the hand-over of tile step t - 1 to that of t, loads
    // 2 t + RING - 2 and the next go out
    constexpr bool B_FIRST = RING % 2 != 0;
    auto load_place = [&](auto place, uint32_t first, uint32_t second) {
      each<2 * NLD>([&](auto n) {
        if constexpr (n * PLACES / (2 * NLD) == place) {
          constexpr int i = n % NLD;
          constexpr bool of_b = (n < NLD) == B_FIRST;
          const uint32_t lds = lds0 + (n < NLD ? first : second);
          if constexpr (of_b) fdb.load(i, lds, wave); else fda.load(i, lds, wave);
          if constexpr (i == NLD - 1) { if constexpr (of_b) fdb.advance(); else fda.advance(); }
        }
      });
    };
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < MI; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;

#pragma unroll
    for (int n = 0; n < RING - 2; ++n) {
#pragma unroll
      for (int i = 0; i < NLD; ++i) {
        if (n % 2) fdb.load(i, lds0 + n * SLOT, wave); else fda.load(i, lds0 + n * SLOT, wave);
      }
      if (n % 2) fdb.advance(); else fda.advance();
    }
    // every read of the two slots is done and the next two have arrived (younger loads may be on their way): the barrier
    // hands all four over
    constexpr int FLYING = (RING - 4) * NLD;
    auto hand_over = [&]() {
      asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(FLYING) : "memory");
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
    };
    hand_over();
    auto after = [](int slot, int by) { slot += by * SLOT; return slot >= RING * SLOT ? slot - RING * SLOT : slot; };
    int at = 0;  // the slot of A, in bytes; B's is the next one
    // operands of the MFMAs, by group; read number i of a step's set
    V fa[4][MI], fb[4][MI];
    auto read_of = [&](auto set, auto i, const unsigned char* sa, const unsigned char* sb) {
      constexpr int g = group_of(set, i, MI), r = i % MI;
      if constexpr (g < 4) fa[g][r] = FA::read(sa, wm * W + r * 32, g, lane);
      else fb[g - 4][r] = FB::read(sb, wn * W + r * 32, g - 4, lane);
    };
    each<(S::N - S::HAND) * MFMAS>([&](auto n) { load_place(n, (RING - 2) * SLOT, (RING - 1) * SLOT); });
    each<__builtin_popcount(S::FIRST) * MI>([&](auto i) { read_of(std::integral_constant<int, S::FIRST>{}, i, smem, smem + SLOT); });
    for (int t = 0; t < total; ++t) {
      if constexpr (TWICE && !LEADING && BETWEEN != 1.f) {
        if (t == once) times_between(acc);
      }
      const unsigned char *sa = smem + at, *sb = smem + after(at, 1), *na = smem + after(at, 2), *nb = smem + after(after(at, 2), 1);
      const int free0 = after(at, RING - 2), free1 = after(at, RING - 1);
      // Nothing is moved across the bars between MFMAs, or the compiler reads each operand right before its use.
      each<S::N>([&](auto s) {
        if constexpr (s == S::HAND) hand_over();
        __builtin_amdgcn_sched_barrier(0);
        constexpr int set = S::reads(s), count = __builtin_popcount(set) * MI, per = (count + MFMAS - 1) / MFMAS;
        each<MFMAS>([&](auto n) {
          if constexpr (!LEADING || (S::a(s) == 0 && S::b(s) == 0))
            acc[n / MI][n % MI] = Op<T>::mma(fa[S::a(s)][n / MI], fb[S::b(s)][n % MI], acc[n / MI][n % MI]);
          __builtin_amdgcn_sched_barrier(0);
          each<per>([&](auto j) {  // (of the last tile step: what is read is not used)
            constexpr int i = n * per + j;
            if constexpr (i < count)
              read_of(std::integral_constant<int, set>{}, std::integral_constant<int, i>{}, s < S::HAND ? sa : na, s < S::HAND ? sb : nb);
          });
          if constexpr (s < S::HAND) load_place(std::integral_constant<int, (s + S::N - S::HAND) * MFMAS + n>{}, free0, free1);
          else load_place(std::integral_constant<int, (s - S::HAND) * MFMAS + n>{}, at, after(at, 1));
          __builtin_amdgcn_sched_barrier(0);
        });
      });
      at = after(at, 2);
    }
    // (the epilogue writes LDS: what was loaded past the end has to be there first)
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  }

  // After `out`: whether any thread's flag is set.  (Not __syncthreads_or, which waits until memory has taken the tile.)
  __device__ static __forceinline__ bool any_of(unsigned char* smem, bool flag) {
    volatile uint32_t* words = reinterpret_cast<volatile uint32_t*>(smem + LDS - 16);
    const uint32_t any = __any(flag);
    if ((threadIdx.x & 63) == 0) words[threadIdx.x >> 6] = any;
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    return (words[0] | words[1] | words[2] | words[3]) != 0;
  }

  // the place in the tile of a thread's eight values number `idx` on their way out
  static constexpr int LPR = W / 8, RPP = 64 / LPR, PASSES = 32 / RPP, GROUPS = MI * PASSES;  // lanes per row, rows per pass; groups of a thread
  __device__ static __forceinline__ void place(int idx, int& r, int& c) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    r = (wave >> 1) * W + idx / PASSES * 32 + idx % PASSES * RPP + lane / LPR;
    c = (wave & 1) * W + lane % LPR * 8;
  }

  // A finished tile on its way out.  A wavefront takes 32 rows at a time through its own part of LDS, so that memory sees
  // whole rows. f(idx, row, column, values, n, d) for eight neighbouring columns at a time, n of them inside: row < rows,
  // column < cols, both from the tile's corner.  d = pre(row, column, n) is what f reads from memory.  It is asked for 32
  // rows ahead, which takes a copy of f for every eight values of a thread; with LONG, an f of many instructions, one copy
  // serves them in turn (with GELU in 32 copies, read once per tile and run once, 8192 x 2048 -> 8192 took 50 us more).
  // TURNED: the same for the transposed tile, with eight neighbouring rows: f(idx, column, row, ...).
  template <bool TURNED, bool LONG, class P, class F>
  __device__ static __forceinline__ void out(unsigned char* smem, const Acc& acc, int rows, int cols, P&& pre, F&& f) {
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave >> 1, wn = wave & 1, c0 = wn * W;
    float* area = reinterpret_cast<float*>(smem) + wave * (32 * EPITCH);
    constexpr int N = TURNED ? W / 16 : PASSES;
    typedef decltype(pre(0, 0, 0)) D;
    // row and column (from the wavefront's corner) of a thread's group in a pass
    auto row_in = [&](int p) { return TURNED ? (lane >> 4) * 8 : p * RPP + lane / LPR; };
    auto col_in = [&](int p) { return TURNED ? p * 16 + (lane & 15) : (lane % LPR) * 8; };
    auto ask = [&](int i, int p) {
      const int r = wm * W + i * 32 + row_in(p), c = c0 + col_in(p);
      if (r < rows && c < cols) return TURNED ? pre(c, r, min(8, rows - r)) : pre(r, c, min(8, cols - c));
      return D{};
    };
    auto give = [&](int i, int p, const D& d) {
      const int lr = row_in(p), lc = col_in(p), r = wm * W + i * 32 + lr, c = c0 + lc;
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = TURNED ? area[(lr + e) * EPITCH + lc] : area[lr * EPITCH + lc + e];
      if (r < rows && c < cols) {
        if (TURNED) f(i * N + p, c, r, v, min(8, rows - r), d);
        else f(i * N + p, r, c, v, min(8, cols - c), d);
      }
    };
    if constexpr (LONG) {
      each<MI>([&](auto i) {
        put_rows(area, acc[i], lane);
#pragma unroll 1
        for (int p = 0; p < N; ++p) give(i, p, ask(i, p));
        asm volatile("" ::: "memory");
      });
    } else {
      D d[2][N];
      each<N>([&](auto p) { d[0][p] = ask(0, p); });
      each<MI>([&](auto i) {
        if constexpr (i + 1 < MI) each<N>([&](auto p) { d[(i + 1) & 1][p] = ask(i + 1, p); });
        put_rows(area, acc[i], lane);
        each<N>([&](auto p) { give(i, p, d[i & 1][p]); });
        asm volatile("" ::: "memory");
      });
    }
  }
  // The same for a tile of a symmetric matrix: f changes the values, g(row, column, values) stores them, and where `both`
  // gt(column, row, values) eight neighbouring rows at the transposed place.  rows and cols are multiples of eight.
  template <class P, class F, class G, class GT>
  __device__ static __forceinline__ void out_symmetric(unsigned char* smem, const Acc& acc, int rows, int cols, bool both, P&& pre, F&& f, G&& g,
                                                       GT&& gt) {
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave >> 1, wn = wave & 1, c0 = wn * W;
    float* area = reinterpret_cast<float*>(smem) + wave * (32 * EPITCH);
    typedef decltype(pre(0, 0)) D;
    D d[2][PASSES];
    auto ask = [&](auto i) {
      each<PASSES>([&](auto p) {
        const int r = wm * W + i * 32 + p * RPP + lane / LPR, c = c0 + (lane % LPR) * 8;
        if (r < rows && c < cols) d[i & 1][p] = pre(r, c);
      });
    };
    ask(std::integral_constant<int, 0>{});
    each<MI>([&](auto i) {
      if constexpr (i + 1 < MI) ask(std::integral_constant<int, i + 1>{});
      const int r0 = wm * W + i * 32;
      put_rows(area, acc[i], lane);
      each<PASSES>([&](auto p) {
        const int r = p * RPP + lane / LPR, c = (lane % LPR) * 8;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = area[r * EPITCH + c + e];
        if (r0 + r < rows && c0 + c < cols) {
          f(r0 + r, c0 + c, v, d[i & 1][p]);
          g(r0 + r, c0 + c, v);
        }
        if (both) {
#pragma unroll
          for (int e = 0; e < 8; ++e) area[r * EPITCH + c + e] = v[e];
        }
      });
      asm volatile("" ::: "memory");
      if (both)
        each<W / 16>([&](auto p) {
          const int c = p * 16 + (lane & 15), r = (lane >> 4) * 8;
          float v[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = area[(r + e) * EPITCH + c];
          if (r0 + r < rows && c0 + c < cols) gt(c0 + c, r0 + r, v);
        });
      asm volatile("" ::: "memory");
    });
  }

 private:
  // Sums times BETWEEN, each where it lies.  (As ordinary multiplications the compiler moves all of a 256 x 256 tile's out of the
  // accumulation registers at once and spills, in the loop too.)  It does not see into the block, so what an MFMA and a use of its result
  // have to be apart is said here: 19 cycles before, 2 behind.
  __device__ static __forceinline__ void times_between(Acc& acc) {
    asm volatile("s_nop 15\n\ts_nop 15");
    each<MI * MI * 16>([&](auto n) {
      float x = acc[n / 16 / MI][n / 16 % MI][n % 16], t;
      asm volatile("v_accvgpr_read_b32 %1, %0\n\tv_mul_f32 %1, %2, %1\n\tv_accvgpr_write_b32 %0, %1" : "+a"(x), "=&v"(t) : "s"(BETWEEN));
      acc[n / 16 / MI][n / 16 % MI][n % 16] = x;
    });
    asm volatile("s_nop 7");
  }
  // 32 rows of a wavefront's sums to its part of LDS
  __device__ static __forceinline__ void put_rows(float* area, const v16f (&acc)[MI], int lane) {
#pragma unroll
    for (int j = 0; j < MI; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) area[(8 * (e >> 2) + 4 * (lane >> 5) + (e & 3)) * EPITCH + j * 32 + (lane & 31)] = acc[j][e];
    asm volatile("" ::: "memory");
  }
};

}  // namespace mat
}  // namespace oseq
