// Losses of softmax(s), s = (x w^T + bias) / temperature, against a label or a teacher's distribution over some classes:
//   loss = sum over classes of q (log q - s) + lse(s),   ds = p - q,   p = exp(s - lse).
// The logits are made tile by tile (mat_core.h) and never leave the block that makes them: forward it keeps of each row the maximum of its
// columns, the sum of their exponentials above it and the targets' logits, which a second kernel joins; backward it turns them into ds, in
// planes of the storage type (two of 16 bits) and for a piece of the classes at a time, which the gradients' products read (k_loss_grad.hip).  What a row's target is at some of its
// columns is put into the tile on its way through LDS, where the row's values lie side by side.
// Large calls are bound by the matrix cores: 8192 x 4096 -> 128000 in bf16 6.33 ms forward (1360 TFLOP/s, matrix cores busy 75 % of the kernel) and
// 35.3 ms backward (five such products, two each for dx and dw, 1220 TFLOP/s); few rows by memory (the weights at 4.8 TB/s), small calls by their launches.
#include "mat_layout.h"
#include "parts.h"

namespace oseq {

namespace {

constexpr float LOG2E = 1.4426950408889634f;

// ---- operands laid out anew --------------------------------------------------------------------------------------------
// Columns are filled up to whole blocks (block_of) with zeros.  With `info`, rows times their power of two; `twice`: all rows once more behind them,
// for the second plane of ds, over what that is held larger by.
struct Layout { const void* src; int64_t ld, rows; int cols; void* dst; const float4* info; const float* scale; bool twice; };
template <class S, class T, int PL> __device__ __forceinline__ void lay_out_rows(const Layout& a, int block, int blocks) {
  const int c8 = (a.cols + block_of(PL) - 1) / block_of(PL) * (block_of(PL) / 8);
  const int64_t n = a.rows * c8 * (a.twice ? 2 : 1);
  const float largest = a.info ? *a.scale : 1.f;
  for (int64_t i = (int64_t)block * 256 + threadIdx.x; i < n; i += (int64_t)blocks * 256) {
    const int64_t r = i / c8, from = r < a.rows ? r : r - a.rows;
    const int c = (int)(i - r * c8) * 8;
    float v[8];
    load8<S>((const S*)a.src + from * a.ld + c, max(0, min(8, a.cols - c)), v);
    if (a.info) {
      const float4 row = a.info[from];
      const float f = row.w / largest * (r < a.rows ? 1.f : Tile<T, PL, 32, false, false>::BETWEEN);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = row.z == 0.f ? 0.f : v[e] * f;
    }
    store_planes8<PL, T>((T*)a.dst + r * c8 * (8 * span_of(PL)), c, v);
  }
}

// ---- logits -------------------------------------------------------------------------------------------------------------
struct Logits {
  const void *x, *w; int ldx, ldw;  // operands, mat_core.h
  int64_t M;
  int N, K, first;                  // classes of this piece, values of a row, the piece's first class
  int tiles_m, tiles_n;
  const float* bias;                // of all classes, or null
  float per_temperature;
  const int32_t* labels;
  // a teacher: its entries in order of their classes, `top` a row; where those of a run of W columns begin
  int top, columns;
  const int32_t* index; const float2* target; const uint16_t* start;
  // forward
  float2* sums; float* totals; float* picked;
  // backward
  const float4* info;
  float spread, hit, scale;         // label_smoothing / classes; 1 - label_smoothing; what ds is held times
  void* ds; int64_t ds_row;
  int64_t low;                      // 16 bits: rows of ds behind which its second plane goes
  float* bias_sums;
  Layout xs; int xs_blocks;         // blocks behind the tiles' lay out x for dw, or 0
};

// What the backward pass knows of a row, four floats: its lse; what p and the target are multiplied by (the second is 0 in a row that is
// left out); the factor of everything that comes of the row.

// v of a lane and of the one 32 further on (or before), in both
__device__ __forceinline__ void halves(float v, float& a, float& b) {
  const u32x2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  a = __uint_as_float(r.x);
  b = __uint_as_float(r.y);
}
__device__ __forceinline__ float halves_max(float v) { float a, b; halves(v, a, b); return fmaxf(a, b); }
__device__ __forceinline__ float halves_sum(float v) { float a, b; halves(v, a, b); return a + b; }

// In 16 bits exp(k' (v - from)) is one multiply-add, 2^(k v - r), r = k from as rounded, k = k' log2(e): off by a factor that is the same for all v
// and is made up for.  That goes where rounding k from costs 2^-13 at most.  (A mask's logits, of 1e10 or a type's lowest value, are beyond: rounding
// k from alone would make exp of them 2^100, or k from infinite.)  Farther ones have `from` taken off first, a row of them beside others that stay as
// they are: a row's bits are its own.
__device__ __forceinline__ bool far_off(float exponent) { return !(fabsf(exponent) <= 4096.f); }

// An accumulator's value.  256 x 256 tiles have all of their accumulation registers full: as an ordinary copy the compiler moves them out at
// once where the block's paths part, and spills.  It does not see into the instruction, so what lies between a tile's last MFMA and
// the first of these is said where they begin (settled).
template <int W> __device__ __forceinline__ float value_of(float acc) {
  if (W < 128) return acc;
  float v;
  asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(v) : "a"(acc));
  return v;
}
template <int W> __device__ __forceinline__ void settled() {
  if (W == 128) asm volatile("s_nop 15\n\ts_nop 15");
}

// A tile's logits: the weights are the products' first operand, the samples the second, so that a lane has one sample of 32 and, with the lane 32
// further on, all W classes of its wavefront: maximum, sum and exponentials need no other lane's values.  Where a target falls among
// these classes the 32 samples' values pass LDS, 16 bytes at a time, for the lane to find its own; ds leaves through LDS as it is stored, so
// that memory sees whole rows.  (With the samples first, a row is spread over 32 lanes and all of it has to pass LDS in fp32: the tile's end took
// 12 to 14 us of a block's time, so 5 to 8.)
template <class S, class T, int W, bool TOP, bool GRAD>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(W == 128 ? 1 : 2, W == 128 ? 1 : 8)))
logits_kernel(Logits a) {
  constexpr int PL = sizeof(S) == 4 ? 3 : 1;
  constexpr bool FULL = PL == 3;
  typedef Tile<T, PL, W, false, false> G;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  const int total = a.tiles_m * a.tiles_n;
  const uint32_t block = blockIdx.y * gridDim.x + blockIdx.x;
  // neighbouring tiles on one XCD: each of the eight takes a run of them, eight rows of tiles at a time
  const int per = (total + 7) / 8, id = (block & 7) * per + (block >> 3);
  if (GRAD && (int)(block >> 3) >= per) {
    const int copy = (int)block - per * 8;
    if (copy < a.xs_blocks) lay_out_rows<S, T, PL>(a.xs, copy, a.xs_blocks);
    return;
  }
  if ((int)(block >> 3) >= per || id >= total) return;
  const int band = id / (8 * a.tiles_n), rows_in = min(8, a.tiles_m - band * 8), u = id - band * 8 * a.tiles_n;
  const int tn = u / rows_in, tm = band * 8 + u - tn * rows_in;
  const int64_t m0 = (int64_t)tm * G::EDGE;
  const int n0 = tn * G::EDGE, rows = (int)min<int64_t>(G::EDGE, a.M - m0), cols = min(G::EDGE, a.N - n0);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave >> 1, wn = wave & 1, half = lane >> 5, sl = lane & 31;
  const int c0 = wm * W, inside = min(W, cols - c0);          // the wavefront's classes, of the tile
  const int first = a.first + n0 + c0, column = first / W;    // ... of all, and their run
  // a lane's samples, one of each 32: what is known of them, and the targets among these classes: entries [k0, k1), or the label's place k0
  int k0[G::MI], k1[G::MI];
  float4 info[GRAD ? G::MI : 1];
  each<G::MI>([&](auto j) {
    const int r = wn * W + j * 32 + sl;
    const int64_t row = m0 + min(r, rows - 1);
    if (GRAD) info[j] = a.info[row];
    if (TOP) {
      const uint16_t* s = a.start + row * (a.columns + 1) + min(column, a.columns - 1);
      k0[j] = s[0];
      k1[j] = s[1];
    } else {
      k0[j] = a.labels[row] - first;
      k1[j] = k0[j] >= 0 && k0[j] < inside ? k0[j] + 1 : k0[j];
    }
    if (r >= rows) k1[j] = k0[j];
  });
  typename G::Acc acc;
  G::product(smem, Operand<T>{(const T*)a.w + (int64_t)n0 * a.ldw, a.ldw, cols}, Operand<T>{(const T*)a.x + m0 * a.ldx, a.ldx, rows}, a.K, acc);
  settled<W>();
  if (inside <= 0) return;
  // a wavefront's part of LDS: 32 rows of W values, or of as many places as ds takes of them
  constexpr int PITCH = W * span_of(PL) + 8, PART = 32 * (GRAD && PITCH * 2 > G::EPITCH * 4 ? PITCH * 2 : G::EPITCH * 4);
  static_assert(4 * PART + 4 * W * 4 <= G::LDS, "the rows on their way out do not fit");
  float* area = reinterpret_cast<float*>(smem + wave * PART);
  T* out = reinterpret_cast<T*>(smem + wave * PART);
  // a lane's values of a block of samples: class 32 i + 8 q + 4 half + e at 16 i + 4 q + e
  constexpr int NV = G::MI * 16;
  auto class_of = [&](int n) { return n / 16 * 32 + n % 16 / 4 * 8 + half * 4 + n % 4; };
  float* bias = reinterpret_cast<float*>(smem + 4 * PART) + wave * W;  // (from LDS for each block of samples: registers are short)
  if (a.bias) {
    for (int c = lane; c < inside; c += 64) bias[c] = a.bias[first + c];
    asm volatile("" ::: "memory");
  }
  const float k = a.per_temperature * LOG2E;
  float sums[GRAD ? NV : 1];
  if (GRAD) {
#pragma unroll
    for (int n = 0; n < NV; ++n) sums[n] = 0.f;
  }
  each<G::MI>([&](auto j) {
    const int r = wn * W + j * 32 + sl;
    const bool real = r < rows;
    const int64_t row = m0 + min(r, rows - 1);
    float v[NV];
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int n = 0; n < NV; ++n) v[n] = value_of<W>(acc[n / 16][j][n % 16]);
    if (a.bias) {
#pragma unroll
      for (int n = 0; n < NV; n += 4) {
        const float4 b = *reinterpret_cast<const float4*>(bias + class_of(n));
        v[n] += b.x; v[n + 1] += b.y; v[n + 2] += b.z; v[n + 3] += b.w;
      }
    }
    const bool any = __any(k1[j] > k0[j]);
    // the values in rows of LDS, W of a sample, whose first lane takes its entries in turn
    auto put = [&]() {
#pragma unroll
      for (int n = 0; n < NV; n += 4)
        *reinterpret_cast<float4*>(area + sl * G::EPITCH + class_of(n)) = make_float4(v[n], v[n + 1], v[n + 2], v[n + 3]);
      asm volatile("" ::: "memory");
    };
    if constexpr (!GRAD) {
      if (any) {
        put();
        if (!half) {
          if (TOP) {
            for (int t = k0[j]; t < k1[j]; ++t) a.picked[row * a.top + t] = area[sl * G::EPITCH + a.index[row * a.top + t] - first] * a.per_temperature;
          } else if (k1[j] > k0[j]) {
            a.picked[row] = area[sl * G::EPITCH + k0[j]] * a.per_temperature;
          }
        }
        asm volatile("" ::: "memory");
      }
      float all = 0.f;
      if (a.totals && inside == W) {
#pragma unroll
        for (int n = 0; n < NV; ++n) all += v[n];
      } else if (a.totals) {
#pragma unroll
        for (int n = 0; n < NV; ++n) all += class_of(n) < inside ? v[n] : 0.f;
      }
      if (inside < W) {
#pragma unroll
        for (int n = 0; n < NV; ++n) v[n] = class_of(n) < inside ? v[n] : -__builtin_inff();
      }
      float most = v[0];
#pragma unroll
      for (int n = 1; n < NV; ++n) most = fmaxf(most, v[n]);
      most = halves_max(most);
      // (nothing but -infinity: a sum of zero; an infinity: an infinite sum, above the largest finite maximum)
      const bool infinite = most == __builtin_inff();
      const float above = infinite || most == -__builtin_inff() ? 0.f : most;
      const bool far = FULL || far_off(above * k);
      const float from = far ? above : 0.f, r2 = far ? 0.f : above * k;
      if (FULL || __any(far)) {
#pragma unroll
        for (int n = 0; n < NV; ++n) v[n] -= from;
      }
      float sum = 0.f, sum2 = 0.f;
#pragma unroll
      for (int n = 0; n < NV; n += 2) {
        sum += __builtin_amdgcn_exp2f(FULL ? v[n] * k : __fmaf_rn(v[n], k, -r2));
        sum2 += __builtin_amdgcn_exp2f(FULL ? v[n + 1] * k : __fmaf_rn(v[n + 1], k, -r2));
      }
      sum += sum2;
      if (!FULL) sum *= __builtin_amdgcn_exp2f(__fmaf_rn(from - above, k, r2));
      sum = halves_sum(sum);
      if (a.totals) all = halves_sum(all) * a.per_temperature;
      if (!half && real) {
        const int64_t at = (int64_t)column * a.M + row;
        a.sums[at] = make_float2(infinite ? 3.4028235e38f : most * a.per_temperature, sum);
        if (a.totals) a.totals[at] = all;
      }
    } else {
      // (16 bits: what rounding lse log2(e) leaves goes into the row's factor of p)
      const float lse = info[j].x, lse2 = lse * LOG2E, spread = a.spread * info[j].z;
      const bool used = real && info[j].z != 0.f;
      const bool far = FULL || far_off(lse2);
      const float kp = far ? LOG2E : k, r2 = far ? 0.f : lse2;
      const float factor_p = far ? info[j].y : info[j].y * __fmaf_rn(__fmaf_rn(lse, LOG2E, -lse2), -0.69314718f, 1.f);
      if (FULL || __any(far)) {
#pragma unroll
        for (int n = 0; n < NV; ++n) v[n] = far ? v[n] * a.per_temperature - lse : v[n];
      }
#pragma unroll
      for (int n = 0; n < NV; ++n)
        v[n] = __fmaf_rn(__builtin_amdgcn_exp2f(FULL ? v[n] * kp : __fmaf_rn(v[n], kp, -r2)), factor_p, -spread);
      if (inside < W) {
#pragma unroll
        for (int n = 0; n < NV; ++n) v[n] = class_of(n) < inside ? v[n] : 0.f;
      }
      if (any) {
        put();
        if (!half) {
          if (TOP) {
            for (int t = k0[j]; t < k1[j]; ++t) area[sl * G::EPITCH + a.index[row * a.top + t] - first] -= a.target[row * a.top + t].x * info[j].z;
          } else if (k1[j] > k0[j]) {
            area[sl * G::EPITCH + k0[j]] -= a.hit * info[j].z;
          }
        }
        asm volatile("" ::: "memory");
#pragma unroll
        for (int n = 0; n < NV; n += 4) {
          const float4 t = *reinterpret_cast<const float4*>(area + sl * G::EPITCH + class_of(n));
          v[n] = t.x; v[n + 1] = t.y; v[n + 2] = t.z; v[n + 3] = t.w;
        }
      }
#pragma unroll
      for (int n = 0; n < NV; ++n) v[n] = used ? v[n] : 0.f;
      if (a.bias_sums) {
        const float factor = used ? info[j].w : 0.f;
#pragma unroll
        for (int n = 0; n < NV; ++n) sums[n] = __fmaf_rn(v[n], factor, sums[n]);
      }
      // out: rows of places, 16 bytes a lane; the columns up to whole blocks (block_of) are zeros already
      constexpr int LANES = W * span_of(PL) / 8, AT_ONCE = 64 / LANES > 0 ? 64 / LANES : 1;  // lanes of a row, rows at once
      const int padded = ((a.N + block_of(PL) - 1) / block_of(PL) * block_of(PL) - n0 - c0) * span_of(PL);
      // 16 bits: two planes, ds rounded and what that leaves, in fp16 2048 times larger (mat_core.h); an infinity is in the first one alone
      constexpr int PLANES = PL == 1 ? 2 : 1;
      for (int plane = 0; plane < PLANES; ++plane) {
#pragma unroll
        for (int n = 0; n < NV; n += 4) {
          const int c = class_of(n);
          float q[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) q[e] = v[n + e] * a.scale;
          if constexpr (PL == 1) {
            Vec<T, 4> t = round_vec<T, 4>(q);
            if (plane) {
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const float rest = q[e] - to_f32(t.v[e]);
                q[e] = finite(rest) ? rest * (1.f / G::BETWEEN) : 0.f;
              }
              t = round_vec<T, 4>(q);
            }
            *reinterpret_cast<Vec<T, 4>*>(out + sl * PITCH + c) = t;
          } else {
            // (values within 2, or NaN, which then is in every plane: no cases)
#pragma unroll
            for (int p = 0; p < 3; ++p) {
              const Vec<T, 4> t = round_vec<T, 4>(q);
              *reinterpret_cast<Vec<T, 4>*>(out + sl * PITCH + place_of<PL>(c, p)) = t;
#pragma unroll
              for (int e = 0; e < 4; ++e) q[e] -= (float)t.v[e];
            }
          }
        }
        asm volatile("" ::: "memory");
        T* ds = (T*)a.ds + (m0 + plane * a.low) * a.ds_row + place_of<PL>(n0 + c0);
#pragma unroll
        for (int q = 0; q < 32 / AT_ONCE; ++q) {
          const int o = q * AT_ONCE + lane / LANES, p = lane % LANES * 8, to = wn * W + j * 32 + o;
          const Chunk t = *reinterpret_cast<const Chunk*>(out + o * PITCH + p);
          if (to < rows && p < padded && !(PL == 3 && p % 64 >= 48)) *reinterpret_cast<Chunk*>(ds + to * a.ds_row + p) = t;
        }
        asm volatile("" ::: "memory");
      }
    }
  });
  if constexpr (GRAD) {
    if (!a.bias_sums) return;
    // over the 32 lanes of a half
#pragma unroll
    for (int n = 0; n < NV; ++n) sums[n] = lanes_sum<32>(sums[n]);
    if (sl == 0) {
      float* out = a.bias_sums + (int64_t)(tm * 2 + wn) * a.N + n0 + c0;
#pragma unroll
      for (int n = 0; n < NV; ++n)
        if (class_of(n) < inside) out[class_of(n)] = sums[n];
    }
  }
}

// ---- few rows ----------------------------------------------------------------------------------------------------------
// Up to 64 rows whose weights would have to be laid out anew (fp32, or off the alignment of 16 bytes): straight from memory into 16 x 16
// MFMAs, as the layers do it, 64, 32 or 16 classes of up to 16, 32 or 64 rows a block (what is read of x, and split into planes, serves all of
// them), its wavefronts (4 to 16) sharing the reduction.  The forward pass alone; a row's sums are of runs of 16 classes.
// 16 x 2048 -> 65536 in fp32: 112 us so, 890 by way of planes in memory; 18 x 3549 -> 29711 in fp16 105 us.
constexpr int SKINNY_ROWS = 64;
template <class S, class T, int MB, Loads L, bool TOP>
__global__ void __launch_bounds__(1024) few_logits_kernel(Logits a, int k_wave) {
  constexpr int PL = sizeof(S) == 4 ? 3 : 1, CB = 4 / MB, U = PL == 3 || L == SINGLE ? 1 : L == ODD ? 2 : 4;
  typedef typename Op<T>::V V;
  extern __shared__ float red[];  // [wavefront][CB][MB][256]
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  const int64_t block0 = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * (16 * CB);
  if (block0 >= a.N) return;
  const int r16 = lane & 15, kc = (lane >> 4) * 8;
  const int k0 = wave * k_wave, k1 = min(a.K, k0 + k_wave);
  const S *one[CB], *many[MB];
#pragma unroll
  for (int c = 0; c < CB; ++c) one[c] = (const S*)a.w + min(block0 + c * 16 + r16, (int64_t)a.N - 1) * a.ldw;
#pragma unroll
  for (int m = 0; m < MB; ++m) many[m] = (const S*)a.x + min<int64_t>(m * 16 + r16, a.M - 1) * a.ldx;
  v4f acc[CB][MB], rest[CB][MB];
#pragma unroll
  for (int c = 0; c < CB; ++c)
#pragma unroll
    for (int m = 0; m < MB; ++m) acc[c][m] = rest[c][m] = v4f{0.f, 0.f, 0.f, 0.f};
  for (int k = k0; k < k1; k += 32 * U) {
    Raw8<S> ro[U][CB], rm[U][MB];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int c = 0; c < CB; ++c) ro[u][c] = raw8<S, L>(one[c], k + u * 32 + kc, k1);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int m = 0; m < MB; ++m) rm[u][m] = raw8<S, L>(many[m], k + u * 32 + kc, k1);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      auto add = [&](int c, int m, const V (&po)[PL], const V (&pm)[PL]) {
#pragma unroll
        for (int i = PL - 1; i >= 0; --i)
#pragma unroll
          for (int j = PL - 1 - i; j >= 0; --j) {
            v4f& sum = i + j ? rest[c][m] : acc[c][m];
            sum = mma16(po[i], pm[j], sum);
          }
      };
      V po[PL], pm[CB == 1 ? 1 : MB][PL];  // (one block of classes: the rows' planes in turn)
      if constexpr (CB == 1) {
        planes8<S, T>(ro[u][0], po);
#pragma unroll
        for (int m = 0; m < MB; ++m) {
          planes8<S, T>(rm[u][m], pm[0]);
          add(0, m, po, pm[0]);
        }
      } else {
#pragma unroll
        for (int m = 0; m < MB; ++m) planes8<S, T>(rm[u][m], pm[m]);
#pragma unroll
        for (int c = 0; c < CB; ++c) {
          planes8<S, T>(ro[u][c], po);
#pragma unroll
          for (int m = 0; m < MB; ++m) add(c, m, po, pm[m]);
        }
      }
    }
  }
#pragma unroll
  for (int c = 0; c < CB; ++c)
#pragma unroll
    for (int m = 0; m < MB; ++m) {
      if constexpr (PL == 3) {
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[c][m][e] += finite(acc[c][m][e]) ? rest[c][m][e] : 0.f;
      }
      *reinterpret_cast<v4f*>(red + (((wave * CB + c) * MB + m) * 64 + lane) * 4) = acc[c][m];
    }
  __syncthreads();
  // a wavefront has 16 rows, four threads each with four of the classes
  const int i = threadIdx.x, row = (i >> 6) % MB * 16 + (i & 15), c = (i & 63) >> 4;
  const int64_t first = block0 + (i >> 6) / MB * 16;
  if (i >= CB * MB * 64 || first >= a.N) return;
  float v[4] = {0.f, 0.f, 0.f, 0.f};
  for (int q = 0; q < waves; ++q) {
    const v4f t = *reinterpret_cast<const v4f*>(red + (q * CB * MB * 64 + i) * 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] += t[e];
  }
  const bool real = row < a.M;
  const int cls = a.first + (int)first + c * 4, inside = min(4, (int)(a.N - first) - c * 4);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (a.bias && e < inside) v[e] += a.bias[cls + e];
    v[e] *= a.per_temperature;
  }
  const int column = (a.first + (int)first) / 16;
  if (real) {
    if (TOP) {
      const uint16_t* s = a.start + (int64_t)row * (a.columns + 1) + column;
      for (int t = s[0]; t < s[1]; ++t) {
        const int at = a.index[row * a.top + t] - cls;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (at == e) a.picked[row * a.top + t] = v[e];
      }
    } else {
      const int at = a.labels[row] - cls;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (at == e && e < inside) a.picked[row] = v[e];
    }
  }
  float all = 0.f, most = -__builtin_inff();
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (e < inside) all += v[e];
    v[e] = e < inside ? v[e] : -__builtin_inff();
    most = fmaxf(most, v[e]);
  }
  most = fmaxf(most, __shfl_xor(most, 16));
  most = fmaxf(most, __shfl_xor(most, 32));
  const bool infinite = most == __builtin_inff();  // (as in a tile)
  const float above = infinite || most == -__builtin_inff() ? 0.f : most;
  float sum = 0.f;
#pragma unroll
  for (int e = 0; e < 4; ++e) sum += __builtin_amdgcn_exp2f((v[e] - above) * LOG2E);
  sum += __shfl_xor(sum, 16);
  sum += __shfl_xor(sum, 32);
  all += __shfl_xor(all, 16);
  all += __shfl_xor(all, 32);
  if (real && c == 0) {
    const int64_t at = (int64_t)column * a.M + row;
    a.sums[at] = make_float2(infinite ? 3.4028235e38f : most, sum);
    if (a.totals) a.totals[at] = all;
  }
}

template <class S, class T, int MB, Loads L> void run_few_of(hipStream_t st, const Logits& l) {
  // wavefronts of at least 256 values of k each, more of them where there are few blocks
  const int blocks = ceil_div(l.N, 64 / MB), most = blocks >= 1024 ? 4 : blocks >= 256 ? 8 : 16;
  int waves = 4;
  while (waves < most && waves * 512 <= l.K) waves *= 2;
  const int k_wave = (ceil_div(l.K, waves) + 31) & ~31;
  if (l.labels) OSEQ_LAUNCH((few_logits_kernel<S, T, MB, L, false>), grid_of_blocks(blocks), dim3(waves * 64), (size_t)waves * 4096, st, l, k_wave);
  else OSEQ_LAUNCH((few_logits_kernel<S, T, MB, L, true>), grid_of_blocks(blocks), dim3(waves * 64), (size_t)waves * 4096, st, l, k_wave);
}
template <class S, class T, Loads L> void run_few_by(hipStream_t st, const Logits& l) {
  if (l.M <= 16) run_few_of<S, T, 1, L>(st, l);
  else if (l.M <= 32) run_few_of<S, T, 2, L>(st, l);
  else run_few_of<S, T, 4, L>(st, l);
}
template <class S, class T> void run_few(hipStream_t st, const Logits& l) {
  const bool odd = sizeof(S) == 2 && (l.K % 2 || l.ldx % 2 || l.ldw % 2 || (uintptr_t)l.x % 4 || (uintptr_t)l.w % 4);
  if (l.K < 8) return run_few_by<S, T, SINGLE>(st, l);
  if constexpr (sizeof(S) == 2) {
    if (odd) return run_few_by<S, T, ODD>(st, l);
  }
  run_few_by<S, T, WIDE>(st, l);
}

// Up to 16 rows of aligned 16-bit operands: the weights are what is read, 16 classes at a time by all wavefronts of a block, 512 values of k
// each, and the next 16 classes on their way; the rows of x stay in registers as operands.  A block walks its groups of classes, a wavefront in turn
// adds up a group's sums and goes on with the rows' maxima and sums of exponentials: one of each row for every block.
// 16 x 2048 -> 65536, ten such matrices of 268 MB in turn, which no cache holds: 55 us and 5 for the join (4.8 TB/s); a call 62, as tiles 73.
struct Stream { Logits l; int groups; };
constexpr int STREAM_ROWS = 16, KS = 16;  // (32 rows of 256 values of k: 80 us, as tiles 72)
template <class T, bool TOP>
__global__ void __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2, 2))) stream_logits_kernel(Stream s) {
  typedef typename Op<T>::V V;
  const Logits& a = s.l;
  extern __shared__ float red[];  // [2][wavefront][256]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  const int r16 = lane & 15, kc = (lane >> 4) * 8, k0 = wave * (32 * KS);
  const V zero = {};
  V px[KS], pw[2][KS];
  const T* x = (const T*)a.x + min<int64_t>(r16, a.M - 1) * a.ldx;
#pragma unroll
  for (int u = 0; u < KS; ++u) {
    const int k = k0 + u * 32 + kc;
    px[u] = k < a.K ? *reinterpret_cast<const V*>(x + k) : zero;
  }
  // (past a row's end its first values, taken for zeros)
  auto fetch = [&](int g, V (&p)[KS]) {
    const T* w = (const T*)a.w + (int64_t)min(g * 16 + r16, a.N - 1) * a.ldw;
#pragma unroll
    for (int u = 0; u < KS; ++u) {
      const int k = k0 + u * 32 + kc;
      p[u] = __builtin_nontemporal_load(reinterpret_cast<const V*>(w + (k < a.K ? k : 0)));
    }
  };
  // of a lane's row: what its wavefront has seen
  float most = -__builtin_inff(), sum = 0.f, all = 0.f;
  auto group = [&](int g, int turn, const V (&p)[KS]) {
    v4f acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int u = 0; u < KS; ++u) acc = mma16(k0 + u * 32 + kc < a.K ? p[u] : zero, px[u], acc);
    float* r = red + (turn & 1) * (waves * 256);
    *reinterpret_cast<v4f*>(r + (wave * 64 + lane) * 4) = acc;
    __syncthreads();
    if (turn % waves != wave) return;
    const int cls = a.first + g * 16 + (lane >> 4) * 4, inside = min(4, a.N - g * 16 - (lane >> 4) * 4);
    {
      float v[4] = {0.f, 0.f, 0.f, 0.f};
      for (int q = 0; q < waves; ++q) {
        const v4f t = *reinterpret_cast<const v4f*>(r + (q * 64 + lane) * 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += t[e];
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (a.bias && e < inside) v[e] += a.bias[cls + e];
        v[e] *= a.per_temperature;
      }
      const int row = r16;
      if (row < a.M) {
        if (TOP) {
          const uint16_t* st = a.start + (int64_t)row * (a.columns + 1) + (a.first + g * 16) / 16;
          for (int t = st[0]; t < st[1]; ++t) {
            const int at = a.index[row * a.top + t] - cls;
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (at == e) a.picked[row * a.top + t] = v[e];
          }
        } else {
          const int at = a.labels[row] - cls;
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (at == e && e < inside) a.picked[row] = v[e];
        }
      }
      float top = most;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (e < inside) all += v[e];
        v[e] = e < inside ? v[e] : -__builtin_inff();
        top = fmaxf(top, v[e]);
      }
      // (an infinity: an infinite sum, above the largest finite maximum, as in a tile)
      const float above = top == -__builtin_inff() || top == __builtin_inff() ? 0.f : top;
      float more = sum == 0.f ? 0.f : sum * __builtin_amdgcn_exp2f((most - above) * LOG2E);
#pragma unroll
      for (int e = 0; e < 4; ++e) more += __builtin_amdgcn_exp2f((v[e] - above) * LOG2E);
      sum = more;
      most = top == __builtin_inff() ? 3.4028235e38f : top;
    }
  };
  int g = blockIdx.x, turn = 0;
  if (g < s.groups) fetch(g, pw[0]);
  for (; g < s.groups; g += 2 * gridDim.x, turn += 2) {
    const int g1 = g + gridDim.x, g2 = g1 + gridDim.x;
    if (g1 < s.groups) fetch(g1, pw[1]);
    group(g, turn, pw[0]);
    if (g1 >= s.groups) break;
    if (g2 < s.groups) fetch(g2, pw[0]);
    group(g1, turn + 1, pw[1]);
  }
  // the wavefronts' and the lanes' joined: red holds (maximum, sum, all) of each
  __syncthreads();
  float* mine = red + (wave * 64 + lane) * 3;
  mine[0] = most; mine[1] = sum; mine[2] = all;
  __syncthreads();
  if (const int row = threadIdx.x; row < a.M) {
    float top = -__builtin_inff(), total = 0.f, every = 0.f;
    for (int i = 0; i < waves * 4; ++i) {
      const float* r = red + ((i >> 2) * 64 + (i & 3) * 16 + row) * 3;
      const float up = fmaxf(top, r[0]);
      total = up == -__builtin_inff() ? total + r[1] : total * __builtin_amdgcn_exp2f((top - up) * LOG2E) + r[1] * __builtin_amdgcn_exp2f((r[0] - up) * LOG2E);
      top = up;
      every += r[2];
    }
    a.sums[(int64_t)blockIdx.x * a.M + row] = make_float2(top, total);
    if (a.totals) a.totals[(int64_t)blockIdx.x * a.M + row] = every;
  }
}

template <class T> void run_stream(hipStream_t st, const Logits& l, int blocks) {
  const int waves = ceil_div(l.K, 32 * KS);
  Stream s = {l, ceil_div(l.N, 16)};
  const size_t lds = (size_t)waves * 2048;
  if (l.labels) OSEQ_LAUNCH((stream_logits_kernel<T, false>), dim3(blocks), dim3(waves * 64), lds, st, s);
  else OSEQ_LAUNCH((stream_logits_kernel<T, true>), dim3(blocks), dim3(waves * 64), lds, st, s);
}
// Blocks of the kernel above, eight wavefronts on a CU, or 0 where tiles are taken: rows of little less than 2048 or 4096 values.  A call of 16 rows, the
// weights in no cache, us so / as tiles: 2048 -> 1000 13 / 20, -> 32000 39 / 39, -> 65536 62 / 73, -> 96000 84 / 88, -> 128000 107 / 104, -> 160000 128 / 154; 4096 -> 1000
// 20 / 32, -> 32000 63 / 67, -> 65536 108 / 128, -> 96000 154 / 151, -> 128000 199 / 190, -> 160000 245 / 249: tiles are ahead by 5 % where they fill the card evenly.
// (Weights that the last-level cache still has, 2048 -> 32000: 37 / 27.)  Other widths leave wavefronts without work: 3000 -> 30000 56 / 44, 1024 -> 32000 25 / 20,
// 256 -> 50000 20 / 16.
int stream_blocks(int64_t rows, int classes, int k) {
  const int waves = ceil_div(k, 32 * KS);
  const bool suits = rows <= STREAM_ROWS && (waves == 4 || waves == 8) && k * 10 >= waves * 32 * KS * 9;
  return suits ? std::min(ceil_div(classes, 16), 256 * (8 / waves)) : 0;
}

// ---- a teacher's entries -----------------------------------------------------------------------------------------------
// Those of a row in order of their classes (then of their places), entries of one class added up in the first of them; softmax of their logits, whose
// distance from the row's largest is what is divided by the temperature: the logits themselves may be a type's lowest and largest values; where the entries of each run of `width` classes begin.  Threads N a row, N a power of two of at least `top`.
struct Teacher {
  const int32_t* indices; int64_t ldi;
  const void* logits; int64_t ldt;
  int64_t rows;
  int top, classes, width, columns;
  float per_temperature;
  int32_t* index; float2* target; uint16_t* start; float* flag;
};

// the threads of a row (a wavefront's own accesses to LDS are in order)
template <int N> __device__ __forceinline__ void row_sync() {
  if (N <= 64) asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); else __syncthreads();
}
// thread t ^ o's value: by LDS from another wavefront (all by LDS, with a wait or barrier for each: ten entries of 128 rows 5.9 us, so 4.4)
template <int N, class V> __device__ __forceinline__ V across(V v, V* lds, int t, int o) {
  if (o < 64) return __shfl_xor(v, o);
  lds[t] = v;
  row_sync<N>();
  v = lds[t ^ o];
  row_sync<N>();
  return v;
}
template <int N, class F> __device__ __forceinline__ float over_row(float v, float* lds, int t, F&& f) {
#pragma unroll
  for (int o = N / 2; o > 0; o >>= 1) v = f(v, across<N>(v, lds, t, o));
  return v;
}

template <class S, int N>
__global__ void __launch_bounds__(N < 256 ? 256 : N) teacher_kernel(Teacher a) {
  constexpr int BLOCK = N < 256 ? 256 : N, ROWS = BLOCK / N;
  __shared__ uint32_t keys[ROWS][N];
  __shared__ float values[ROWS][N];
  const int t = threadIdx.x % N, r = threadIdx.x / N;
  const int64_t wanted = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * ROWS + r, row = min(wanted, a.rows - 1);
  int c = -1;
  float v = -__builtin_inff();
  if (t < a.top) {
    c = a.indices[row * a.ldi + t];
    if (c >= 0) v = to_f32(((const S*)a.logits)[row * a.ldt + t]);
  }
  const bool valid = c >= 0 && v != -__builtin_inff(), wrong = valid && (c >= a.classes || !(fabsf(v) <= 3.4028235e38f));
  if (!valid) v = -__builtin_inff();
  auto most_of = [](float p, float q) { return fmaxf(p, q); };
  auto sum_of = [](float p, float q) { return p + q; };
  const float most = over_row<N>(v, values[r], t, most_of);
  const float d = (v - most) * a.per_temperature, e = valid ? __builtin_amdgcn_exp2f(d * LOG2E) : 0.f;
  const float sum = over_row<N>(e, values[r], t, sum_of);
  const float any_wrong = over_row<N>(wrong ? 1.f : 0.f, values[r], t, most_of);
  const float log_q = d - logf(sum);
  uint32_t key = valid && !wrong ? (uint32_t)c << 10 | t : 0xffffffffu;
  // bitonic: pairs of keys at a distance of `o` in runs of `run`
#pragma unroll
  for (int run = 2; run <= N; run *= 2)
#pragma unroll
    for (int o = run / 2; o > 0; o >>= 1) {
      const uint32_t other = across<N>(key, keys[r], t, o);
      const bool least = ((t & o) == 0) == ((t & run) == 0);
      key = least ? min(key, other) : max(key, other);
    }
  keys[r][t] = key;
  values[r][t] = log_q;
  row_sync<N>();
  const bool real = wanted < a.rows;
  if (real && t < a.top && key != 0xffffffffu) {
    const uint32_t mine = key >> 10;
    float q = 0.f, lq = 0.f;
    if (t == 0 || keys[r][t - 1] >> 10 != mine) {  // the first of its class
      lq = values[r][key & 1023];
      q = expf(lq);
      bool alone = true;
      for (int k = t + 1; k < N && keys[r][k] != 0xffffffffu && keys[r][k] >> 10 == mine; ++k, alone = false) q += expf(values[r][keys[r][k] & 1023]);
      if (!alone) lq = logf(q);
    }
    a.index[row * a.top + t] = (int32_t)mine;
    a.target[row * a.top + t] = make_float2(q, lq);
  }
  if (real && t == 0) a.flag[row] = any_wrong != 0.f ? __builtin_nanf("") : most == -__builtin_inff() ? 0.f : 1.f;
  for (int s = t; s <= a.columns; s += N) {
    // entries of lower classes than the run's first
    const uint64_t bound = (uint64_t)s * a.width << 10;
    int lo = 0, hi = N;
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if (keys[r][mid] != 0xffffffffu && (s == a.columns || keys[r][mid] < bound)) lo = mid + 1; else hi = mid;
    }
    if (real) a.start[row * (a.columns + 1) + s] = (uint16_t)lo;
  }
}

// ---- forward: a row's sums joined --------------------------------------------------------------------------------------
struct Join {
  const float2* sums; const float* totals; const float* picked;
  int64_t rows;
  int columns, runs, log_rows;     // of the table of a teacher's entries, of the sums; a block's rows: 1 << log_rows
  const int32_t* labels; int classes;
  float smoothing, z_loss;
  int top; const float2* target; const float* flag; const uint16_t* start;
  float *loss, *lse;
};

// 16 rows a block, or one where there are few.  8192 rows of 1000 runs, 66 MB: 16 us so, 33 with 64 rows for each of 128 blocks
constexpr int JOIN_THREADS = 1024, JOIN_ROWS = 16;
__global__ void __launch_bounds__(JOIN_THREADS) loss_join_kernel(Join a) {
  __shared__ float2 part[JOIN_THREADS];
  __shared__ float more[JOIN_THREADS];
  const int rows = 1 << a.log_rows, rl = threadIdx.x & (rows - 1), slot = threadIdx.x >> a.log_rows, slots = JOIN_THREADS >> a.log_rows;
  const int64_t wanted = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * rows + rl, row = min(wanted, a.rows - 1);
  float most = -__builtin_inff(), sum = 0.f, extra = 0.f;
  auto join = [&](float& m, float& l, float m2, float l2) {
    // (a maximum that is NaN has a sum that is; one of -infinity a sum of zero)
    const float top = fmaxf(m, m2);
    if (top != -__builtin_inff()) l = l * __builtin_amdgcn_exp2f((m - top) * LOG2E) + l2 * __builtin_amdgcn_exp2f((m2 - top) * LOG2E);
    else l += l2;
    m = top;
  };
  // eight runs of columns at a time
  constexpr int AT_ONCE = 8;
  float m4[AT_ONCE], l4[AT_ONCE];
#pragma unroll
  for (int q = 0; q < AT_ONCE; ++q) { m4[q] = -__builtin_inff(); l4[q] = 0.f; }
  for (int c = slot; c < a.runs; c += AT_ONCE * slots) {
    float2 t[AT_ONCE];
#pragma unroll
    for (int q = 0; q < AT_ONCE; ++q) {
      const int at = c + q * slots;
      t[q] = at < a.runs ? a.sums[(int64_t)at * a.rows + row] : make_float2(-__builtin_inff(), 0.f);
      if (a.totals && at < a.runs) extra += a.totals[(int64_t)at * a.rows + row];
    }
#pragma unroll
    for (int q = 0; q < AT_ONCE; ++q) join(m4[q], l4[q], t[q].x, t[q].y);
  }
#pragma unroll
  for (int q = 0; q < AT_ONCE; ++q) join(most, sum, m4[q], l4[q]);
  // a teacher: its entries in turn; q (log q - s), and the sum of q for lse
  float entropy = 0.f, q_all = 0.f;
  const bool teacher = a.labels == nullptr;
  if (teacher) {
    const int n = a.start[row * (a.columns + 1) + a.columns];
    for (int k = slot; k < n; k += slots) {
      const float2 q = a.target[row * a.top + k];
      if (q.x > 0.f) entropy += q.x * (q.y - a.picked[row * a.top + k]);
      q_all += q.x;
    }
  }
  part[threadIdx.x] = make_float2(most, sum);
  more[threadIdx.x] = extra;
  __syncthreads();
  for (int o = slots / 2; o > 0; o >>= 1) {
    if (slot < o) {
      float2 p = part[threadIdx.x];
      const float2 q = part[threadIdx.x + (o << a.log_rows)];
      join(p.x, p.y, q.x, q.y);
      part[threadIdx.x] = p;
      more[threadIdx.x] += more[threadIdx.x + (o << a.log_rows)];
    }
    __syncthreads();
  }
  const float2 all = part[rl];
  const float total = more[rl];
  __syncthreads();
  if (teacher) {
    part[threadIdx.x] = make_float2(entropy, q_all);
    __syncthreads();
    for (int o = slots / 2; o > 0; o >>= 1) {
      if (slot < o) {
        part[threadIdx.x].x += part[threadIdx.x + (o << a.log_rows)].x;
        part[threadIdx.x].y += part[threadIdx.x + (o << a.log_rows)].y;
      }
      __syncthreads();
    }
  }
  if (slot || wanted >= a.rows) return;
  const float lse = all.x + logf(all.y);
  float loss;
  if (teacher) {
    const float flag = a.flag[row];
    loss = flag == 0.f ? 0.f : flag != flag ? flag : part[rl].x + lse * part[rl].y;
  } else {
    // (terms of a factor of zero are none: a logit or lse that is infinite would make NaN of them)
    const int y = a.labels[row];
    loss = y < 0 ? 0.f : y >= a.classes ? __builtin_nanf("") : lse;
    if (y >= 0 && y < a.classes) {
      if (a.smoothing < 1.f) loss -= (1.f - a.smoothing) * a.picked[row];
      if (a.z_loss > 0.f) loss += a.z_loss * lse * lse;
      if (a.totals) loss -= a.smoothing * (total / (float)a.classes);
    }
  }
  a.loss[row] = loss;
  a.lse[row] = lse;
}

// ---- backward: what a row's values are multiplied by ----------------------------------------------------------------------
// A row's dloss / temperature (times f = max(1, 1 + 2 z_loss lse), which keeps the rest within 2) is c m 2^e, c the largest of the rows', m
// in (1/2, 1] and e <= 0.  ds is held as m (p (1 + 2 z_loss lse) - target) / f, and what is left is the factor of dx afterwards and of x in
// dw, where a power of two costs no bits in bf16 and fp32.  (All of it in x would round every value of x a second time.)  In fp16 x has few
// steps below 1, and two planes of ds more than they need: values of 2^-38 keep eleven bits.  So the first 2^11 of a row's 2^e are ds', and x
// begins to lose bits only in rows below that (values of 0.1: with 1e-5 of the largest row's dloss 1.1e-2 of what they add to dw, all of it in x,
// so none).  Where dloss is the same for all rows, a mean's, m is 1, and the value that counts most, -1 at a label that the network does not know, is exact.
// Up to 8192 rows one block (7 us for 4096 rows, 14 for 8192; two launches take a call of 2048 to 8192 rows 1.5 us longer); more rows two launches of
// up to 256 blocks, the largest factors of the blocks first.
struct Rows {
  const float *dloss, *lse, *flag;
  const int32_t* labels;
  int64_t rows;
  int classes;
  float z_loss, per_temperature;
  int in_ds;                    // of a row's 2^e, the powers of two that ds takes
  float4* info; float* scale;
  float* largest; int blocks;   // of the blocks, or null and 1
};
// f(row, whether it is used, whether its target cannot be, lse, factor of p, f, whole factor) for the rows of a block, eight a thread on their way
// at once
template <int THREADS, class F> __device__ __forceinline__ void each_row(const Rows& a, int block, F&& f) {
  const float nan = __builtin_nanf("");
  for (int64_t base = (int64_t)block * 8 * THREADS + threadIdx.x; base < a.rows; base += (int64_t)a.blocks * 8 * THREADS) {
    float target[8], lse[8], g[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t r = min(base + i * THREADS, a.rows - 1);
      if (a.labels) {
        const int y = a.labels[r];
        target[i] = y < 0 ? 0.f : y >= a.classes ? nan : 1.f;
      } else {
        target[i] = a.flag[r];
      }
      lse[i] = a.lse[r];
      g[i] = a.dloss[r];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (base + i * THREADS >= a.rows) break;
      const float p = a.z_loss != 0.f ? 1.f + 2.f * a.z_loss * lse[i] : 1.f, top = fmaxf(1.f, fabsf(p));
      f(base + i * THREADS, target[i] != 0.f, target[i] != target[i], lse[i], p, top, g[i] * a.per_temperature * top);
    }
  }
}
// the largest of a block's values, in every thread
template <int THREADS> __device__ __forceinline__ float block_max(float v, float* part) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) v = fmaxf(v, part[w]);
  return v;
}
template <int THREADS> __device__ __forceinline__ float largest_of(const Rows& a, int block, float* part) {
  float most = 0.f;
  each_row<THREADS>(a, block, [&](int64_t, bool used, bool, float, float, float, float g) {
    if (used && finite(g)) most = fmaxf(most, fabsf(g));
  });
  return block_max<THREADS>(most, part);
}
template <int THREADS> __device__ __forceinline__ void rows_of(const Rows& a, int block, float* part) {
  const float nan = __builtin_nanf("");
  float c = a.largest ? block_max<THREADS>((int)threadIdx.x < a.blocks ? a.largest[threadIdx.x] : 0.f, part) : largest_of<THREADS>(a, 0, part);
  if (c == 0.f) c = 1.f;
  if (block == 0 && threadIdx.x == 0) *a.scale = c;
  each_row<THREADS>(a, block, [&](int64_t r, bool used, bool wrong, float lse, float p, float f, float g) {
    float m = g / c, power = 1.f;
    if (finite(m) && m != 0.f) {
      int e;
      frexpf(m, &e);  // |m| in [2^(e - 1), 2^e)
      if (fabsf(m) == ldexpf(0.5f, e)) --e;
      e = max(e, -120);
      const int held = min(-e, a.in_ds);
      power = ldexpf(1.f, e + held);
      m = ldexpf(m, -e - held);
    }
    a.info[r] = used ? make_float4(lse, wrong ? nan : p / f * m, wrong ? nan : m / f, c * power) : make_float4(0.f, 0.f, 0.f, 0.f);
  });
}
__global__ void __launch_bounds__(1024) rows_kernel(Rows a) {
  __shared__ float part[16];
  rows_of<1024>(a, blockIdx.x, part);
}
__global__ void __launch_bounds__(1024) largest_kernel(Rows a) {
  __shared__ float part[16];
  const float c = largest_of<1024>(a, blockIdx.x, part);
  if (threadIdx.x == 0) a.largest[blockIdx.x] = c;
}
constexpr int ROWS_AT_ONCE = 8192, ROW_BLOCKS = 256;

// sums of 64 rows each
__global__ void __launch_bounds__(256) fold_kernel(const float* sums, int64_t rows, int cols, float* out) {
  const int64_t i = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 256 + threadIdx.x, g = i / cols;
  if (g * 64 >= rows) return;
  const float* p = sums + g * 64 * cols + (i - g * cols);
  const int n = (int)min<int64_t>(64, rows - g * 64);
  float s = 0.f;
  for (int r = 0; r < n; ++r) s += p[(int64_t)r * cols];
  out[i] = s;
}

// What a call begins with, in one launch: operands that are laid out anew, and (the first block, where there is one) the rows' values
struct Prepare { Layout x, w; int x_blocks, w_blocks; Rows rows; int row_blocks; };
template <class S, class T, int PL> __global__ void __launch_bounds__(256) prepare_kernel(Prepare p) {
  __shared__ float part[4];
  int block = blockIdx.x;
  if (block < p.row_blocks) { rows_of<256>(p.rows, 0, part); return; }
  block -= p.row_blocks;
  if (block < p.x_blocks) lay_out_rows<S, T, PL>(p.x, block, p.x_blocks);
  else lay_out_rows<S, T, PL>(p.w, block - p.x_blocks, p.w_blocks);
}
int layout_blocks(int64_t rows, int cols) { return grid_of(rows * ((cols + 7) / 8)); }

template <class S, class T, int W, bool TOP, bool GRAD> void run_logits_w(hipStream_t st, Logits& l) {
  typedef Tile<T, sizeof(S) == 4 ? 3 : 1, W, false, false> G;
  l.tiles_m = ceil_div(l.M, 2 * W);
  l.tiles_n = ceil_div(l.N, 2 * W);
  const int64_t per = ((int64_t)l.tiles_m * l.tiles_n + 7) / 8;
  auto k = logits_kernel<S, T, W, TOP, GRAD>;
  // (more LDS than a launch gets unasked; set again on every launch: which devices know it is not ours to remember)
  if (G::LDS > 65536) (void)hipFuncSetAttribute((const void*)k, hipFuncAttributeMaxDynamicSharedMemorySize, G::LDS);
  OSEQ_LAUNCH(k, grid_of_blocks(per * 8 + l.xs_blocks), dim3(256), G::LDS, st, l);
}
template <class S, class T, bool GRAD> void run_logits(hipStream_t st, Logits& l, int wave) {
  if (l.labels) {
    if (wave == 128) run_logits_w<S, T, 128, false, GRAD>(st, l);
    else if (wave == 64) run_logits_w<S, T, 64, false, GRAD>(st, l);
    else run_logits_w<S, T, 32, false, GRAD>(st, l);
  } else {
    if (wave == 128) run_logits_w<S, T, 128, true, GRAD>(st, l);
    else if (wave == 64) run_logits_w<S, T, 64, true, GRAD>(st, l);
    else run_logits_w<S, T, 32, true, GRAD>(st, l);
  }
}

template <class S> void run_teacher(hipStream_t st, const Teacher& t) {
  if (t.top <= 64) OSEQ_LAUNCH((teacher_kernel<S, 64>), grid_of_blocks((t.rows + 3) / 4), dim3(256), 0, st, t);
  else if (t.top <= 256) OSEQ_LAUNCH((teacher_kernel<S, 256>), grid_of_blocks(t.rows), dim3(256), 0, st, t);
  else OSEQ_LAUNCH((teacher_kernel<S, 1024>), grid_of_blocks(t.rows), dim3(1024), 0, st, t);
}

// The weights of the piece from class `first` on as operands: as they lie, or where they are laid out
template <class S, int PL> void weights_of(const optorch_softmax_loss_t& a, const LossPlan& p, int first, Logits& l) {
  l.w = p.pack_w ? (const void*)((char*)a.workspace + p.off_w) : (const void*)((const S*)a.w + first * a.ldw);
  l.ldw = p.pack_w ? row_of<PL>(a.in_features) : (int)a.ldw;
  l.first = first;
  l.N = std::min(p.piece, a.classes - first);
}
template <class S> Layout weights_anew(const optorch_softmax_loss_t& a, const LossPlan& p, const Logits& l) {
  return {(const S*)a.w + l.first * a.ldw, a.ldw, l.N, a.in_features, (char*)a.workspace + p.off_w, nullptr, nullptr};
}

// What both directions begin with: a teacher's entries in order, the rows' values (backward), operands laid out anew
template <class S, class T, int PL> Logits begin(const optorch_softmax_loss_t& a, const LossPlan& p, Rows* rows) {
  hipStream_t st = (hipStream_t)a.hip_stream;
  char* ws = (char*)a.workspace;
  Logits l = {};
  l.x = p.pack_x ? ws + p.off_x : a.x;
  l.ldx = p.pack_x ? row_of<PL>(a.in_features) : (int)a.ldx;
  l.M = a.rows; l.K = (int)up8(a.in_features);  // (up to the zeros behind a row)
  l.bias = a.bias;
  l.per_temperature = a.labels ? 1.f : 1.f / a.temperature;
  l.labels = a.labels;
  l.columns = p.columns;
  weights_of<S, PL>(a, p, 0, l);
  if (!a.labels) {
    Teacher t = {a.indices, a.ldi, a.teacher, a.ldt, a.rows, a.top, a.classes, p.wave, p.columns, l.per_temperature,
                 (int32_t*)(ws + p.off_index), (float2*)(ws + p.off_target), (uint16_t*)(ws + p.off_start), (float*)(ws + p.off_flag)};
    if (a.teacher_precision == OPTORCH_FP32) run_teacher<float>(st, t);
    else if (a.teacher_precision == OPTORCH_BF16) run_teacher<bf16_t>(st, t);
    else run_teacher<f16_t>(st, t);
    l.top = a.top;
    l.index = t.index; l.target = t.target; l.start = t.start;
  }
  if (rows) {
    *rows = {a.dloss, a.lse, (const float*)(ws + p.off_flag), a.labels, a.rows, a.classes, a.labels ? a.z_loss : 0.f, l.per_temperature,
             a.precision == OPTORCH_FP16 ? 11 : 0, (float4*)(ws + p.off_info), (float*)(ws + p.off_scale), nullptr, 1};
    if (a.rows > ROWS_AT_ONCE) {
      rows->largest = rows->scale + 64;
      rows->blocks = (int)std::min<int64_t>((a.rows + ROWS_AT_ONCE - 1) / ROWS_AT_ONCE, ROW_BLOCKS);
      OSEQ_LAUNCH(largest_kernel, dim3(rows->blocks), dim3(1024), 0, st, *rows);
      OSEQ_LAUNCH(rows_kernel, dim3(rows->blocks), dim3(1024), 0, st, *rows);
    }
  }
  const bool wait = rows && !rows->largest;  // rows whose values are still to be made
  Prepare q = {};
  if (p.pack_x) { q.x = {a.x, a.ldx, a.rows, a.in_features, ws + p.off_x, nullptr, nullptr}; q.x_blocks = layout_blocks(a.rows, a.in_features); }
  if (p.pack_w) { q.w = weights_anew<S>(a, p, l); q.w_blocks = layout_blocks(l.N, a.in_features); }
  if (q.x_blocks + q.w_blocks) {
    if (wait) { q.rows = *rows; q.row_blocks = 1; }
    OSEQ_LAUNCH((prepare_kernel<S, T, PL>), dim3(q.row_blocks + q.x_blocks + q.w_blocks), dim3(256), 0, st, q);
  } else if (wait) {
    OSEQ_LAUNCH(rows_kernel, dim3(1), dim3(1024), 0, st, *rows);
  }
  return l;
}

// f() for each piece, its weights in l
template <class S, class T, int PL, class F> void each_piece(const optorch_softmax_loss_t& a, const LossPlan& p, Logits& l, F&& f) {
  for (int v = 0; v < a.classes; v += p.piece) {
    weights_of<S, PL>(a, p, v, l);
    if (v && p.pack_w) {
      Prepare q = {};
      q.w = weights_anew<S>(a, p, l);
      q.w_blocks = layout_blocks(l.N, a.in_features);
      OSEQ_LAUNCH((prepare_kernel<S, T, PL>), dim3(q.w_blocks), dim3(256), 0, (hipStream_t)a.hip_stream, q);
    }
    f();
  }
}

template <class S, class T, int PL> void forward_of(const optorch_softmax_loss_t& a, const LossPlan& p) {
  hipStream_t st = (hipStream_t)a.hip_stream;
  char* ws = (char*)a.workspace;
  Logits l = begin<S, T, PL>(a, p, nullptr);
  l.sums = (float2*)(ws + p.off_sums);
  l.picked = (float*)(ws + p.off_picked);
  if (a.labels && a.label_smoothing != 0.f) l.totals = (float*)(ws + p.off_totals);
  if (p.stream) {
    if constexpr (PL == 1) run_stream<T>(st, l, p.stream);
  } else if (p.few) {
    l.K = a.in_features;
    run_few<S, T>(st, l);
  } else {
    each_piece<S, T, PL>(a, p, l, [&] { run_logits<S, T, false>(st, l, p.wave); });
  }
  Join j = {};
  j.sums = l.sums; j.totals = l.totals; j.picked = l.picked;
  j.rows = a.rows; j.columns = p.columns; j.runs = p.stream ? p.stream : p.columns;
  // (few rows: a block each)
  while (a.rows > SKINNY_ROWS && (1 << j.log_rows) < JOIN_ROWS) ++j.log_rows;
  j.labels = a.labels; j.classes = a.classes;
  j.smoothing = a.label_smoothing; j.z_loss = a.z_loss;
  j.top = a.top; j.target = l.target; j.start = l.start;
  j.flag = (const float*)(ws + p.off_flag);
  j.loss = a.loss; j.lse = a.lse;
  OSEQ_LAUNCH(loss_join_kernel, grid_of_blocks(ceil_div(a.rows, 1 << j.log_rows)), dim3(JOIN_THREADS), 0, st, j);
}

// rows of sums for dbias from which on they are added up 64 at a time first
constexpr int FOLD_FROM = 2048;

template <class S, class T, int PL> void backward_of(const optorch_softmax_loss_t& a, const LossPlan& p) {
  hipStream_t st = (hipStream_t)a.hip_stream;
  char* ws = (char*)a.workspace;
  Rows rows;
  Logits l = begin<S, T, PL>(a, p, &rows);
  float4* info = rows.info;
  float* scale = rows.scale;
  // (x for dw beside the first piece's tiles, which need nothing of it: 4096 x 2048 -> 100 in fp16 8.5 us less)
  if (a.dw) {
    l.xs = {a.x, a.ldx, a.rows, a.in_features, ws + p.off_xs, info, scale, p.copies > 1};
    l.xs_blocks = std::min(grid_of(a.rows * p.copies * ((a.in_features + 7) / 8)), 1024);
  }
  l.info = info;
  l.spread = a.labels ? a.label_smoothing / (float)a.classes : 0.f;
  l.hit = 1.f - a.label_smoothing;
  l.scale = loss_scale_of(a.precision);
  l.ds = ws + p.off_ds; l.ds_row = p.ds_row;
  l.low = a.rows;
  l.bias_sums = a.dbias ? (float*)(ws + p.off_bias) : nullptr;
  LossPiece g = {};
  g.ds = l.ds; g.ds_row = p.ds_row; g.second = PL == 1 && p.copies == 1 ? a.rows * p.ds_row : 0;
  g.xs = ws + p.off_xs; g.ldxs = row_of<PL>(a.in_features);
  g.info = info; g.scale = scale;
  g.acc = (float*)(ws + p.off_acc); g.parts = (float*)(ws + p.off_parts);
  g.dx = p.dx; g.dw = p.dw;
  g.copies = p.copies; g.both = p.both; g.dx_parts = p.dx_parts;
  each_piece<S, T, PL>(a, p, l, [&] {
    run_logits<S, T, true>(st, l, p.wave);
    l.xs_blocks = 0;
    g.bias_sums = l.bias_sums; g.bias_rows = 2 * l.tiles_m;
    if (a.dbias && g.bias_rows > FOLD_FROM) {
      const int64_t folded = ((int64_t)g.bias_rows + 63) / 64;
      float* out = l.bias_sums + (int64_t)g.bias_rows * l.N;
      OSEQ_LAUNCH(fold_kernel, grid_of_blocks((folded * l.N + 255) / 256), dim3(256), 0, st, (const float*)l.bias_sums, (int64_t)g.bias_rows, l.N, out);
      g.bias_sums = out; g.bias_rows = (int)folded;
    }
    g.w = l.w; g.ldw = l.ldw;
    g.first = l.first; g.count = l.N;
    g.start = l.first == 0; g.end = l.first + l.N == a.classes;
    launch_loss_piece(a, g);
  });
}

template <class S> __global__ void __launch_bounds__(256) loss_clear_kernel(S* p, int64_t rows, int cols, int64_t ld) {
  const int64_t n = rows * cols;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) p[i / cols * ld + i % cols] = from_f32<S>(0.f);
}
template <class S> void clear_of(const optorch_softmax_loss_t& a) {
  hipStream_t st = (hipStream_t)a.hip_stream;
  if (a.dw) OSEQ_LAUNCH(loss_clear_kernel<S>, dim3(grid_of((int64_t)a.classes * a.in_features)), dim3(256), 0, st, (S*)a.dw, (int64_t)a.classes, a.in_features, a.lddw);
  if (a.dbias) OSEQ_LAUNCH(loss_clear_kernel<float>, dim3(grid_of(a.classes)), dim3(256), 0, st, a.dbias, (int64_t)1, a.classes, (int64_t)a.classes);
}

// A piece of ds (and of weights that are laid out anew) takes at most about this; more of it would be faster, and the caller's memory.  In ms with
// 300 / 600 / 1200 MB: 8192 x 4096 -> 128000 in bf16 38.8 / 35.3 / 34.4, 4096 x 2048 -> 65536 4.71 / 4.62 / 4.60, 16384 x 512 -> 32000 3.25 / 3.19 / 2.91,
// 8192 x 1024 -> 50257 4.99 / 4.73 / 4.54; fp32 4096 x 1024 -> 32000 3.92 / 3.70 / 3.67.
constexpr int64_t LOSS_PIECE_BYTES = 600ll << 20;

}  // namespace

// Products of less time together than this are one launch.  The whole call, us as two launches / as one: fp16 128 x 512 -> 1000 27.8 / 23.3,
// 700 x 333 -> 9000 78 / 65; bf16 512 x 1024 -> 8000 76.6 / 73.4, 1000 x 768 -> 20000 208 / 208; fp32 300 x 512 -> 8000 84 / 77.
constexpr float BOTH_US = 60.f;

LossPlan plan_loss(const optorch_softmax_loss_t& a, bool backward) {
  LossPlan p = {};
  const bool f32 = a.precision == OPTORCH_FP32, teacher = a.labels == nullptr;
  const uint64_t in_row = 2 * (uint64_t)(f32 ? row_of<3>(a.in_features) : row_of<1>(a.in_features));
  p.pack_x = f32 || !direct(a.x, a.ldx, a.in_features);
  p.pack_w = f32 || !direct(a.w, a.ldw, a.in_features);
  p.few = !backward && a.rows <= SKINNY_ROWS && p.pack_w;
  if (p.few) p.pack_x = p.pack_w = false;
  if (!backward && !p.pack_x && !p.pack_w && !p.few) p.stream = stream_blocks(a.rows, a.classes, a.in_features);
  // pieces of a multiple of 256 classes, all alike but the last
  int64_t most = a.classes;
  const int64_t each = f32 ? 8 : 4;
  if (backward) most = std::min(most, LOSS_PIECE_BYTES / (each * a.rows));
  if (p.pack_w) most = std::min(most, LOSS_PIECE_BYTES / (int64_t)in_row);
  const int64_t pieces = (a.classes + std::max<int64_t>(256, most) - 1) / std::max<int64_t>(256, most);
  p.piece = pieces == 1 ? a.classes : (int)(((a.classes + pieces - 1) / pieces + 255) / 256 * 256);
  p.wave = p.few || p.stream ? 16 : shape_of(a.rows, p.piece, a.in_features, f32, 1).wave;
  // (a tile's end costs more where ds leaves it than the estimate has: tiles of 256 / 128, us in bf16 4096 x 256 -> 8192 161 / 147, 8192 x
  // 512 -> 4096 238 / 231, 4096 x 1024 -> 32000 1250 / 1289; fp32 414 / 361, 643 / 589, 3708 / 3757)
  if (backward && p.wave == 128 && a.in_features <= 640) p.wave = 64;
  p.columns = (a.classes + p.wave - 1) / p.wave;
  p.ds_row = f32 ? row_of<3>(p.piece) : row_of<1>(p.piece);
  // 16 bits: ds rounded to one plane adds as much as the results' own rounding (dx and dw in bf16 2.3e-3 off, so 1.7e-3; fp16 2.9e-4, 2.1e-4), so
  // it has two, and the products twice as much to do (8192 x 4096 -> 128000 in bf16 20.0 ms with one, 4096 x 256 -> 8192 106 us, so 35.3 and 147).  Few
  // rows: the second plane as further rows of them, which the weights bound.  In us as the second half of the reduction / as rows: bf16
  // 64 x 2048 -> 32000 156 / 131, 16 x 2048 -> 65536 333 / 266, 16 x 512 -> 1000 21 / 21.
  p.copies = backward && !f32 && a.rows <= SKINNY_ROWS ? 2 : 1;
  uint64_t o = 0;
  auto take = [&](uint64_t n) { const uint64_t at = o; o = up256(o + n); return at; };
  const uint64_t rows = a.rows;
  if (p.pack_x) p.off_x = take(rows * in_row);
  if (p.pack_w) p.off_w = take((uint64_t)p.piece * in_row);
  if (teacher) {
    p.off_index = take(rows * a.top * 4);
    p.off_target = take(rows * a.top * 8);
    p.off_start = take(rows * (p.columns + 1) * 2);
    p.off_flag = take(rows * 4);
  }
  if (!backward) {
    const uint64_t runs = p.stream ? p.stream : p.columns;
    p.off_sums = take(rows * runs * 8);
    if (!teacher && a.label_smoothing != 0.f) p.off_totals = take(rows * runs * 4);
    p.off_picked = take(rows * (teacher ? a.top : 1) * 4);
  } else {
    p.off_info = take(rows * 16);
    p.off_scale = take(4 * (64 + ROW_BLOCKS));
    if (a.dw) p.off_xs = take(rows * p.copies * in_row);
    p.off_ds = take(rows * p.ds_row * (f32 ? 2 : 4));
    if (a.dx && p.piece < a.classes) p.off_acc = take(rows * up8(a.in_features) * 4);
    const uint64_t bias_rows = 2 * (uint64_t)ceil_div(a.rows, 2 * p.wave);
    if (a.dbias) p.off_bias = take((bias_rows + (bias_rows > FOLD_FROM ? (bias_rows + 63) / 64 : 0)) * p.piece * 4);
    auto floats = [](const ProductShape& s, int copies, int64_t M, int64_t N) { return s.parts * copies > 1 ? s.parts * M * up8(N) : 0; };
    const int64_t in = a.in_features, rows2 = a.rows * p.copies;
    p.dx = shape_of(rows2, in, p.piece, f32);
    p.dw = shape_of(p.piece, in, rows2, f32);
    // Neither product fills the card: both in one launch, with the tiles that suit the two together best.  (The same ones where only one
    // is asked for: a gradient's bits are the same beside the others and alone.)
    if (p.dx.wave < 128 && p.dw.wave < 128 && p.dx.us + p.dw.us < BOTH_US) {
      p.both = a.dx && a.dw;
      float least = 0.f;
      for (int w : {64, 32}) {
        const ProductShape dx = shape_of(rows2, in, p.piece, f32, 32, w), dw = shape_of(p.piece, in, rows2, f32, 32, w);
        if (least != 0.f && dx.us + dw.us >= least) continue;
        least = dx.us + dw.us;
        p.dx = dx;
        p.dw = dw;
      }
    }
    p.dx_parts = a.dx ? floats(p.dx, p.copies, rows2, in) : 0;
    const int64_t dw_parts = a.dw ? floats(p.dw, 1, p.piece, in) : 0;
    const uint64_t parts = 4 * (uint64_t)(p.both ? p.dx_parts + dw_parts : std::max(p.dx_parts, dw_parts));
    if (parts) p.off_parts = take(parts);
  }
  p.bytes = o;
  return p;
}

void launch_loss_forward(const optorch_softmax_loss_t& a, const LossPlan& p) {
  if (a.precision == OPTORCH_FP32) forward_of<float, bf16_t, 3>(a, p);
  else if (a.precision == OPTORCH_BF16) forward_of<bf16_t, bf16_t, 1>(a, p);
  else forward_of<f16_t, f16_t, 1>(a, p);
}

void launch_loss_backward(const optorch_softmax_loss_t& a, const LossPlan& p) {
  if (a.rows == 0) {
    if (a.precision == OPTORCH_FP32) clear_of<float>(a);
    else if (a.precision == OPTORCH_BF16) clear_of<bf16_t>(a);
    else clear_of<f16_t>(a);
    return;
  }
  if (a.precision == OPTORCH_FP32) backward_of<float, bf16_t, 3>(a, p);
  else if (a.precision == OPTORCH_BF16) backward_of<bf16_t, bf16_t, 1>(a, p);
  else backward_of<f16_t, f16_t, 1>(a, p);
}

}  // namespace oseq
