// The matrix product x w^T with what follows it in its epilogue: bias, activation, scale and residual (wfst_linear), or
// bias, log-softmax and log priors (wfst_loglikes).
#ifndef WFST_LINEAR_H_
#define WFST_LINEAR_H_

#include "wfst_elements.h"

namespace wfst_ops {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

struct LinearArgs {
  const void *x, *w, *bias, *residual;
  void *y;
  int64_t rows, x_stride, w_stride, residual_stride, y_stride;
  int32_t k, n, bias_dtype, out_dtype, activation;
  float scale;
  int32_t tiles_n;               // tiles along n; the grid has tiles_n times the tiles along the rows
};

// p(x) by Horner's rule, coefficients from the constant one on
template <int N> __device__ __forceinline__ float horner(const float (&c)[N], float x) {
  float p = c[N - 1];
#pragma unroll
  for (int i = N - 2; i >= 0; --i) p = __builtin_fmaf(p, x, c[i]);
  return p;
}

// gelu: z / 2 erfc(-z / sqrt 2).  With a = |z|: erfc(a / sqrt 2) = e^(-a^2 / 2) F(a), and F, which falls from 1 like 0.8 / a, is a
// polynomial in t = 1 / (1 + 0.35 a), fitted to the least relative error over a <= 16 (e^-128 is 0 in fp32), so that the lower tail
// has as many digits as the rest.
// FINE, for fp32 results: within 8 (z < 0) and 2.5 (z > 0) times 2^-24 of itself, by an odd polynomial for erf below a = 1 (1 - F e^..
// would lose digits near 0) and the exponent with what its square lost.  Else, for a result that is rounded to 16 bits: within 8e-6, the
// fit 2.2e-6.  A formula within 1.5e-7 of erf itself, which has no digit left at z = -6, measured 2.2 us less at 14,803 x 177 x 333 in fp32
// (29.6, this 31.8) and 20 less at 118,417 x 512 x 2048 in bf16 (352, 372).
template <bool FINE> __device__ __forceinline__ float gelu(float z) {
  const float a = fabsf(z), s = a * a, t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.35f, a, 1.0f));      // (0 for a = inf, and then e^.. is too)
  if (!FINE) {
    constexpr float kF[] = {2.794835269e-01f, 2.748588622e-01f, 2.794893980e-01f, 3.817887977e-02f, 3.908216059e-01f, -3.448736966e-01f, 8.203927428e-02f};
    const float p = horner(kF, t) * t * __builtin_amdgcn_exp2f(s * (-0.5f * kLog2e));
    return 0.5f * z * (z < 0.0f ? p : 2.0f - p);
  }
  constexpr float kErf[] = {7.978845835e-01f, -1.329807192e-01f, 1.994664595e-02f, -2.372659976e-03f, 2.269727411e-04f, -1.530841655e-05f};
  constexpr float kF[] = {-5.743541806e-06f, 2.794096172e-01f, 2.776412368e-01f, 2.542950809e-01f, 1.474193186e-01f,
                          1.310321689e-01f, 1.578007825e-03f, -1.610362828e-01f, 6.988771260e-02f};
  const float p = horner(kF, t) * exp_near(s, __builtin_fmaf(a, a, -s), -0.5f);
  return 0.5f * z * (a < 1.0f ? 1.0f + z * horner(kErf, s) : z < 0.0f ? p : 2.0f - p);
}

// relu, silu and gelu as the header defines them; a NaN stays one.  silu FINE is within 5 times 2^-24 of itself, else within 1.25 |z| 2^-24
// more, where a 16-bit rounding is 2^13 of those.
template <bool FINE> __device__ __forceinline__ float activate(float z, int act) {
  if (act == 1) return z < 0.0f ? 0.0f : z;
  if (act == 2) return FINE ? z / (1.0f + exp_near(-z)) : z * __builtin_amdgcn_rcpf(1.0f + exp_fast(-z));   // (1 / x of the hardware: 1 ulp)
  if (act == 3) return gelu<FINE>(z);
  return z;
}

// 8 values to or from 8 neighbouring elements (a 16-byte access may start at any of them), or the first `count` < 8 one by one
typedef f32x4 f32x4_any __attribute__((aligned(4)));
typedef bf16x8 bf16x8_any __attribute__((aligned(2)));
typedef f16x8 f16x8_any __attribute__((aligned(2)));
__device__ __forceinline__ void load8(const void *p, int64_t i, int dtype, int count, float (&v)[8]) {
  if (count < 8) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < count ? load_as(p, i + e, dtype) : 0.0f;
  } else if (dtype == 0) {
    const f32x4_any *q = reinterpret_cast<const f32x4_any *>(static_cast<const float *>(p) + i);
    const f32x4 lo = q[0], hi = q[1];
#pragma unroll
    for (int e = 0; e < 4; ++e) { v[e] = lo[e]; v[4 + e] = hi[e]; }
  } else if (dtype == 1) {
    const f16x8 h = *reinterpret_cast<const f16x8_any *>(static_cast<const _Float16 *>(p) + i);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (float)h[e];
  } else {
    const bf16x8 h = *reinterpret_cast<const bf16x8_any *>(static_cast<const __bf16 *>(p) + i);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (float)h[e];
  }
}
// (Stored past the caches, as streams: tiles written through them leave in no order, which the memory pays for.  118,417 x 2,048
// results of 16 bits: 409 us for the whole product by way of the caches, 331 past them; never slower, down to the smallest calls.)
__device__ __forceinline__ void store8(void *p, int64_t i, int dtype, int count, const float (&v)[8]) {
  if (count < 8) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < count) store_as(p, i + e, dtype, v[e]);
  } else if (dtype == 0) {
    f32x4_any *q = reinterpret_cast<f32x4_any *>(static_cast<float *>(p) + i);
    __builtin_nontemporal_store(f32x4{v[0], v[1], v[2], v[3]}, q);
    __builtin_nontemporal_store(f32x4{v[4], v[5], v[6], v[7]}, q + 1);
  } else if (dtype == 1) {
    f16x8 h;
#pragma unroll
    for (int e = 0; e < 8; ++e) h[e] = (_Float16)v[e];
    __builtin_nontemporal_store(h, reinterpret_cast<f16x8_any *>(static_cast<_Float16 *>(p) + i));
  } else {
    bf16x8 h;
#pragma unroll
    for (int e = 0; e < 8; ++e) h[e] = (__bf16)v[e];
    __builtin_nontemporal_store(h, reinterpret_cast<bf16x8_any *>(static_cast<__bf16 *>(p) + i));
  }
}

template <bool FINE> __device__ __forceinline__ void activate_all(int activation, float (&v)[8]) {
  if (activation == 1) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = activate<FINE>(v[e], 1);
  } else if (activation == 2) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = activate<FINE>(v[e], 2);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = activate<FINE>(v[e], 3);
  }
}

// what follows the sums v (product and bias) of columns col.. of row m
__device__ __forceinline__ void finish(const LinearArgs &a, int64_t m, int col, float (&v)[8]) {
  const int count = a.n - col;
  if (a.activation) {
    if (a.out_dtype == 0) activate_all<true>(a.activation, v);
    else activate_all<false>(a.activation, v);
  }
  if (a.scale != 1.0f) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] *= a.scale;
  }
  if (a.residual) {
    float r[8];
    load8(a.residual, m * a.residual_stride + col, a.out_dtype, count, r);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += r[e];
  }
  store8(a.y, m * a.y_stride + col, a.out_dtype, count, v);
}

// ---- the product of a tile
//
// A matrix instruction takes 16-byte chunks: a lane holds one chunk (8 elements of 16 bits, 4 of 32) of a row of w and one of a row of
// x, and gets 16 of the 32 x 32 sums.  w is the first operand, so that the sums of a lane are of ONE row of x (lane % 32) and
// of 4 neighbouring columns each (of 8 i + 4 (lane / 32), i = 0..3): results leave 16 bytes at a time, and a softmax
// over the columns stays in the lane but for one exchange with lane ^ 32.
template <class E> struct Mma {                        // 32 bytes of k per step
  static __device__ __forceinline__ f32x16 run(i32x4 w, i32x4 x, f32x16 c);
};
template <> __device__ __forceinline__ f32x16 Mma<BF16>::run(i32x4 w, i32x4 x, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, x), c, 0, 0, 0);
}
template <> __device__ __forceinline__ f32x16 Mma<F16>::run(i32x4 w, i32x4 x, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, w), __builtin_bit_cast(f16x8, x), c, 0, 0, 0);
}
// fp32: the instruction takes one element of k per half wave.  Which one is free, as long as w and x agree: element i of the chunk.
template <> __device__ __forceinline__ f32x16 Mma<F32>::run(i32x4 w, i32x4 x, f32x16 c) {
  const f32x4 a = __builtin_bit_cast(f32x4, w), b = __builtin_bit_cast(f32x4, x);
#pragma unroll
  for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i], b[i], c, 0, 0, 0);
  return c;
}

template <int N> __device__ __forceinline__ void wait_loads() {       // at most N vector loads are still on their way
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | 0x0f70);
}
// all LDS reads of this wave are done, then all waves' are
__device__ __forceinline__ void meet() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xc07f);                                  // lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// A range of memory whose accesses are held against its end; what is behind that is not read.
typedef __amdgpu_buffer_rsrc_t Buffer;
__device__ __forceinline__ Buffer buffer(const void *p, uint32_t bytes) {
  // (word 3 of the descriptor: data format "32 bits", no swizzling)
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), 0, (int)bytes, 0x00020000);
}
// from the first of `rows` rows on to the end of the last one, at most what an offset of 32 bits reaches
__device__ __forceinline__ uint32_t bytes_behind(int64_t rows, int64_t stride, int k, int size) {
  const int64_t n = ((rows - 1) * stride + k) * size;
  return n < 0xfffffff0ll ? (uint32_t)n : 0xfffffff0u;
}

// 16 bytes from byte `off` of a row of k_bytes, zero behind its end
template <class E> __device__ __forceinline__ i32x4 chunk_of(const char *row, int64_t off, int64_t k_bytes) {
  constexpr int kSize = (int)sizeof(typename E::T);
  i32x4 c = {0, 0, 0, 0};
  if (off + 16 <= k_bytes) {
    __builtin_memcpy(&c, __builtin_assume_aligned(row + off, kSize), 16);
  } else if (off < k_bytes) {
    typename E::T e[16 / kSize];
#pragma unroll
    for (int i = 0; i < 16 / kSize; ++i)
      e[i] = off + i * kSize < k_bytes ? reinterpret_cast<const typename E::T *>(row + off)[i] : (typename E::T)0.0f;
    __builtin_memcpy(&c, e, 16);
  }
  return c;
}

// A tile of BM rows of x by GROUPS times BN rows of w, WM x WN of each group per wave.  Its product goes by parts: ROW bytes of k of the
// rows of x and of one group of w, the groups in turn.  LDS holds STAGES parts, chunk c of a row at c ^ swizzle(row): the 16
// lanes that read a column of chunks together are then in different banks.
template <class E, int BM, int BN, int WM, int WN, int ROW, int STAGES = 3, int GROUPS = 1>
struct Tile {
  static constexpr int kWavesM = BM / WM, kWavesN = BN / WN, kWaves = kWavesM * kWavesN, kThreads = 64 * kWaves;
  static constexpr int kChunks = ROW / 16, kSteps = kChunks / 2;
  static constexpr int kStage = (BM + BN) * ROW, kPieces = kStage / 1024;      // 1024 bytes per wave and load
  static constexpr int kLoads = (kPieces + kWaves - 1) / kWaves;
  static constexpr int kTM = WM / 32, kTN = WN / 32;
  static_assert(kStage % 1024 == 0 && BM % (64 / kChunks) == 0 && WM % 32 == 0 && WN % 32 == 0, "whole loads, of x or of w");
  static_assert((ROW == 64 || ROW == 128) && STAGES >= 2 && STAGES <= 4, "an even number of steps; stages as the kernels have them");
  // parts in a row whose stage and group are the same again behind them
  static constexpr int kTurn = STAGES % GROUPS == 0 ? STAGES : GROUPS % STAGES == 0 ? GROUPS : STAGES == 4 && GROUPS == 2 ? 4 : STAGES * GROUPS;
  typedef f32x16 Sums[GROUPS][kTN][kTM];

  static __device__ __forceinline__ int swizzle(int row) { return ROW == 64 ? (row >> 2) & 3 : (row >> 1) & 7; }

  // Piece i of this wave: 1024 bytes of a stage, 64 / kChunks rows of it.  Row r of a part is x's row r for r < BM, row r - BM of the
  // group of w behind that; a piece is of one of them.  (If the waves do not share them out evenly, some load the last piece again.)
  static __device__ __forceinline__ int piece(int i) {
    const int n = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) + kWaves * i;
    return kPieces % kWaves != 0 && n >= kPieces ? kPieces - 1 : n;
  }
  static __device__ __forceinline__ bool piece_of_x(int i) { return piece(i) * (64 / kChunks) < BM; }
  static __device__ __forceinline__ int piece_row(int i) { return piece(i) * (64 / kChunks) + (threadIdx.x & 63) / kChunks; }
  static __device__ __forceinline__ int piece_chunk(int i) { return ((threadIdx.x & 63) % kChunks) ^ swizzle(piece_row(i)); }

  // Where this lane's chunks of the pieces lie behind the start of x or w, in bytes; a group of w behind the one before it.
  int at[kLoads], group_bytes;
  // offset_of(r): of row r of the first group's parts.  A row behind the end may be any other one, or lie out of bounds.
  template <class OffsetOf> __device__ __forceinline__ void aim(OffsetOf offset_of, int bytes) {
    group_bytes = bytes;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) at[i] = offset_of(piece_row(i)) + piece_chunk(i) * 16;
  }
  // Part `k` of k and group `h` on its way into `stage`, without a register between.  Chunks behind the end of a row are whatever
  // lies there, or nothing if that is out of bounds (all of the offset is held against the end): they are put to zero where
  // they are used.
  __device__ __forceinline__ void load(Buffer x, Buffer w, char *stage, int k, int h) const {
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(piece_of_x(i) ? x : w, (__attribute__((address_space(3))) void *)(stage + piece(i) * 1024), 16,
                                               at[i] + (k * ROW + (GROUPS > 1 && !piece_of_x(i) ? h * group_bytes : 0)), 0, 0, 0);
  }

  // What a wave multiplies in one step: 16 bytes of k per lane, half of the wave each of two neighbouring chunks.
  struct Step { i32x4 w[kTN], x[kTM]; };
  static __device__ __forceinline__ void read(Step &f, const char *stage, int step) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, q = 2 * step + (lane >> 5);
    const int m0 = (wave / kWavesN) * WM + (lane & 31), n0 = BM + (wave % kWavesN) * WN + (lane & 31);
#pragma unroll
    for (int i = 0; i < kTN; ++i) f.w[i] = *reinterpret_cast<const i32x4 *>(stage + (n0 + 32 * i) * ROW + (q ^ swizzle(n0 + 32 * i)) * 16);
#pragma unroll
    for (int i = 0; i < kTM; ++i) f.x[i] = *reinterpret_cast<const i32x4 *>(stage + (m0 + 32 * i) * ROW + (q ^ swizzle(m0 + 32 * i)) * 16);
  }
  // acc[n][m] += the step's products.
  static __device__ __forceinline__ void multiply(const Step &f, f32x16 (&acc)[kTN][kTM]) {
#pragma unroll
    for (int i = 0; i < kTN; ++i)
#pragma unroll
      for (int j = 0; j < kTM; ++j) acc[i][j] = Mma<E>::run(f.w[i], f.x[j], acc[i][j]);
  }
  // `left` bytes of k are left at the part's start: what is behind them counts as zero, in x and in w (it may be NaN in either).
  static __device__ __forceinline__ void cut(Step &f, int step, int left) {
    if ((2 * step + ((threadIdx.x & 63) >> 5)) * 16 >= left) {
#pragma unroll
      for (int i = 0; i < kTN; ++i) f.w[i] = i32x4{0, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < kTM; ++i) f.x[i] = i32x4{0, 0, 0, 0};
    }
  }
  // Part I of a turn that begins at part k of k.  The next step's chunks are read while a step is multiplied, across the parts too:
  // before the last step the waves meet; the part behind has arrived then, and nobody reads this one's stage any more, so that
  // the part STAGES further on can come there.
  template <int I, bool LAST>
  __device__ __forceinline__ void part(int k, int k_bytes, Buffer x, Buffer w, char *const (&stage)[STAGES], Step (&f)[2], Sums &acc, unsigned used) {
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      if (s + 1 < kSteps) {
        read(f[(s + 1) & 1], stage[I % STAGES], s + 1);
      } else {
        wait_loads<(STAGES - 2) * kLoads>();
        meet();
        read(f[0], stage[(I + 1) % STAGES], 0);
        __builtin_amdgcn_sched_barrier(0);
        load(x, w, stage[I % STAGES], k + (I + STAGES) / GROUPS, (I + STAGES) % GROUPS);
      }
      __builtin_amdgcn_sched_barrier(0);             // the reads go out before the products that hide them
      if (LAST) cut(f[s & 1], s, k_bytes - (k + I / GROUPS) * ROW);
      if (GROUPS == 1 || (used >> (I % GROUPS) & 1)) multiply(f[s & 1], acc[I % GROUPS]);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  template <int I, bool LAST>
  __device__ __forceinline__ void turn(int k, int parts, int k_bytes, Buffer x, Buffer w, char *const (&stage)[STAGES], Step (&f)[2], Sums &acc, unsigned used) {
    if constexpr (I < kTurn) {
      if (!LAST || k * GROUPS + I < parts * GROUPS) part<I, LAST>(k, k_bytes, x, w, stage, f, acc, used);
      turn<I + 1, LAST>(k, parts, k_bytes, x, w, stage, f, acc, used);
    }
  }
  // The whole product.  Ends with all waves done with LDS.  (STAGES parts behind the last one are loaded too, while the last ones
  // are multiplied, and not used: so every wait has the same number of loads behind it.)  used: a bit per group, whether this
  // wave's sums of it are (uniform).  before, after: what is to be done while the first parts are on their way, before and behind a meeting
  // of the waves; `after` puts the sums to what they begin with.
  template <class Before, class After>
  __device__ __forceinline__ void product(Buffer x, Buffer w, char *const (&stage)[STAGES], int k_bytes, Sums &acc, Before before, After after,
                                          unsigned used = ~0u) {
    static_assert(kTurn % GROUPS == 0 && kTurn % STAGES == 0, "a turn ends where it began");
    constexpr int kStep = kTurn / GROUPS;            // parts of k in a turn
    const int parts = (k_bytes + ROW - 1) / ROW;
    Step f[2];
#pragma unroll
    for (int i = 0; i < STAGES; ++i) load(x, w, stage[i], i / GROUPS, i % GROUPS);
    before();
    wait_loads<(STAGES - 1) * kLoads>();
    meet();
    read(f[0], stage[0], 0);
    after();
    int k = 0;
    for (; k + kStep < parts; k += kStep) turn<0, false>(k, parts, k_bytes, x, w, stage, f, acc, used);
    for (; k < parts; k += kStep) turn<0, true>(k, parts, k_bytes, x, w, stage, f, acc, used);
    wait_loads<0>();
    meet();
  }

  // The same by way of registers, for rows whose chunks are no multiples of 16 bytes in memory (a 16-byte load may start anywhere) or end
  // inside one; what is behind the end of a row is zero.  row_of(r): start of row r of the first group's parts; a row behind the
  // end may be any other one.  rows_w: rows of w from the first group's first one on.
  static __device__ __forceinline__ void fetch(i32x4 (&reg)[kLoads], const char *const (&from)[kLoads], int k, int h, int64_t group, int rows_w, int k_bytes) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const bool there = GROUPS == 1 || piece_of_x(i) || piece_row(i) - BM + h * BN < rows_w;
      const char *p = from[i] + (GROUPS > 1 && !piece_of_x(i) && there ? h * group : 0);
      reg[i] = chunk_of<E>(p, k * ROW + piece_chunk(i) * 16, there ? k_bytes : 0);
    }
  }
  static __device__ __forceinline__ void put(char *stage, const i32x4 (&reg)[kLoads]) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) *reinterpret_cast<i32x4 *>(stage + piece(i) * 1024 + (threadIdx.x & 63) * 16) = reg[i];
  }
  template <class RowOf, class Before, class After>
  static __device__ __forceinline__ void product_staged(RowOf row_of, int64_t group, int rows_w, char *s0, char *s1, int k_bytes, Sums &acc,
                                                        Before before, After after, unsigned used = ~0u) {
    constexpr int kTwo = GROUPS % 2 == 0 ? GROUPS : 2 * GROUPS;                 // parts in a turn of two stages
    const int parts = (k_bytes + ROW - 1) / ROW;
    const char *from[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) from[i] = row_of(piece_row(i));
    i32x4 ahead[2][kLoads];                            // the next two parts, on their way
    fetch(ahead[0], from, 0, 0, group, rows_w, k_bytes);
    fetch(ahead[1], from, 1 / GROUPS, 1 % GROUPS, group, rows_w, k_bytes);
    before();
    put(s0, ahead[0]);
    meet();
    after();
    for (int k = 0; k < parts; k += kTwo / GROUPS) {
#pragma unroll
      for (int i = 0; i < kTwo; ++i) {
        if (k + i / GROUPS >= parts) break;
        fetch(ahead[i & 1], from, k + (i + 2) / GROUPS, (i + 2) % GROUPS, group, rows_w, k_bytes);
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
          Step f;
          read(f, i & 1 ? s1 : s0, s);
          if (GROUPS == 1 || (used >> (i % GROUPS) & 1)) multiply(f, acc[i % GROUPS]);
        }
        put(i & 1 ? s0 : s1, ahead[1 - (i & 1)]);      // nobody reads there since the waves last met
        meet();
      }
    }
  }
};

// Tile `block` of the grid in an order that suits the dies: workgroup b runs on die b % 8, each of which has its own L2, and
// gets neighbouring tiles there, along n first (they share their rows of x, and all of them w).
__device__ __forceinline__ int64_t tile_of(int64_t block, int64_t tiles) {
  const int64_t per = tiles / 8, more = tiles % 8, die = block % 8, i = block / 8;
  return die * per + (die < more ? die : more) + i;
}

// DIRECT: rows of x and w start at multiples of 16 bytes and are whole chunks, and a tile's rows lie within 2 GB
template <class E, int BM, int BN, int WM, int WN, int ROW, int STAGES, bool DIRECT>
__global__ __launch_bounds__(64 * (BM / WM) * (BN / WN), (BM / WM) * (BN / WN) >= 8 ? 4 : (BM / WM) * (BN / WN) >= 4 ? 3 : 1) void linear_kernel(LinearArgs a) {
  using T = Tile<E, BM, BN, WM, WN, ROW, STAGES>;
  constexpr int kPitch = WN + 4;                        // floats; 32 rows of it per wave in the epilogue
  constexpr int kWaveOut = 32 * kPitch * 4, kPer = (T::kWaves + STAGES - 1) / STAGES;      // waves per stage there
  constexpr int kLds = T::kStage > kWaveOut * kPer ? T::kStage : kWaveOut * kPer;
  static_assert(T::kThreads >= BN, "a thread per column");
  __shared__ __align__(16) char s0[kLds], s1[kLds], s2[kLds], s3[STAGES > 3 ? kLds : 16];
  __shared__ __align__(16) float bias[BN];
  const int64_t tile = tile_of(blockIdx.x, gridDim.x);
  const int64_t m0 = tile / a.tiles_n * BM;
  const int n0 = (int)(tile % a.tiles_n) * BN;
  const char *x = static_cast<const char *>(a.x), *w = static_cast<const char *>(a.w);
  constexpr int kSize = (int)sizeof(typename E::T);
  typename T::Sums sums;
  f32x16 (&acc)[T::kTN][T::kTM] = sums[0];
  // The sums begin with the bias, which comes while the first parts do: the epilogue, which nothing hides, is shorter for it.
  const int my = threadIdx.x;
  const float my_bias = a.bias && my < BN && n0 + my < a.n ? load_as(a.bias, n0 + my, a.bias_dtype) : 0.0f;
  const auto before = [&] { if (my < BN) bias[my] = my_bias; };
  const auto after = [&] {
    const int c0 = (threadIdx.x >> 6) % T::kWavesN * WN + 4 * ((threadIdx.x & 63) >> 5);
#pragma unroll
    for (int i = 0; i < T::kTN; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const f32x4 b = *reinterpret_cast<const f32x4 *>(bias + c0 + 32 * i + 8 * q);
#pragma unroll
        for (int j = 0; j < T::kTM; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[i][j][4 * q + e] = b[e];
      }
  };
  const char *xt = x + m0 * a.x_stride * kSize, *wt = w + (int64_t)n0 * a.w_stride * kSize;   // the tile's first rows
  if (DIRECT) {
    T t;
    t.aim([&](int r) { return r < BM ? r * (int)a.x_stride * kSize : (r - BM) * (int)a.w_stride * kSize; }, 0);
    char *const all[4] = {s0, s1, s2, s3};
    char *stage[STAGES];
#pragma unroll
    for (int i = 0; i < STAGES; ++i) stage[i] = all[i];
    t.product(buffer(xt, bytes_behind(a.rows - m0, a.x_stride, a.k, kSize)), buffer(wt, bytes_behind(a.n - n0, a.w_stride, a.k, kSize)), stage,
              a.k * kSize, sums, before, after);
  } else {
    T::product_staged([&](int r) {
      const int64_t m = m0 + r < a.rows ? r : a.rows - 1 - m0, n = n0 + (r - BM) < a.n ? r - BM : a.n - 1 - n0;
      return r < BM ? xt + m * a.x_stride * kSize : wt + n * a.w_stride * kSize;
    }, 0, 0, s0, s1, a.k * kSize, sums, before, after);
  }

  // Epilogue: 32 rows at a time go through the wave's own part of LDS, so that a lane gets 8 neighbouring columns of a row.
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  float *out = reinterpret_cast<float *>((wave / kPer == 0 ? s0 : wave / kPer == 1 ? s1 : wave / kPer == 2 ? s2 : s3) + (wave % kPer) * kWaveOut);
  const int nw = n0 + (wave % T::kWavesN) * WN;
  const int64_t mw = m0 + (wave / T::kWavesN) * WM;
  constexpr int kLanes = WN / 8, kRows = 64 / kLanes;   // lanes per row, rows at a time
  const int col = nw + (lane % kLanes) * 8;
#pragma unroll
  for (int j = 0; j < T::kTM; ++j) {
#pragma unroll
    for (int i = 0; i < T::kTN; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<f32x4 *>(out + (lane & 31) * kPitch + 32 * i + 8 * q + 4 * (lane >> 5)) =
            f32x4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
    for (int r = 0; r < 32; r += kRows) {
      const int64_t m = mw + 32 * j + r + lane / kLanes;
      const float *z = out + (r + lane / kLanes) * kPitch + (lane % kLanes) * 8;
      const f32x4 z0 = *reinterpret_cast<const f32x4 *>(z), z1 = *reinterpret_cast<const f32x4 *>(z + 4);
      float v[8] = {z0[0], z0[1], z0[2], z0[3], z1[0], z1[1], z1[2], z1[3]};
      if (m < a.rows && col < a.n) finish(a, m, col, v);
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// Few rows: 16 rows of x by 16 of w per workgroup of 8 waves, which share out k (16 bytes per lane and step, 64 of a row, from
// memory into registers: nothing is used twice, and all loads of 4 KB of a row are on their way at once) and add their sums up
// through LDS, in the order of the waves.
template <class E> struct MmaFew {                     // 64 bytes of k per step, a quarter of them per 16 lanes
  static __device__ __forceinline__ f32x4 run(i32x4 w, i32x4 x, f32x4 c);
};
template <> __device__ __forceinline__ f32x4 MmaFew<BF16>::run(i32x4 w, i32x4 x, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, x), c, 0, 0, 0);
}
template <> __device__ __forceinline__ f32x4 MmaFew<F16>::run(i32x4 w, i32x4 x, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, w), __builtin_bit_cast(f16x8, x), c, 0, 0, 0);
}
template <> __device__ __forceinline__ f32x4 MmaFew<F32>::run(i32x4 w, i32x4 x, f32x4 c) {
  const f32x4 a = __builtin_bit_cast(f32x4, w), b = __builtin_bit_cast(f32x4, x);
#pragma unroll
  for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
  return c;
}

template <class E>
__global__ __launch_bounds__(512) void linear_few_kernel(LinearArgs a) {
  constexpr int kWaves = 8, kSteps = 8;
  __shared__ __align__(16) float part[kWaves][16][20];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t m0 = (int64_t)(blockIdx.x / a.tiles_n) * 16;
  const int n0 = (int)(blockIdx.x % a.tiles_n) * 16;
  constexpr int kSize = (int)sizeof(typename E::T);
  const int64_t m = m0 + (lane & 15) < a.rows ? m0 + (lane & 15) : a.rows - 1;
  const int64_t n = n0 + (lane & 15) < a.n ? n0 + (lane & 15) : a.n - 1;
  const char *x = static_cast<const char *>(a.x) + m * a.x_stride * kSize, *w = static_cast<const char *>(a.w) + n * a.w_stride * kSize;
  const int64_t k_bytes = (int64_t)a.k * kSize;
  f32x4 acc = {};
  for (int64_t at = wave * 64 + (lane >> 4) * 16; at - (lane >> 4) * 16 < k_bytes; at += kWaves * kSteps * 64) {
    i32x4 xf[kSteps], wf[kSteps];
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      wf[i] = chunk_of<E>(w, at + i * (kWaves * 64), k_bytes);
      xf[i] = chunk_of<E>(x, at + i * (kWaves * 64), k_bytes);
    }
#pragma unroll
    for (int i = 0; i < kSteps; ++i) acc = MmaFew<E>::run(wf[i], xf[i], acc);
  }
  *reinterpret_cast<f32x4 *>(&part[wave][lane & 15][4 * (lane >> 4)]) = acc;       // a lane's 4 sums: columns 4 (lane / 16).. of row lane % 16
  __syncthreads();
  const int r = threadIdx.x >> 1, col = (threadIdx.x & 1) * 8;         // the first 32 threads: 8 columns each
  if (r >= 16 || m0 + r >= a.rows || n0 + col >= a.n) return;
  float v[8] = {}, bias[8];
#pragma unroll
  for (int i = 0; i < kWaves; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += part[i][r][col + e];
#pragma unroll
  for (int e = 0; e < 8; ++e) bias[e] = a.bias && n0 + col + e < a.n ? load_as(a.bias, n0 + col + e, a.bias_dtype) : 0.0f;
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] += bias[e];
  finish(a, m0 + r, n0 + col, v);
}

// ---- wfst_loglikes

struct LoglikesArgs {
  const void *x, *w, *bias;
  const float *log_prior;
  const int32_t *lengths;
  void *out;
  int64_t x_seq_stride, x_stride, w_stride, out_seq_stride, out_stride;
  int32_t seqs, frames, k, v, bias_dtype, out_dtype;
};

// 4 neighbouring results, or the first `count` of them
__device__ __forceinline__ void store4(void *p, int64_t i, int dtype, int count, const float (&v)[4]) {
  if (count < 4) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < count) store_as(p, i + e, dtype, v[e]);
  } else if (dtype == 0) {
    *reinterpret_cast<f32x4_any *>(static_cast<float *>(p) + i) = f32x4{v[0], v[1], v[2], v[3]};
  } else if (dtype == 1) {
    typedef _Float16 four __attribute__((ext_vector_type(4), aligned(2)));
    *reinterpret_cast<four *>(static_cast<_Float16 *>(p) + i) = four{(_Float16)v[0], (_Float16)v[1], (_Float16)v[2], (_Float16)v[3]};
  } else {
    typedef __bf16 four __attribute__((ext_vector_type(4), aligned(2)));
    *reinterpret_cast<four *>(static_cast<__bf16 *>(p) + i) = four{(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
  }
}

// The product with log-softmax behind it: a workgroup has BM whole rows, GROUPS * BN classes wide.  A lane has 16 sums of one row per 32
// classes: the row's maximum and sum are the lane's own, then its neighbour's across the half wave, then, if waves lie side
// by side (kWavesN > 1), theirs through LDS.  The log-probabilities leave from the registers, 4 neighbours at a time: a wave's
// stores together fill whole lines of the L2.
// Tiles differ with the number of classes and of frames; what a frame gets does not: k goes by 32 bytes at a time in every one of
// them, and a row's sum is that of its 32 classes at a time, in their order.
template <class E, int BM, int BN, int WM, int WN, int ROW, int STAGES, int GROUPS, bool DIRECT, int PER_SIMD>
__global__ __launch_bounds__(64 * (BM / WM) * (BN / WN), PER_SIMD) void loglikes_kernel(LoglikesArgs a) {
  using T = Tile<E, BM, BN, WM, WN, ROW, STAGES, GROUPS>;
  constexpr int kSize = (int)sizeof(typename E::T);
  constexpr bool kAlone = T::kWavesN == 1;
  __shared__ __align__(16) char s0[T::kStage], s1[T::kStage], s2[STAGES > 2 ? T::kStage : 16], s3[STAGES > 3 ? T::kStage : 16];
  __shared__ int64_t x_at[BM], out_at[BM];             // where a row's frame is, in bytes behind x, and its results (-1: nowhere)
  __shared__ float row_part[kAlone ? 1 : GROUPS * BN / 32][BM];       // of 32 classes each
  constexpr int kClasses = GROUPS * BN, kMine = (kClasses + T::kThreads - 1) / T::kThreads;
  constexpr int kPacked = 1024;
  static_assert(kClasses * 8 <= T::kStage && (kPacked + 1) * 4 <= T::kStage, "what a stage holds before and behind the product fits");
  float *bias = reinterpret_cast<float *>(s0), *prior = bias + kClasses;      // (there behind the product)
  const unsigned rows = (unsigned)a.seqs * a.frames, m0 = blockIdx.x * BM, frames = a.frames;      // (at most 2^31 - 1 rows)
  // The frames of the tile.  With lengths they are taken from those before them only, one sequence's behind the other's, so that no
  // tile has padding in it (more than kPacked sequences: padding stays among them, and is not written).
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (a.lengths && a.seqs <= kPacked) {
    int *start = reinterpret_cast<int *>(s0);          // of a sequence's frames among all
    for (int i = threadIdx.x; i < a.seqs; i += T::kThreads) {
      const int n = a.lengths[i];
      start[i + 1] = n < 0 ? 0 : n < a.frames ? n : a.frames;
    }
    __syncthreads();
    if (wave == 0) {
      const int each = (a.seqs + 63) / 64, from = lane * each, to = from + each < a.seqs ? from + each : a.seqs;
      int sum = 0;
      for (int i = from; i < to; ++i) sum += start[i + 1];
      int before = sum;
      for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(before, d);
        before += lane >= d ? o : 0;
      }
      before -= sum;
      for (int i = from; i < to; ++i) start[i + 1] = before += start[i + 1];
      if (lane == 0) start[0] = 0;
    }
    __syncthreads();
    const unsigned total = start[a.seqs];
    if (m0 >= total) return;
    for (int r = threadIdx.x; r < BM; r += T::kThreads) {
      const unsigned i = m0 + r < total ? m0 + r : total - 1;
      int s = 0;                                       // the last sequence that starts at i or before it
      for (int d = kPacked; d; d >>= 1)
        if (s + d < a.seqs && (unsigned)start[s + d] <= i) s += d;
      const int t = (int)i - start[s];
      x_at[r] = (s * a.x_seq_stride + t * a.x_stride) * kSize;
      out_at[r] = m0 + r < total ? s * a.out_seq_stride + t * a.out_stride : -1;
    }
  } else {
    bool any = false;
    for (int r = threadIdx.x; r < BM; r += T::kThreads) {
      const unsigned i = m0 + r < rows ? m0 + r : rows - 1;
      const int s = (int)(i / frames), n = a.lengths ? a.lengths[s] : a.frames;
      int t = (int)(i % frames);
      const bool there = m0 + r < rows && t < n;
      out_at[r] = there ? s * a.out_seq_stride + t * a.out_stride : -1;
      if (t >= n) t = n > 0 ? n - 1 : 0;               // (not used: the sequence's last frame before the length stands in)
      x_at[r] = (s * a.x_seq_stride + t * a.x_stride) * kSize;
      any |= there;
    }
    if (!__syncthreads_or(any)) return;
  }
  __syncthreads();
  const char *x = static_cast<const char *>(a.x), *w = static_cast<const char *>(a.w);
  auto w_offset = [&](int r) { return (int64_t)(r - BM < a.v ? r - BM : a.v - 1) * a.w_stride * kSize; };
  const int wm = wave / T::kWavesN, wn = wave % T::kWavesN;
  unsigned used = 0;                                   // groups in which this wave has classes before v
#pragma unroll
  for (int h = 0; h < GROUPS; ++h) used |= h * BN + wn * WN < a.v ? 1u << h : 0;
  used = __builtin_amdgcn_readfirstlane(used);
  float my_bias[kMine], my_prior[kMine];               // on their way while the product is taken
#pragma unroll
  for (int i = 0; i < kMine; ++i) {
    const int c = threadIdx.x + i * T::kThreads;
    my_bias[i] = a.bias && c < a.v ? load_as(a.bias, c, a.bias_dtype) : 0.0f;
    my_prior[i] = a.log_prior && c < a.v ? a.log_prior[c] : 0.0f;
  }
  typename T::Sums acc;
  const auto nothing = [] {};
  const auto zero = [&] {
#pragma unroll
    for (int h = 0; h < GROUPS; ++h)
#pragma unroll
      for (int i = 0; i < T::kTN; ++i)
#pragma unroll
        for (int j = 0; j < T::kTM; ++j) acc[h][i][j] = f32x16{};
  };
  if (DIRECT) {
    T t;
    t.aim([&](int r) { return (int)(r < BM ? x_at[r] : w_offset(r)); }, BN * (int)a.w_stride * kSize);
    const int64_t x_end = (int64_t)(a.seqs - 1) * a.x_seq_stride + (int64_t)(a.frames - 1) * a.x_stride + a.k;      // (within 2 GB here)
    char *const all[4] = {s0, s1, s2, s3};
    char *stage[STAGES];
#pragma unroll
    for (int i = 0; i < STAGES; ++i) stage[i] = all[i];
    t.product(buffer(x, (uint32_t)(x_end * kSize)), buffer(w, bytes_behind(a.v, a.w_stride, a.k, kSize)), stage, a.k * kSize, acc, nothing, zero, used);
  } else {
    T::product_staged([&](int r) { return r < BM ? x + x_at[r] : w + w_offset(r); }, BN * a.w_stride * kSize, a.v, s0, s1, a.k * kSize, acc, nothing, zero, used);
  }

#pragma unroll
  for (int i = 0; i < kMine; ++i) {
    const int c = threadIdx.x + i * T::kThreads;
    if (c < kClasses) { bias[c] = my_bias[i]; prior[c] = my_prior[i]; }
  }
  __syncthreads();
  // sums -> z = sum + bias; classes behind v count as -inf
  float m[T::kTM], ls[T::kTM];
#pragma unroll
  for (int j = 0; j < T::kTM; ++j) m[j] = -__builtin_inff();
#pragma unroll
  for (int h = 0; h < GROUPS; ++h)
#pragma unroll
    for (int i = 0; i < T::kTN; ++i) {
      const int c0 = h * BN + wn * WN + 32 * i + 4 * (lane >> 5);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const f32x4 b = *reinterpret_cast<const f32x4 *>(bias + c0 + 8 * q);
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int j = 0; j < T::kTM; ++j) acc[h][i][j][4 * q + e] += b[e];
      }
      if (h * BN + wn * WN + 32 * i + 32 > a.v) {
#pragma unroll
        for (int q = 0; q < 16; ++q)
#pragma unroll
          for (int j = 0; j < T::kTM; ++j) acc[h][i][j][q] = c0 + 8 * (q / 4) + q % 4 < a.v ? acc[h][i][j][q] : -__builtin_inff();
      }
#pragma unroll
      for (int j = 0; j < T::kTM; ++j)
#pragma unroll
        for (int q = 0; q < 16; ++q) m[j] = fmaxf(m[j], acc[h][i][j][q]);
    }
  // the rows' maxima
#pragma unroll
  for (int j = 0; j < T::kTM; ++j) {
    m[j] = fmaxf(m[j], __shfl_xor(m[j], 32));
    if (!kAlone && lane < 32) row_part[wn][wm * WM + 32 * j + lane] = m[j];
  }
  if (!kAlone) {
    __syncthreads();
#pragma unroll
    for (int j = 0; j < T::kTM; ++j)
#pragma unroll
      for (int n = 0; n < T::kWavesN; ++n) m[j] = fmaxf(m[j], row_part[n][wm * WM + 32 * j + (lane & 31)]);
    __syncthreads();
  }
  // sums of e^(z - m).  (Of -inf alone: -inf - -inf is NaN, as documented; a NaN or +inf becomes one here as well.)
#pragma unroll
  for (int j = 0; j < T::kTM; ++j) {
    ls[j] = 0.0f;
#pragma unroll
    for (int h = 0; h < GROUPS; ++h)
#pragma unroll
      for (int i = 0; i < T::kTN; ++i) {
        float part = 0.0f;
#pragma unroll
        for (int q = 0; q < 16; ++q) {
          acc[h][i][j][q] -= m[j];
          part += exp_fast(acc[h][i][j][q]);
        }
        part += __shfl_xor(part, 32);
        ls[j] += part;
        if (!kAlone && lane < 32) row_part[h * (BN / 32) + wn * T::kTN + i][wm * WM + 32 * j + lane] = part;
      }
  }
  if (!kAlone) {
    __syncthreads();
    const int parts = (a.v - 1) / 32 + 1;
#pragma unroll
    for (int j = 0; j < T::kTM; ++j) ls[j] = 0.0f;
#pragma unroll 8
    for (int n = 0; n < parts; ++n)
#pragma unroll
      for (int j = 0; j < T::kTM; ++j) ls[j] += row_part[n][wm * WM + 32 * j + (lane & 31)];
  }
#pragma unroll
  for (int j = 0; j < T::kTM; ++j) {
    const float log_sum = logf(ls[j]);
    const int64_t to = out_at[wm * WM + 32 * j + (lane & 31)];
    if (to < 0) continue;
#pragma unroll
    for (int h = 0; h < GROUPS; ++h)
#pragma unroll
      for (int i = 0; i < T::kTN; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int c = h * BN + wn * WN + 32 * i + 8 * q + 4 * (lane >> 5);
          if (c >= a.v) continue;
          float l[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) l[e] = acc[h][i][j][4 * q + e] - log_sum;
          if (a.log_prior) {
            const f32x4 off = *reinterpret_cast<const f32x4 *>(prior + c);
#pragma unroll
            for (int e = 0; e < 4; ++e) l[e] -= off[e];
          }
          store4(a.out, to + c, a.out_dtype, a.v - c, l);
        }
  }
}

}  // namespace wfst_ops

#endif  // WFST_LINEAR_H_
