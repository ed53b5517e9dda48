// Log-probabilities of given tokens, entropy and top alternatives of rows of scores, and their gradient.
//
// With m a row's maximum and d = x - m: S = sum e^d, lse = m + ln S, log p = d - ln S, entropy = ln S - (sum e^d d) / S.  All four
// come out of one reading of the row.  Every sum has a fixed order: lanes, then waves, then parts of a row.
#ifndef WFST_LOGPROBS_H_
#define WFST_LOGPROBS_H_

#include "wfst_elements.h"

namespace wfst_ops {

struct LogprobsArgs {
  const void *scores;
  const int32_t *tokens, *lengths;
  float *logprobs, *lse, *entropy, *maximum, *log_sum;
  int32_t *top_ids;
  float *top_logprobs;
  void *workspace;
  int64_t seq_stride, stride;
  int32_t seqs, frames, v, given, top;
  int32_t splits, split_size;                          // long rows: parts of a row, elements of a part
};

struct BackwardArgs {
  const void *scores;
  const int32_t *tokens, *lengths;
  const float *maximum, *log_sum, *entropy;
  const int32_t *top_ids;
  const float *grad_logprobs, *grad_lse, *grad_entropy, *grad_top;
  void *grad_scores;
  int64_t seq_stride, stride, grad_seq_stride, grad_stride;
  int32_t seqs, frames, v, given, top;
  int32_t splits;                                      // long rows: workgroups per row
};

constexpr int kMaxGiven = 256, kMaxTop = 64;
constexpr int kShortRow = 2048;                        // rows of up to so many scores are held in registers

// A float as a whole number that orders alike: -0 and +0 are one, every NaN is above +inf.  Never kNothing.
constexpr int kNothing = INT32_MIN;
__device__ __forceinline__ int order_of(float x) {
  const int b = __float_as_int(x + 0.0f), o = b < 0 ? b ^ 0x7fffffff : b;
  return x != x ? 0x7fffffff : o;
}
__device__ __forceinline__ float float_of(int order) { return __int_as_float(order < 0 ? order ^ 0x7fffffff : order); }
// (order, lower index first) as one number; 0 is below all of them
__device__ __forceinline__ unsigned long long key_of(int order, int j) {
  return ((unsigned long long)((unsigned)order ^ 0x80000000u) << 32) | (unsigned)~j;
}
__device__ __forceinline__ int index_of(unsigned long long key) { return (int)~(unsigned)key; }
__device__ __forceinline__ float score_of(unsigned long long key) { return float_of((int)((unsigned)(key >> 32) ^ 0x80000000u)); }

__device__ __forceinline__ float neg_inf() { return -__builtin_inff(); }

// A row that rules everything out.  (The maximum passes over a NaN, the sum does not.)
__device__ __forceinline__ bool is_empty(float m, float ls) { return m == neg_inf() && ls == neg_inf(); }
// log-probability of a score in a row with this maximum and log of the sum behind it: in an empty row it is -inf
__device__ __forceinline__ float logprob_of(float x, float m, float ls) { return is_empty(m, ls) ? m : (x - m) - ls; }

// e^d d, 0 for d = -inf (e^d is 0 then, so that any finite d does); a NaN stays one through e^d
__device__ __forceinline__ float weighted(float e, float d) { return e * fmaxf(d, -1e4f); }

// ---- reductions over the 16 lanes of a row of the wave (rotations by 8, 4, 2, 1), or over all 64: every lane gets the result
template <int CTRL> __device__ __forceinline__ float turned(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
template <int CTRL> __device__ __forceinline__ int turned(int v) { return __builtin_amdgcn_update_dpp(0, v, CTRL, 0xf, 0xf, true); }
template <int LANES, class V, class Op> __device__ __forceinline__ V reduce(V v, Op op) {
  v = op(v, turned<0x128>(v));
  v = op(v, turned<0x124>(v));
  v = op(v, turned<0x122>(v));
  v = op(v, turned<0x121>(v));
  if (LANES == 64) {
    v = op(v, __shfl_xor(v, 16));
    v = op(v, __shfl_xor(v, 32));
  }
  return v;
}
template <int LANES> __device__ __forceinline__ float max_over(float v) { return reduce<LANES>(v, [](float a, float b) { return fmaxf(a, b); }); }
template <int LANES> __device__ __forceinline__ float sum_over(float v) { return reduce<LANES>(v, [](float a, float b) { return a + b; }); }
template <int LANES> __device__ __forceinline__ int max_over(int v) { return reduce<LANES>(v, [](int a, int b) { return a > b ? a : b; }); }
template <int LANES> __device__ __forceinline__ int min_over(int v) { return reduce<LANES>(v, [](int a, int b) { return a < b ? a : b; }); }

// what a row's own results are; one lane writes them
__device__ __forceinline__ void write_row(const LogprobsArgs &a, int64_t row, float m, float sum, float weighted_sum, float ls) {
  if (a.lse) a.lse[row] = m + ls;
  if (a.maximum) a.maximum[row] = m;
  if (a.log_sum) a.log_sum[row] = ls;
  if (a.entropy) a.entropy[row] = is_empty(m, ls) ? 0.0f : ls - weighted_sum / sum;
}
template <class E>
__device__ __forceinline__ float given_logprob(const typename E::T *x, int v, int token, float m, float ls) {
  if (token == -1) return 0.0f;
  if (token < 0 || token >= v) return __builtin_nanf("");
  return logprob_of(E::get(x[token]), m, ls);
}

// How many of n keys are above k (n reads in flight, not one after the other)
__device__ __forceinline__ int place_of(unsigned long long k, const unsigned long long *keys, int n) {
  int place = 0, f = 0;
  for (; f + 8 <= n; f += 8)
#pragma unroll
    for (int i = 0; i < 8; ++i) place += keys[f + i] > k;
  for (; f < n; ++f) place += keys[f] > k;
  return place;
}

// Between a wave's writes to LDS and its reads of them: they are carried out in order, the compiler has to leave them so.
__device__ __forceinline__ void in_order() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// ---- rows of up to 2,048 scores: LANES lanes hold a row, EACH scores per lane, in registers.  16 lanes for up to 256: a reduction
// then stays within the rotations, and serves four rows.
template <class E, int LANES, int EACH, bool MANY>
__global__ __launch_bounds__(256) void logprobs_short_kernel(LogprobsArgs a) {
  const int lane = threadIdx.x % LANES;
  const unsigned row = blockIdx.x * (256 / LANES) + threadIdx.x / LANES, rows = (unsigned)a.seqs * a.frames;
  const unsigned s = row / (unsigned)a.frames, t = row % (unsigned)a.frames;
  // (lanes without a row go along with the others as far as they exchange values; they have no scores and write nothing)
  const bool live = row < rows && (!a.lengths || (int)t < a.lengths[s]);
  const typename E::T *x = static_cast<const typename E::T *>(a.scores) + (live ? s * a.seq_stride + t * a.stride : 0);
  float z[EACH];
#pragma unroll
  for (int e = 0; e < EACH; ++e) z[e] = live && lane + LANES * e < a.v ? E::get(x[lane + LANES * e]) : neg_inf();
  float m = neg_inf();
#pragma unroll
  for (int e = 0; e < EACH; ++e) m = fmaxf(m, z[e]);
  m = max_over<LANES>(m);
  const float base = m == neg_inf() ? 0.0f : m;
  float sum = 0.0f, wsum = 0.0f;
#pragma unroll
  for (int e = 0; e < EACH; ++e) {
    const float d = z[e] - base, p = exp_fast(d);
    sum += p;
    wsum += weighted(p, d);
  }
  sum = sum_over<LANES>(sum);
  wsum = sum_over<LANES>(wsum);
  const float ls = logf(sum);
  if (live) {
    if (lane == 0) write_row(a, row, m, sum, wsum, ls);
    if (a.logprobs)
      for (int g = lane; g < a.given; g += LANES)
        a.logprobs[(int64_t)row * a.given + g] = given_logprob<E>(x, a.v, a.tokens[(int64_t)row * a.given + g], m, ls);
  }
  if (a.top == 0) return;
  int order[EACH];
#pragma unroll
  for (int e = 0; e < EACH; ++e) order[e] = live && lane + LANES * e < a.v ? order_of(z[e]) : kNothing;
  if constexpr (MANY) {
    // The top-th largest of the lanes' maxima is a bound that as many scores reach; what reaches it is listed and finds its place there.
    constexpr int kList = LANES == 64 ? 128 : 64;
    __shared__ __align__(16) int maxima[256 / LANES][LANES];
    __shared__ unsigned long long list[256 / LANES][kList];
    __shared__ int bounds[256 / LANES];
    const int group = threadIdx.x / LANES;
    int own = order[0], rank = 0, mine = 0;
#pragma unroll
    for (int e = 1; e < EACH; ++e) own = order[e] > own ? order[e] : own;
    maxima[group][lane] = own;
    in_order();
#pragma unroll
    for (int i = 0; i < LANES; i += 4) {
      const int4 o = *reinterpret_cast<const int4 *>(&maxima[group][i]);
      rank += (o.x > own || (o.x == own && i < lane)) + (o.y > own || (o.y == own && i + 1 < lane)) + (o.z > own || (o.z == own && i + 2 < lane)) +
              (o.w > own || (o.w == own && i + 3 < lane));
    }
    if (rank == a.top - 1) bounds[group] = own;
    in_order();
    const int bound = bounds[group] > kNothing ? bounds[group] : kNothing + 1;
#pragma unroll
    for (int e = 0; e < EACH; ++e) mine += order[e] >= bound;
    int to = mine;                                     // the lanes' lists lie one behind the other
    for (int d = 1; d < LANES; d <<= 1) {
      const int o = __shfl_up(to, d, LANES);
      to += lane >= d ? o : 0;
    }
    const int total = __shfl(to, LANES - 1, LANES);
    to -= mine;
    if (!__any(total > kList)) {                       // (else too many are equal)
#pragma unroll
      for (int e = 0; e < EACH; ++e)
        if (order[e] >= bound) list[group][to++] = key_of(order[e], lane + LANES * e);
      in_order();
      for (int i = lane; i < total && live; i += LANES) {
        const unsigned long long key = list[group][i];
        const int place = place_of(key, list[group], total);
        if (place >= a.top) continue;
        if (a.top_ids) a.top_ids[(int64_t)row * a.top + place] = index_of(key);
        if (a.top_logprobs) a.top_logprobs[(int64_t)row * a.top + place] = logprob_of(score_of(key), m, ls);
      }
      return;
    }
  }
  // One after the other: every lane's best, the best of them, and its lane goes on to its next one.
  for (int i = 0; i < a.top; ++i) {
    int best = order[0], at = 0;
#pragma unroll
    for (int e = 1; e < EACH; ++e) {                   // (of equal ones the lower index)
      at = order[e] > best ? e : at;
      best = order[e] > best ? order[e] : best;
    }
    const int top = max_over<LANES>(best);
    const int j = min_over<LANES>(best == top ? lane + LANES * at : INT32_MAX);
#pragma unroll
    for (int e = 0; e < EACH; ++e) order[e] = j == lane + LANES * e ? kNothing : order[e];
    if (live && lane == 0) {
      if (a.top_ids) a.top_ids[(int64_t)row * a.top + i] = j;
      if (a.top_logprobs) a.top_logprobs[(int64_t)row * a.top + i] = logprob_of(float_of(top), m, ls);
    }
  }
}

// ---- longer rows: a workgroup per part of a row
//
// A lane takes 16 bytes at a time, keeps the maximum of what it has seen, and scales its sums when that grows.  The top ones need
// no list on the way: the k-th largest of the lanes' maxima (of four lanes together up to k = 32) is a bound that at least k scores reach,
// and what reaches it lies with the lanes whose own maximum does.  Those, little more than k of 256 unless scores are equal, are
// read again and what reaches the bound is sorted.  Where more reach it than the list holds (a mask that leaves few scores, or equal ones), what is
// above it is listed and the first equal ones are taken in one more reading.  Only rows with a NaN, or with more than the list holds above
// the bound, have their top ones searched one after the other.
constexpr int kLongThreads = 256, kLongLoads = 4, kFound = 1024;

template <class E> struct Chunk {                       // 16 bytes of scores, from any address
  static constexpr int kN = 16 / (int)sizeof(typename E::T);
  typedef typename E::T Vec __attribute__((ext_vector_type(16 / sizeof(typename E::T))));
  typedef Vec Any __attribute__((aligned(sizeof(typename E::T))));
  static __device__ __forceinline__ Vec load(const typename E::T *p) { return *reinterpret_cast<const Any *>(p); }
  static __device__ __forceinline__ void store(typename E::T *p, Vec v) { *reinterpret_cast<Any *>(p) = v; }
};

struct Sums { float m, sum, wsum; };                    // maximum, sum of e^(x - m), sum of e^(x - m) (x - m)

// the sums of two parts as one; a part without scores has m = -inf and sums of 0
__device__ __forceinline__ Sums join(Sums p, Sums q) {
  const float m = fmaxf(p.m, q.m), base = m == neg_inf() ? 0.0f : m;
  const float dp = p.m - base, dq = q.m - base, ep = exp_fast(dp), eq = exp_fast(dq);
  Sums r;
  r.m = m;
  r.sum = ep * p.sum + eq * q.sum;
  r.wsum = ep * (p.wsum + fmaxf(dp, -1e4f) * p.sum) + eq * (q.wsum + fmaxf(dq, -1e4f) * q.sum);
  return r;
}

template <class E> __device__ __forceinline__ float chunk_max(typename Chunk<E>::Vec c) {
  float m = E::get(c[0]);
#pragma unroll
  for (int i = 1; i < Chunk<E>::kN; ++i) m = fmaxf(m, E::get(c[i]));
  return m;
}
template <class E> __device__ __forceinline__ void add_chunk(Sums &s, typename Chunk<E>::Vec c, float base) {
#pragma unroll
  for (int i = 0; i < Chunk<E>::kN; ++i) {
    const float d = E::get(c[i]) - base, e = exp_fast(d);
    s.sum += e;
    s.wsum += weighted(e, d);
  }
}
// the maximum grows to m
__device__ __forceinline__ float grow(Sums &s, float m) {
  const float base = m == neg_inf() ? 0.0f : m, d = s.m - base, e = exp_fast(d);
  s.wsum = e * (s.wsum + fmaxf(d, -1e4f) * s.sum);
  s.sum *= e;
  s.m = m;
  return base;
}

// A part of a row as it is left for the kernel that joins them: sums, then `top` keys, falling.
struct Part { Sums s; float pad; };
__device__ __forceinline__ int64_t part_bytes(int top) { return 16 + 8 * (int64_t)top; }

// What is left of a row once its sums are known, by all threads of a workgroup.  keys: its top ones, falling.
template <class E>
__device__ __forceinline__ void finish_row(const LogprobsArgs &a, int64_t row, const typename E::T *x, Sums s, const unsigned long long *keys) {
  const float ls = logf(s.sum);
  if (threadIdx.x == 0) write_row(a, row, s.m, s.sum, s.wsum, ls);
  if (a.logprobs)
    for (int g = threadIdx.x; g < a.given; g += blockDim.x)
      a.logprobs[row * a.given + g] = given_logprob<E>(x, a.v, a.tokens[row * a.given + g], s.m, ls);
  for (int i = threadIdx.x; i < a.top; i += blockDim.x) {
    if (a.top_ids) a.top_ids[row * a.top + i] = index_of(keys[i]);
    if (a.top_logprobs) a.top_logprobs[row * a.top + i] = logprob_of(score_of(keys[i]), s.m, ls);
  }
}

template <class E>
__global__ __launch_bounds__(kLongThreads) void logprobs_long_kernel(LogprobsArgs a) {
  using C = Chunk<E>;
  constexpr int kWaves = kLongThreads / 64, kStep = kLongThreads * C::kN;       // elements that the workgroup loads at a time
  __shared__ Sums waves[kWaves];
  __shared__ __align__(16) int maxima[kLongThreads];
  __shared__ int picked[kLongThreads], n_picked, n_found, bound_;
  __shared__ unsigned long long found[kFound], keys[kMaxTop], best[kWaves];
  const unsigned row = blockIdx.x / (unsigned)a.splits, split = blockIdx.x % (unsigned)a.splits;
  const unsigned s = row / (unsigned)a.frames, t = row % (unsigned)a.frames;
  if (a.lengths && (int)t >= a.lengths[s]) return;
  const typename E::T *x = static_cast<const typename E::T *>(a.scores) + s * a.seq_stride + t * a.stride;
  const int lo = split * a.split_size, hi = a.v - lo < a.split_size ? a.v : lo + a.split_size;
  const int tid = threadIdx.x, mine = lo + tid * C::kN;        // this lane's first chunk; the next ones are kStep apart
  Sums q = {neg_inf(), 0.0f, 0.0f};
  int64_t j = mine;
  for (; lo + (j - mine) + (int64_t)kStep * kLongLoads <= hi; j += kStep * kLongLoads) {
    typename C::Vec c[kLongLoads];
#pragma unroll
    for (int i = 0; i < kLongLoads; ++i) c[i] = C::load(x + j + i * kStep);
    float m = q.m;
#pragma unroll
    for (int i = 0; i < kLongLoads; ++i) m = fmaxf(m, chunk_max<E>(c[i]));
    const float base = grow(q, m);
#pragma unroll
    for (int i = 0; i < kLongLoads; ++i) add_chunk<E>(q, c[i], base);
  }
  for (; j < hi; j += kStep) {                                  // the rest, whose last chunk may be cut
    typename C::Vec c;
    if (j + C::kN <= hi) {
      c = C::load(x + j);
    } else {
#pragma unroll
      for (int i = 0; i < C::kN; ++i) c[i] = j + i < hi ? x[j + i] : (typename E::T)neg_inf();
    }
    const float base = grow(q, fmaxf(q.m, chunk_max<E>(c)));
    add_chunk<E>(q, c, base);
  }
  const int own = mine < hi ? order_of(q.m) : kNothing;
  const bool fours = a.top <= 32;
  if (fours) {
    int o = turned<0xb1>(own);                                  // of the lane beside, then of the two beside
    o = o > own ? o : own;
    const int p = turned<0x4e>(o);
    if (tid % 4 == 0) maxima[tid / 4] = p > o ? p : o;
  } else {
    maxima[tid] = own;
  }
  if (tid == 0) n_picked = n_found = 0;

  // the workgroup's sums: lanes, then waves
  const float m = max_over<64>(q.m);
  grow(q, m);
  q.sum = sum_over<64>(q.sum);
  q.wsum = sum_over<64>(q.wsum);
  if (tid % 64 == 0) waves[tid / 64] = q;
  __syncthreads();
  q = waves[0];
#pragma unroll
  for (int i = 1; i < kWaves; ++i) q = join(q, waves[i]);

  if (a.top) {
    bool slow = q.sum != q.sum;                                 // a NaN (or +inf): maxima pass over it
    const int n = a.top < hi - lo ? a.top : hi - lo;            // (a row's last part may be shorter)
    if (!slow) {
      // the bound: the n-th largest of the maxima (the lower one breaks ties)
      const int many = fours ? kLongThreads / 4 : kLongThreads;
      if (tid < many) {
        const int mine_ = maxima[tid];
        int rank = 0;
#pragma unroll 4
        for (int i = 0; i < many; i += 4) {
          const int4 o = *reinterpret_cast<const int4 *>(maxima + i);
          rank += (o.x > mine_ || (o.x == mine_ && i < tid)) + (o.y > mine_ || (o.y == mine_ && i + 1 < tid)) +
                  (o.z > mine_ || (o.z == mine_ && i + 2 < tid)) + (o.w > mine_ || (o.w == mine_ && i + 3 < tid));
        }
        if (rank == n - 1) bound_ = mine_;
      }
      __syncthreads();
      const int bound = bound_;
      if (own >= bound && own != kNothing) picked[atomicAdd(&n_picked, 1)] = tid;
      __syncthreads();
      // the picked lanes' chunks again, all threads: scores of an order above `above`
      const auto collect = [&](int above) {
        const int chunks = (hi - lo - 1) / kStep + 1;           // of a lane, at most
        for (int64_t i = tid; i < (int64_t)n_picked * chunks; i += kLongThreads) {
          const int64_t at = lo + picked[i / chunks] * C::kN + (i % chunks) * kStep;
          typename C::Vec c;
          if (at + C::kN <= hi) {
            c = C::load(x + at);
          } else {
#pragma unroll
            for (int e = 0; e < C::kN; ++e) c[e] = at + e < hi ? x[at + e] : (typename E::T)neg_inf();
          }
          if (order_of(chunk_max<E>(c)) <= above) continue;
#pragma unroll
          for (int e = 0; e < C::kN; ++e) {
            const int o = order_of(E::get(c[e]));
            if (o > above && at + e < hi) {
              const int f = atomicAdd(&n_found, 1);
              if (f < kFound) found[f] = key_of(o, (int)(at + e));
            }
          }
        }
        __syncthreads();
        return n_found;
      };
      int many_found = collect(bound > kNothing ? bound - 1 : bound);
      if (many_found > kFound && bound != kNothing) {
        // Too many are equal to the bound (a mask that leaves few scores: -inf): those above it, and the first ones that are equal
        __syncthreads();
        if (tid == 0) n_found = 0;
        __syncthreads();
        many_found = collect(bound);
        int got = many_found;
        for (int64_t from = lo; from < hi && got < n; from += kLongThreads) {
          const bool hit = from + tid < hi && order_of(E::get(x[from + tid])) == bound;
          const unsigned long long hits = __ballot(hit);
          if (tid % 64 == 0) picked[tid / 64] = __popcll(hits);  // (not needed any more)
          __syncthreads();
          int before = got, all_hits = 0;
          for (int w = 0; w < kWaves; ++w) {
            before += w < tid / 64 ? picked[w] : 0;
            all_hits += picked[w];
          }
          before += __popcll(hits & ((1ull << (tid % 64)) - 1));
          if (hit && before < n) keys[before] = key_of(bound, (int)(from + tid));
          got += all_hits;
          __syncthreads();
        }
      }
      slow = many_found > kFound;
      if (!slow) {
        // every key's place among them, whatever order they came in
        for (int i = tid; i < many_found; i += kLongThreads) {
          const int place = place_of(found[i], found, many_found);
          if (place < n) keys[place] = found[i];
        }
      }
    }
    if (slow) {                                                 // one after the other
      unsigned long long last = ~0ull;
      for (int i = 0; i < n; ++i) {
        unsigned long long k = 0;
        for (int64_t e = lo + tid; e < hi; e += kLongThreads) {
          const unsigned long long c = key_of(order_of(E::get(x[e])), (int)e);
          k = c < last && c > k ? c : k;
        }
        for (int d = 1; d < 64; d <<= 1) {
          const unsigned long long o = __shfl_xor(k, d);
          k = o > k ? o : k;
        }
        __syncthreads();
        if (tid % 64 == 0) best[tid / 64] = k;
        __syncthreads();
        for (int w = 0; w < kWaves; ++w) k = best[w] > k ? best[w] : k;
        last = k;
        if (tid == 0) keys[i] = k;
      }
    }
    for (int i = n + tid; i < a.top; i += kLongThreads) keys[i] = 0;
    __syncthreads();
  }
  if (a.splits == 1) {
    finish_row<E>(a, row, x, q, keys);
  } else {
    char *to = static_cast<char *>(a.workspace) + ((int64_t)row * a.splits + split) * part_bytes(a.top);
    if (tid == 0) *reinterpret_cast<Part *>(to) = Part{q, 0.0f};
    for (int i = tid; i < a.top; i += kLongThreads) reinterpret_cast<unsigned long long *>(to + 16)[i] = keys[i];
  }
}

// The parts of a row (at most 64) as one, a workgroup per row: sums in the order of the parts.  The parts' keys are falling, so that p + 1
// of them reach a part's p-th: the bound is the m-th largest of the parts' p-th, m (p + 1) >= `top`, and what reaches it is sorted.
template <class E>
__global__ __launch_bounds__(kLongThreads) void logprobs_join_kernel(LogprobsArgs a) {
  __shared__ unsigned long long keys[kMaxTop], all[64 * kMaxTop], heads[64], bound_;
  __shared__ Sums sums;
  __shared__ int n_all;
  const unsigned row = blockIdx.x, s = row / (unsigned)a.frames, t = row % (unsigned)a.frames;
  if (a.lengths && (int)t >= a.lengths[s]) return;
  const typename E::T *x = static_cast<const typename E::T *>(a.scores) + s * a.seq_stride + t * a.stride;
  const char *from = static_cast<const char *>(a.workspace) + (int64_t)row * a.splits * part_bytes(a.top);
  const int tid = threadIdx.x;
  if (tid < 64) {
    Sums q = {neg_inf(), 0.0f, 0.0f};
    if (tid < a.splits) q = reinterpret_cast<const Part *>(from + tid * part_bytes(a.top))->s;
    grow(q, max_over<64>(q.m));
    q.sum = sum_over<64>(q.sum);
    q.wsum = sum_over<64>(q.wsum);
    if (tid == 0) { sums = q; bound_ = 0; n_all = 0; }
  }
  if (a.top) {
    const int p = (a.top - 1) / a.splits, m = (a.top + p) / (p + 1);
    unsigned long long k = 0;
    if (tid < 64) heads[tid] = k = tid < a.splits ? reinterpret_cast<const unsigned long long *>(from + tid * part_bytes(a.top) + 16)[p] : 0;
    __syncthreads();
    if (tid < 64 && k && place_of(k, heads, 64) == m - 1) bound_ = k;
  }
  __syncthreads();
  if (a.top) {
    for (int i = tid; i < a.splits * a.top; i += kLongThreads) {
      const unsigned long long k = reinterpret_cast<const unsigned long long *>(from + (i / a.top) * part_bytes(a.top) + 16)[i % a.top];
      if (k && k >= bound_) all[atomicAdd(&n_all, 1)] = k;
    }
    __syncthreads();
    for (int i = tid; i < n_all; i += kLongThreads) {
      const int place = place_of(all[i], all, n_all);
      if (place < a.top) keys[place] = all[i];
    }
    __syncthreads();
  }
  finish_row<E>(a, row, x, sums, keys);
}

// ---- the gradient
struct Slope { float c, gh, h, m, ls; };                // of a row: p (c - gh (log p + h))
// a - b and what it lost
__device__ __forceinline__ float minus(float a, float b, float &lost) {
  const float s = a - b, t = s - a;
  lost = (a - (s - t)) - (b + t);
  return s;
}
// For fp32 scores p has all its digits however small it is: the roundings of log p are kept (within 3 times 2^-24 of itself; without
// that 125 times at log p = -80).  It costs 2 us of 27 at 118,417 rows of 129 and nothing at 2,048 of 64,001 (202 us).  For 16-bit scores the
// result's own rounding is 2^13 to 2^16 of those.
template <class E> __device__ __forceinline__ float grad_of(float x, Slope r) {
  float lp, p;
  if constexpr (sizeof(typename E::T) == 4) {
    float lost_m, lost_ls;
    const float d = minus(x, r.m, lost_m);
    lp = minus(d, r.ls, lost_ls);
    p = exp_near(lp, lost_m + lost_ls);
  } else {
    lp = (x - r.m) - r.ls;
    p = exp_fast(lp);
  }
  return p * (r.c - r.gh * (fmaxf(lp, -1e4f) + r.h));
}
// Token i of the given and the top ones, and its gradient; -1 if it has none.
__device__ __forceinline__ int named(const BackwardArgs &a, int64_t row, int i, float &g) {
  if (i < a.given) {
    g = a.grad_logprobs[row * a.given + i];
    const int j = a.tokens[row * a.given + i];
    return j >= 0 && j < a.v ? j : -1;
  }
  g = a.grad_top[row * a.top + (i - a.given)];
  return a.top_ids[row * a.top + (i - a.given)];
}

template <class E, int LANES, int EACH>
__global__ __launch_bounds__(256) void backward_short_kernel(BackwardArgs a) {
  const int lane = threadIdx.x % LANES;
  const unsigned row = blockIdx.x * (256 / LANES) + threadIdx.x / LANES, rows = (unsigned)a.seqs * a.frames;
  const unsigned s = row / (unsigned)a.frames, t = row % (unsigned)a.frames;
  if (row >= rows || (a.lengths && (int)t >= a.lengths[s])) return;      // (nothing is exchanged between lanes)
  const typename E::T *x = static_cast<const typename E::T *>(a.scores) + s * a.seq_stride + t * a.stride;
  typename E::T *dx = static_cast<typename E::T *>(a.grad_scores) + s * a.grad_seq_stride + t * a.grad_stride;
  float z[EACH], extra[EACH];
#pragma unroll
  for (int e = 0; e < EACH; ++e) {
    z[e] = lane + LANES * e < a.v ? E::get(x[lane + LANES * e]) : neg_inf();
    extra[e] = 0.0f;
  }
  Slope r;
  r.m = a.maximum[row];
  r.ls = a.log_sum[row];
  r.c = a.grad_lse ? a.grad_lse[row] : 0.0f;
  r.gh = a.grad_entropy ? a.grad_entropy[row] : 0.0f;
  r.h = a.grad_entropy ? a.entropy[row] : 0.0f;
  for (int i = 0; i < a.given + a.top; ++i) {          // every lane of the row goes over all of them, in their order
    float g;
    const int j = named(a, row, i, g);
    if (j < 0) continue;
    r.c -= g;
#pragma unroll
    for (int e = 0; e < EACH; ++e) extra[e] += j == lane + LANES * e ? g : 0.0f;
  }
  const bool empty = is_empty(r.m, r.ls);
#pragma unroll
  for (int e = 0; e < EACH; ++e)
    if (lane + LANES * e < a.v) dx[lane + LANES * e] = E::put(empty ? 0.0f : grad_of<E>(z[e], r) + extra[e]);
}

// A workgroup per part of a long row.  Scores that a token names are read first (the gradient may take the scores' place) and
// written last, after the rest of the part.
template <class E>
__global__ __launch_bounds__(kLongThreads) void backward_long_kernel(BackwardArgs a) {
  using C = Chunk<E>;
  constexpr int kStep = kLongThreads * C::kN, kPart = kStep * kLongLoads;
  constexpr int kNamed = kMaxGiven + kMaxTop, kMine = (kNamed + kLongThreads - 1) / kLongThreads;
  __shared__ int ids[kNamed];
  __shared__ float grads[kNamed];
  const unsigned row = blockIdx.x / (unsigned)a.splits, split = blockIdx.x % (unsigned)a.splits;
  const unsigned s = row / (unsigned)a.frames, t = row % (unsigned)a.frames;
  if (a.lengths && (int)t >= a.lengths[s]) return;
  const typename E::T *x = static_cast<const typename E::T *>(a.scores) + s * a.seq_stride + t * a.stride;
  typename E::T *dx = static_cast<typename E::T *>(a.grad_scores) + s * a.grad_seq_stride + t * a.grad_stride;
  const int64_t lo = (int64_t)split * kPart, hi = a.v - lo < kPart ? a.v : lo + kPart;
  const int tid = threadIdx.x, n = a.given + a.top;
  typename C::Vec c[kLongLoads];
#pragma unroll
  for (int i = 0; i < kLongLoads; ++i) {
    const int64_t j = lo + tid * C::kN + i * kStep;
    if (j + C::kN <= hi) {
      c[i] = C::load(x + j);
    } else {
#pragma unroll
      for (int e = 0; e < C::kN; ++e) c[i][e] = j + e < hi ? x[j + e] : (typename E::T)0.0f;
    }
  }
  for (int i = tid; i < n; i += kLongThreads) ids[i] = named(a, row, i, grads[i]);
  Slope r;
  r.m = a.maximum[row];
  r.ls = a.log_sum[row];
  r.c = a.grad_lse ? a.grad_lse[row] : 0.0f;
  r.gh = a.grad_entropy ? a.grad_entropy[row] : 0.0f;
  r.h = a.grad_entropy ? a.entropy[row] : 0.0f;
  const bool empty = is_empty(r.m, r.ls);
  __syncthreads();
  for (int i = 0; i < n; ++i) r.c -= ids[i] >= 0 ? grads[i] : 0.0f;
  float late[kMine];
  int where[kMine];
#pragma unroll
  for (int k = 0; k < kMine; ++k) {
    const int i = tid + k * kLongThreads, j = i < n ? ids[i] : -1;
    where[k] = j >= lo && j < hi ? j : -1;
    for (int f = 0; f < i && where[k] >= 0; ++f)
      if (ids[f] == j) where[k] = -1;                  // the first that names it does it
    if (where[k] < 0) continue;
    float extra = 0.0f;
    for (int f = i; f < n; ++f) extra += ids[f] == j ? grads[f] : 0.0f;
    late[k] = empty ? 0.0f : grad_of<E>(E::get(x[j]), r) + extra;
  }
  __syncthreads();                                     // the named scores have been read
#pragma unroll
  for (int i = 0; i < kLongLoads; ++i) {
    const int64_t j = lo + tid * C::kN + i * kStep;
    typename C::Vec d;
#pragma unroll
    for (int e = 0; e < C::kN; ++e) d[e] = E::put(empty ? 0.0f : grad_of<E>(E::get(c[i][e]), r));
    if (j + C::kN <= hi) {
      C::store(dx + j, d);
    } else {
#pragma unroll
      for (int e = 0; e < C::kN; ++e)
        if (j + e < hi) dx[j + e] = d[e];
    }
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kMine; ++k)
    if (where[k] >= 0) dx[where[k]] = E::put(late[k]);
}

}  // namespace wfst_ops

#endif  // WFST_LOGPROBS_H_
