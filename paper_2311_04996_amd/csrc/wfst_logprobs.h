// Log-probabilities of given tokens, entropy and top alternatives of rows of scores, and their gradient.
#ifndef WFST_LOGPROBS_H_
#define WFST_LOGPROBS_H_

#include "wfst_elements.h"

namespace wfst_ops {

struct LogprobsArgs {
  const void *scores;
  const int32_t *tokens, *lengths;
  float *logprobs, *lse, *entropy, *stats;
  int32_t *top_ids;
  float *top_logprobs;
  int64_t seq_stride, stride;
  int32_t seqs, frames, v, given, top;
};

struct BackwardArgs {
  const void *scores;
  const int32_t *tokens, *lengths;
  const float *stats, *entropy;
  const int32_t *top_ids;
  const float *grad_logprobs, *grad_lse, *grad_entropy, *grad_top;
  void *grad_scores;
  int64_t seq_stride, stride, grad_seq_stride, grad_stride;
  int32_t seqs, frames, v, given, top;
};

// A float as a whole number that orders alike: -0 and +0 are one, every NaN is above +inf.
__device__ __forceinline__ int order_of(float x) {
  if (x != x) return 0x7fffffff;
  const int b = __float_as_int(x + 0.0f);
  return b < 0 ? b ^ 0x7fffffff : b;
}
// (order, lower index first) as one number
__device__ __forceinline__ unsigned long long key_of(float x, int j) {
  return ((unsigned long long)((unsigned)order_of(x) ^ 0x80000000u) << 32) | (unsigned)~j;
}

__device__ __forceinline__ float neg_inf() { return -__builtin_inff(); }

// log-probability of a score in a row with this maximum and log of the sum behind it: in an empty row it is -inf
__device__ __forceinline__ float logprob_of(float x, float m, float ls) { return m == neg_inf() ? m : (x - m) - ls; }

// one workgroup of 256 per row, several passes over it
template <class E>
__global__ __launch_bounds__(256) void logprobs_kernel(LogprobsArgs a) {
  __shared__ float part[2][256];
  __shared__ unsigned long long keys[256];
  const int64_t row = blockIdx.x;
  const int s = (int)(row / a.frames), t = (int)(row % a.frames);
  if (a.lengths && t >= a.lengths[s]) return;
  const typename E::T *x = static_cast<const typename E::T *>(a.scores) + s * a.seq_stride + t * a.stride;
  const int tid = threadIdx.x;
  float m = neg_inf();
  for (int j = tid; j < a.v; j += 256) m = fmaxf(m, E::get(x[j]));
  part[0][tid] = m;
  __syncthreads();
  for (int i = 0; i < 256; ++i) m = fmaxf(m, part[0][i]);
  const float base = m == neg_inf() ? 0.0f : m;
  float sum = 0.0f, ent = 0.0f;
  for (int j = tid; j < a.v; j += 256) {
    const float d = E::get(x[j]) - base, e = exp_fast(d);
    sum += e;
    ent += e * fmaxf(d, -1e4f);
  }
  __syncthreads();
  part[0][tid] = sum;
  part[1][tid] = ent;
  __syncthreads();
  sum = ent = 0.0f;
  for (int i = 0; i < 256; ++i) { sum += part[0][i]; ent += part[1][i]; }
  const float ls = logf(sum), lse = m + ls;
  if (tid == 0) {
    if (a.lse) a.lse[row] = lse;
    if (a.stats) { a.stats[2 * row] = m; a.stats[2 * row + 1] = ls; }
    if (a.entropy) a.entropy[row] = m == neg_inf() && sum == 0.0f ? 0.0f : ls - ent / sum;
  }
  if (a.logprobs)
    for (int g = tid; g < a.given; g += 256) {
      const int j = a.tokens[row * a.given + g];
      float lp = __builtin_nanf("");
      if (j == -1) lp = 0.0f;
      else if (j >= 0 && j < a.v) lp = logprob_of(E::get(x[j]), m, ls);
      a.logprobs[row * a.given + g] = lp;
    }
  unsigned long long last = ~0ull;
  for (int i = 0; i < a.top; ++i) {
    unsigned long long best = 0;
    for (int j = tid; j < a.v; j += 256) {
      const unsigned long long k = key_of(E::get(x[j]), j);
      if (k < last && k > best) best = k;
    }
    __syncthreads();
    keys[tid] = best;
    __syncthreads();
    for (int q = 0; q < 256; ++q) best = keys[q] > best ? keys[q] : best;
    last = best;
    if (tid == 0) {
      const int j = (int)~(unsigned)best;
      if (a.top_ids) a.top_ids[row * a.top + i] = j;
      if (a.top_logprobs) a.top_logprobs[row * a.top + i] = logprob_of(E::get(x[j]), m, ls);
    }
  }
}

// one workgroup of 256 per row; the elements that a given token or a top one names are written last
template <class E>
__global__ __launch_bounds__(256) void logprobs_backward_kernel(BackwardArgs a) {
  const int64_t row = blockIdx.x;
  const int s = (int)(row / a.frames), t = (int)(row % a.frames);
  if (a.lengths && t >= a.lengths[s]) return;
  const typename E::T *x = static_cast<const typename E::T *>(a.scores) + s * a.seq_stride + t * a.stride;
  typename E::T *dx = static_cast<typename E::T *>(a.grad_scores) + s * a.grad_seq_stride + t * a.grad_stride;
  const float m = a.stats[2 * row], ls = a.stats[2 * row + 1], h = a.grad_entropy ? a.entropy[row] : 0.0f, gh = a.grad_entropy ? a.grad_entropy[row] : 0.0f;
  const bool empty = m == neg_inf();
  float c = a.grad_lse ? a.grad_lse[row] : 0.0f;
  for (int g = 0; a.grad_logprobs && g < a.given; ++g) {
    const int j = a.tokens[row * a.given + g];
    if (j >= 0 && j < a.v) c -= a.grad_logprobs[row * a.given + g];
  }
  for (int i = 0; a.grad_top && i < a.top; ++i) c -= a.grad_top[row * a.top + i];
  for (int j = threadIdx.x; j < a.v; j += 256) {
    float extra = 0.0f;
    for (int g = 0; a.grad_logprobs && g < a.given; ++g)
      if (a.tokens[row * a.given + g] == j) extra += a.grad_logprobs[row * a.given + g];
    for (int i = 0; a.grad_top && i < a.top; ++i)
      if (a.top_ids[row * a.top + i] == j) extra += a.grad_top[row * a.top + i];
    const float lp = (E::get(x[j]) - m) - ls, p = exp_fast(lp);
    float v = p * (c - gh * (fmaxf(lp, -1e4f) + h)) + extra;
    dx[j] = E::put(empty ? 0.0f : v);
  }
}

}  // namespace wfst_ops

#endif  // WFST_LOGPROBS_H_
