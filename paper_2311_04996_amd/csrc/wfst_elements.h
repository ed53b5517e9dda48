// Element types of the operators beside the decoder: fp32, binary16, bfloat16 (WFST_LOGLIKE_*).  Everything is computed
// in fp32; a 16-bit result is rounded once, to nearest even, where it is stored.
#ifndef WFST_ELEMENTS_H_
#define WFST_ELEMENTS_H_

#include <hip/hip_runtime.h>

#include <cstdint>

namespace wfst_ops {

struct F32 {
  using T = float;
  static __device__ __forceinline__ float get(float v) { return v; }
  static __device__ __forceinline__ float put(float v) { return v; }
};
struct F16 {
  using T = _Float16;
  static __device__ __forceinline__ float get(_Float16 v) { return (float)v; }
  static __device__ __forceinline__ _Float16 put(float v) { return (_Float16)v; }
};
struct BF16 {
  using T = __bf16;
  static __device__ __forceinline__ float get(__bf16 v) { return (float)v; }
  static __device__ __forceinline__ __bf16 put(float v) { return (__bf16)v; }
};

// element i of an array whose type is known at run time only (bias, residual, results): a uniform branch
__device__ __forceinline__ float load_as(const void *p, int64_t i, int dtype) {
  if (dtype == 0) return static_cast<const float *>(p)[i];
  if (dtype == 1) return (float)static_cast<const _Float16 *>(p)[i];
  return (float)static_cast<const __bf16 *>(p)[i];
}
__device__ __forceinline__ void store_as(void *p, int64_t i, int dtype, float v) {
  if (dtype == 0) static_cast<float *>(p)[i] = v;
  else if (dtype == 1) static_cast<_Float16 *>(p)[i] = (_Float16)v;
  else static_cast<__bf16 *>(p)[i] = (__bf16)v;
}

constexpr float kLog2e = 1.44269504088896340736f;

// e^d from the hardware's 2^x (1 ulp).  The product d * log2 e and the constant in it are rounded, so the result is off by up to
// 1.25 |d| 2^-24 of itself besides: 1.2e-6 at d = -16, where the term is 1e-7 of a sum that has a 1 in it.
__device__ __forceinline__ float exp_fast(float d) { return __builtin_amdgcn_exp2f(d * kLog2e); }
// e^(unit (d + rest)), |rest| at most a rounding of d, unit +-2^i, within 2 ulp: what the product lost is put back by
// 2^(q + r) = 2^q (1 + r ln 2).  Where the result is fp32 and e^d not a term of a sum.  (|q| >= 128: 0, infinite, or less than the least normal number.)
__device__ __forceinline__ float exp_near(float d, float rest = 0.0f, float unit = 1.0f) {
  const float hi = kLog2e * unit, lo = 1.92596299e-8f * unit;          // (log2 e - kLog2e)
  const float q = d * hi, e = __builtin_amdgcn_exp2f(q), r = __builtin_fmaf(rest, hi, __builtin_fmaf(d, lo, __builtin_fmaf(d, hi, -q)));
  return fabsf(q) < 128.0f ? __builtin_fmaf(e, r * 0.693147181f, e) : e;
}

}  // namespace wfst_ops

#endif  // WFST_ELEMENTS_H_
