// Device helpers of the sequence kernels.
#pragma once

#include <hip/hip_runtime.h>

#include <string>

#include "seq.h"
#include "seq_pieces.h"

namespace mg3m {

// Element types of dtype: fp32, bf16, fp16.  Conversions from float round to
// nearest, ties to even.
template <typename F>
int with_dtype(int dtype, F&& f) {
  switch (dtype) {
    case MG3M_F32: return f(float{});
    case MG3M_BF16: return f(__bf16{});
    default: return f(_Float16{});
  }
}

// The value of an element loaded into 32 bits.  The empty asm keeps the
// compiler from holding it in 16 across a loop, which takes an instruction
// after the load and so a wait for it.
template <typename T>
__device__ __forceinline__ float raw_value(unsigned v) {
  if constexpr (sizeof(T) == 4) {
    return __builtin_bit_cast(float, v);
  } else {
    asm("" : "+v"(v));
    return (float)__builtin_bit_cast(T, (unsigned short)v);
  }
}

// Whether a launch takes this many work-groups: grids are counted in threads
// of 32 bits.
inline bool fits_launch(long long groups, int threads) {
  return groups <= 0x7fffffffLL && groups * threads <= 0xffffffffLL;
}

inline int launched(const char* what, std::string* err) {
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) return MG3M_OK;
  *err = std::string(what) + " launch: " + hipGetErrorString(e);
  return MG3M_ERR_HIP;
}

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.693147180559945309417f;

__device__ __forceinline__ float sigmoid(float v) {
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-v * kLog2e));
}

// log(1 + exp(v)) = max(v, 0) + log(1 + e), e = exp(-|v|) in (0, 1].  1 + e
// rounds to w and leaves r = e - (w - 1), exactly, so log(1 + e) = log(w) +
// log(1 + r / w); r is at most 2^-24 and r / w differs from r by less than a
// rounding of the result.  Steps far below 2^-24 keep their precision: w is 1
// and r is e.
__device__ __forceinline__ float softplus(float v) {
  const float e = __builtin_amdgcn_exp2f(-fabsf(v) * kLog2e);
  const float w = 1.0f + e;
  const float r = e - (w - 1.0f);
  return fmaxf(v, 0.0f) + fmaf(__builtin_amdgcn_logf(w), kLn2, r);
}

}  // namespace mg3m
