// Device helpers of the sequence kernels.
#pragma once

#include <hip/hip_runtime.h>

#include <string>

#include "seq.h"

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

inline int launched(const char* what, std::string* err) {
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) return MG3M_OK;
  *err = std::string(what) + " launch: " + hipGetErrorString(e);
  return MG3M_ERR_HIP;
}

// The rows of sequence n, inside 0..T whatever begin and end hold.
struct SeqRange {
  int b, e;
};
__device__ __forceinline__ SeqRange seq_range(const int* begin, const int* end, int n, int N, int T) {
  if (begin == nullptr) {
    const int L = T / N;
    return {n * L, n * L + L};
  }
  const int b = min(max(begin[n], 0), T);
  return {b, min(max(end[n], b), T)};
}

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.693147180559945309417f;

__device__ __forceinline__ float sigmoid(float v) {
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-v * kLog2e));
}

// log(1 + exp(v)) = max(v, 0) + log(1 + e), e = exp(-|v|) in (0, 1].  1 + e
// rounds to w; log(w) * e / (w - 1) is log(1 + e) to a few roundings for any e
// (Kahan's correction: log(1 + e) / e is flat where w - 1 differs from e), so
// steps far below 2^-24 keep their relative precision.
__device__ __forceinline__ float softplus(float v) {
  const float e = __builtin_amdgcn_exp2f(-fabsf(v) * kLog2e);
  const float w = 1.0f + e;
  const float d = w - 1.0f;
  const float l = d == 0.0f ? e : __builtin_amdgcn_logf(w) * kLn2 * (e * __builtin_amdgcn_rcpf(d));
  return fmaxf(v, 0.0f) + l;
}

}  // namespace mg3m
