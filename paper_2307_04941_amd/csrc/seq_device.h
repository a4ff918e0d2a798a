// Device helpers of the sequence kernels.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
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

// Sequences cut into pieces of W tokens, numbered without knowing the lengths
// on the host: equal sequences have ceil(L / W) pieces each; otherwise the
// pieces of sequence n are numbered from begin[n] / W + n, which leaves room
// for them (ceil(len / W) <= end / W - begin / W + 1) and grows with n, so a
// piece finds its sequence by bisection.  Numbers that no piece has are left
// out.  W = 0: every sequence is one piece.  Each sequence has at least piece
// 0, an empty one too.
struct Piece {
  int n, k;           // sequence and piece in it; n < 0: none
  int b, e;           // its rows
  bool last;          // the sequence's last piece
};
inline long long piece_count(const int* begin, int N, int T, int W) {
  if (W == 0) return N;
  if (begin == nullptr) return (long long)N * std::max(1, (T / N + W - 1) / W);
  return (long long)T / W + N;
}
__device__ __forceinline__ int piece_base(const int* begin, int n, int T, int W) {
  return (int)((unsigned)min(max(begin[n], 0), T) / (unsigned)W) + n;
}
__device__ __forceinline__ Piece find_piece(const int* begin, const int* end, int N, int T, int W, int id) {
  Piece p{id, 0, 0, 0, true};
  if (W != 0) {
    if (begin == nullptr) {
      const int per = max(1, (T / N + W - 1) / W);
      p.n = id / per;
      p.k = id - p.n * per;
    } else {
      int lo = -1, hi = N;            // base(lo) <= id < base(hi)
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (piece_base(begin, mid, T, W) <= id) lo = mid; else hi = mid;
      }
      p.n = lo;
      if (lo < 0) return p;
      p.k = id - piece_base(begin, lo, T, W);
    }
  }
  const SeqRange r = seq_range(begin, end, p.n, N, T);
  const long long b = (long long)r.b + (long long)p.k * W;
  if (p.k > 0 && b >= r.e) {
    p.n = -1;
    return p;
  }
  p.b = (int)b;
  p.e = r.e;
  if (W != 0 && r.e - p.b > W) {
    p.e = p.b + W;
    p.last = false;
  }
  return p;
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
