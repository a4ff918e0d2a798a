// Causal depthwise convolution along tokens (include/mg3m_seq.h).
#include "seq_device.h"

namespace mg3m {

// One thread per sequence and channel walks the tokens with its last R inputs
// in registers.
template <typename T, int R>
__global__ __launch_bounds__(64) void conv1d_seq(mg3m_conv1d a) {
  const int c = blockIdx.x * 64 + threadIdx.x, n = blockIdx.y;
  if (c >= a.C) return;
  const SeqRange r = seq_range(a.begin, a.end, n, a.N, a.T);
  const T* x = static_cast<const T*>(a.x) + c;
  T* y = static_cast<T*>(a.y) + c;
  T* state = a.state != nullptr && R > 1 ? static_cast<T*>(a.state) + (long long)n * (R - 1) * a.C + c : nullptr;
  float w[R], v[R];
#pragma unroll
  for (int i = 0; i < R; ++i) w[i] = (float)static_cast<const T*>(a.w)[(long long)i * a.C + c];
#pragma unroll
  for (int i = 1; i < R; ++i) v[i] = state != nullptr && a.load_state ? (float)state[(long long)(i - 1) * a.C] : 0.0f;
  const float bias = a.bias != nullptr ? (float)static_cast<const T*>(a.bias)[c] : 0.0f;
  for (int t = r.b; t < r.e; ++t) {
#pragma unroll
    for (int i = 0; i + 1 < R; ++i) v[i] = v[i + 1];
    v[R - 1] = (float)x[t * a.ldx];
    float s = bias;
#pragma unroll
    for (int i = 0; i < R; ++i) s = fmaf(w[i], v[i], s);
    if (a.silu) s *= sigmoid(s);
    y[t * a.ldy] = (T)s;
  }
  if (state != nullptr) {
#pragma unroll
    for (int i = 1; i < R; ++i) state[(long long)(i - 1) * a.C] = (T)v[i];
  }
}

template <typename T>
static int launch_taps(const mg3m_conv1d& a, void* stream, std::string* err) {
  const dim3 grid((a.C + 63) / 64, a.N);
  hipStream_t st = static_cast<hipStream_t>(stream);
  switch (a.R) {
    case 1: conv1d_seq<T, 1><<<grid, 64, 0, st>>>(a); break;
    case 2: conv1d_seq<T, 2><<<grid, 64, 0, st>>>(a); break;
    case 3: conv1d_seq<T, 3><<<grid, 64, 0, st>>>(a); break;
    case 4: conv1d_seq<T, 4><<<grid, 64, 0, st>>>(a); break;
    case 5: conv1d_seq<T, 5><<<grid, 64, 0, st>>>(a); break;
    case 6: conv1d_seq<T, 6><<<grid, 64, 0, st>>>(a); break;
    case 7: conv1d_seq<T, 7><<<grid, 64, 0, st>>>(a); break;
    default: conv1d_seq<T, 8><<<grid, 64, 0, st>>>(a); break;
  }
  return launched("causal convolution", err);
}

int launch_conv1d(const mg3m_conv1d& a, void* stream, std::string* err) {
  return with_dtype(a.dtype, [&](auto t) { return launch_taps<decltype(t)>(a, stream, err); });
}

int launch_conv1d_step(const mg3m_conv1d& a, void* stream, std::string* err) {
  mg3m_conv1d s = a;
  s.T = a.N;
  s.load_state = 1;
  return launch_conv1d(s, stream, err);
}

}  // namespace mg3m
