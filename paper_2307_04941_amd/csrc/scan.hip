// Selective state space scan (include/mg3m_seq.h).
#include "seq_device.h"

namespace mg3m {

// One wave per sequence and channel walks the tokens; lane l holds the states
// l, l + 64, ... and the wave sums their outputs.
template <typename T>
__global__ __launch_bounds__(64) void scan_seq(mg3m_scan a) {
  const int d = blockIdx.x, n = blockIdx.y, lane = threadIdx.x;
  const int g = d / (a.D / a.G);
  const SeqRange r = seq_range(a.begin, a.end, n, a.N, a.T);
  float A[4], h[4];
  float* state = a.state != nullptr ? a.state + ((long long)n * a.D + d) * a.S : nullptr;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int s = lane + 64 * i;
    A[i] = s < a.S ? a.A[(long long)d * a.S + s] * kLog2e : 0.0f;
    h[i] = s < a.S && state != nullptr && a.load_state ? state[s] : 0.0f;
  }
  const float skip = a.D_skip != nullptr ? a.D_skip[d] : 0.0f;
  const float bias = a.dt_bias != nullptr ? a.dt_bias[d] : 0.0f;
  for (long long t = r.b; t < r.e; ++t) {
    const float u = (float)static_cast<const T*>(a.u)[t * a.ldu + d];
    float delta = (float)static_cast<const T*>(a.dt)[t * a.lddt + d] + bias;
    if (a.softplus) delta = softplus(delta);
    float y = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int s = lane + 64 * i;
      if (s < a.S) {
        const float B = (float)static_cast<const T*>(a.B)[t * a.ldb + g * a.S + s];
        const float C = (float)static_cast<const T*>(a.C)[t * a.ldc + g * a.S + s];
        h[i] = fmaf(__builtin_amdgcn_exp2f(delta * A[i]), h[i], delta * u * B);
        y = fmaf(C, h[i], y);
      }
    }
    for (int o = 32; o > 0; o >>= 1) y += __shfl_xor(y, o);
    y = fmaf(skip, u, y);
    if (a.z != nullptr) {
      const float z = (float)static_cast<const T*>(a.z)[t * a.ldz + d];
      y *= z * sigmoid(z);
    }
    if (lane == 0) static_cast<T*>(a.y)[t * a.ldy + d] = (T)y;
  }
  if (state != nullptr) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (lane + 64 * i < a.S) state[lane + 64 * i] = h[i];
  }
}

size_t scan_workspace_bytes(int, int, int, int, int) { return 0; }

int launch_scan(const mg3m_scan& a, void*, void* stream, std::string* err) {
  return with_dtype(a.dtype, [&](auto t) {
    scan_seq<decltype(t)><<<dim3(a.D, a.N), 64, 0, static_cast<hipStream_t>(stream)>>>(a);
    return launched("selective scan", err);
  });
}

int launch_scan_step(const mg3m_scan& a, void* stream, std::string* err) {
  mg3m_scan s = a;
  s.T = a.N;
  s.load_state = 1;
  return launch_scan(s, nullptr, stream, err);
}

}  // namespace mg3m
