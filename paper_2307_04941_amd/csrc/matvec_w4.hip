// Products of few tokens with 4-bit weights (include/mg3m_seq.h).
#include "seq_device.h"

namespace mg3m {

// One wave per output: lane l takes the blocks of 32 weights l, l + 64, ...
// of its row; a block lies in one group.
template <typename T>
__global__ __launch_bounds__(64) void matvec_w4(mg3m_w4 a) {
  const int k = blockIdx.x, m = blockIdx.y, lane = threadIdx.x;
  const int groups = a.C / a.group;
  const T* x = static_cast<const T*>(a.x) + m * a.ldx;
  const uint4* q = reinterpret_cast<const uint4*>(a.q + (long long)k * (a.C / 2));
  float sum = 0.0f;
  for (int b = lane; b < a.C / 32; b += 64) {
    const long long g = (long long)k * groups + b * 32 / a.group;
    const float zero = a.zero != nullptr ? (float)a.zero[g] : 8.0f;
    const uint4 v = q[b];
    const unsigned words[4] = {v.x, v.y, v.z, v.w};
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < 32; ++i)
      s = fmaf((float)x[b * 32 + i], (float)((words[i / 8] >> (4 * (i % 8))) & 15u) - zero, s);
    sum = fmaf(s, (float)static_cast<const T*>(a.scale)[g], sum);
  }
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
  if (lane == 0) static_cast<T*>(a.y)[m * a.ldy + k] = (T)sum;
}

int launch_w4(const mg3m_w4& a, void* stream, std::string* err) {
  return with_dtype(a.dtype, [&](auto t) {
    matvec_w4<decltype(t)><<<dim3(a.K, a.M), 64, 0, static_cast<hipStream_t>(stream)>>>(a);
    return launched("4-bit product", err);
  });
}

}  // namespace mg3m
