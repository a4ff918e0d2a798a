// Products of few tokens with 4-bit weights (include/mg3m_seq.h).
//
// Bound by the weights' bytes: with one token each weight is used once, with
// 16 still only 16 times.  What has to be cheap is a weight's way from four
// bits to a matrix instruction.  v_mfma_f32_16x16x32 takes 16 tokens (rows)
// times 16 weight rows (columns): a lane holds eight consecutive channels of
// one row, which is one dword of 4-bit weights, so no weight moves between
// lanes.  Shifted so that a nibble is the top of a 16-bit float's mantissa
// under the exponent of 16, w & mask | exponent is the pair of numbers 16 + q,
// exact in bf16 and in fp16: two instructions for two weights.  The 16 and the
// zero point leave the sum through a second product, with ones:
//   sum x (q - zero) = sum x (16 + q) - (16 + zero) sum x,
// whose terms are 31/8 the size of the result's, so two of fp32's 24 bits.
// fp32 tokens go in as three bf16 parts (exact, as in conv_b3.h).
//
// A work-group has eight waves: RW tiles of 16 weight rows times CW slices of
// the channels, whose sums are joined through LDS in a fixed order.  It keeps
// x in LDS in the order the matrix instruction takes it, eight channels of a
// token together, permuted as the weights come out of a dword; long rows in
// slabs.  A wave has four blocks of 128 channels of weights under way.
#include "seq_device.h"

namespace mg3m {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr int kUnit = 128;          // channels per wave and step: 16 bytes of weights per lane
constexpr int kAhead = 4;           // steps whose weights are under way

struct W4Args {
  mg3m_w4 p;
  int slab_log2;   // units of x in LDS, CW at least
  int vec;         // x rows are 16-byte aligned
};

template <typename T>
struct W4Type;
template <>
struct W4Type<__bf16> {
  static constexpr int kParts = 1, kShift = 3;
  static constexpr unsigned kSixteen = 0x41804180u, kOnes = 0x3f803f80u;
};
template <>
struct W4Type<float> : W4Type<__bf16> {
  static constexpr int kParts = 3;
};
template <>
struct W4Type<_Float16> {
  static constexpr int kParts = 1, kShift = 6;
  static constexpr unsigned kSixteen = 0x4c004c00u, kOnes = 0x3c003c00u;
};

template <typename T>
__device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
  if constexpr (W4Type<T>::kShift == 6)
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// The eight weights of a dword as 16 + q, in the order 0 4 1 5 2 6 3 7.
template <typename T>
__device__ __forceinline__ u32x4 expand(unsigned w) {
  constexpr int s = W4Type<T>::kShift;
  constexpr unsigned mask = 0x000f000fu << s;
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int by = 4 * i - s;
    r[i] = ((by < 0 ? w << -by : w >> by) & mask) | W4Type<T>::kSixteen;
  }
  return r;
}

__device__ __forceinline__ unsigned pack2(unsigned short lo, unsigned short hi) { return lo | (unsigned)hi << 16; }

// Eight channels of a token as the MFMA takes them, in `parts` 16-byte units.
template <typename T>
__device__ __forceinline__ void arrange(const T (&v)[8], u32x4 (&out)[W4Type<T>::kParts]) {
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      out[0][i] = pack2(__builtin_bit_cast(unsigned short, v[i]), __builtin_bit_cast(unsigned short, v[i + 4]));
  } else {
    unsigned short b[3][8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      // a part is the float's upper 16 bits: the rest is exact
      float r = v[i];
#pragma unroll
      for (int q = 0; q < 3; ++q) {
        const unsigned top = __builtin_bit_cast(unsigned, r) & 0xffff0000u;
        b[q][i] = (unsigned short)(top >> 16);
        r -= __builtin_bit_cast(float, top);
      }
    }
#pragma unroll
    for (int q = 0; q < 3; ++q)
#pragma unroll
      for (int i = 0; i < 4; ++i) out[q][i] = pack2(b[q][i], b[q][i + 4]);
  }
}

// WHOLE: a group covers whole units.  Otherwise the lanes' dwords are
// transposed (lane quarter against dword), after which an MFMA covers 32
// consecutive channels, which lie in one group.
template <typename T, int RW, int CW, bool WHOLE>
__global__ __launch_bounds__(512) void matvec_w4(W4Args a) {
  constexpr int kParts = W4Type<T>::kParts;
  extern __shared__ u32x4 xs[];                  // [unit][part][16 blocks of 8 channels][tokens]
  const mg3m_w4& p = a.p;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int rw = wave / CW, cw = wave - rw * CW;
  const int col = lane & 15, quarter = lane >> 4;
  const int row_blocks = (p.K + 16 * RW - 1) / (16 * RW);
  const int mb = blockIdx.x / row_blocks;
  const int m0 = mb * 16, tokens = min(16, p.M - m0);
  const int row = (int)(blockIdx.x - mb * row_blocks) * (16 * RW) + rw * 16 + col;
  const bool live = row < p.K;
  const long long r = min(row, p.K - 1);
  const int units = (p.C + kUnit - 1) / kUnit, groups = p.C / p.group;
  const unsigned char* q = p.q + r * (p.C / 2);
  const T* scale = static_cast<const T*>(p.scale) + r * groups;
  const unsigned char* zero = p.zero != nullptr ? p.zero + r * groups : nullptr;
  const int token = min(col, tokens - 1);        // columns behind the last token repeat it

  // unit i of this wave; behind the end the row's first bytes, against x = 0
  auto weights = [&](int i) {
    const int c = (i * CW + cw) * kUnit + quarter * 32;
    return *reinterpret_cast<const u32x4*>(q + (c < p.C ? c / 2 : 0));
  };
  u32x4 w[kAhead];
#pragma unroll
  for (int i = 0; i < kAhead; ++i) w[i] = weights(i);

  const u32x4 ones = {W4Type<T>::kOnes, W4Type<T>::kOnes, W4Type<T>::kOnes, W4Type<T>::kOnes};
  f32x4 y = {};
  const int slab = 1 << a.slab_log2, per_slab = slab / CW;
  const int rounds = ((units + slab - 1) >> a.slab_log2) * per_slab;     // the same for all waves

  auto stage = [&](int unit0) {
    const int blocks = min(slab, units - unit0) * (kUnit / 8), row_log2 = a.slab_log2 + 4;
    for (int i = threadIdx.x; i < tokens << row_log2; i += 512) {
      const int m = i >> row_log2, b = i & ((1 << row_log2) - 1);
      if (b >= blocks) continue;
      const int c = unit0 * kUnit + b * 8;
      const T* x = static_cast<const T*>(p.x) + (m0 + m) * p.ldx + c;
      T v[8];
      if (c < p.C) {
        if (a.vec) {
#pragma unroll
          for (int k = 0; k < (int)sizeof(T) / 2; ++k)
            *reinterpret_cast<u32x4*>(v + k * 16 / sizeof(T)) = reinterpret_cast<const u32x4*>(x)[k];
        } else {
#pragma unroll
          for (int k = 0; k < 8; ++k) v[k] = x[k];
        }
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = (T)0.0f;
      }
      u32x4 o[kParts];
      arrange(v, o);
      const int u = b / 16;
#pragma unroll
      for (int part = 0; part < kParts; ++part) xs[((u * kParts + part) * 16 + b % 16) * tokens + m] = o[part];
    }
  };

  for (int i0 = 0; i0 < rounds; i0 += kAhead) {
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int i = i0 + k;
      if (i >= rounds) break;
      if ((i & (per_slab - 1)) == 0) {
        if (i > 0) __syncthreads();
        stage(i * CW);
        __syncthreads();
      }
      const int unit = i * CW + cw;
      if (unit < units) {
        u32x4 v = w[k];
        if constexpr (!WHOLE) {
          const auto s02 = __builtin_amdgcn_permlane32_swap(v[0], v[2], false, false);
          const auto s13 = __builtin_amdgcn_permlane32_swap(v[1], v[3], false, false);
          const auto s01 = __builtin_amdgcn_permlane16_swap(s02[0], s13[0], false, false);
          const auto s23 = __builtin_amdgcn_permlane16_swap(s02[1], s13[1], false, false);
          v = u32x4{s01[0], s01[1], s23[0], s23[1]};
        }
        const u32x4* x = xs + (unit & (slab - 1)) * kParts * 16 * tokens + token;
        auto scaled = [&](f32x4 dot, f32x4 sum, int c) {
          const int g = min(c, p.C - 1) / p.group;
          const float s = (float)scale[g], z = 16.0f + (zero != nullptr ? (float)zero[g] : 8.0f);
#pragma unroll
          for (int e = 0; e < 4; ++e) y[e] = fmaf(s, fmaf(-z, sum[e], dot[e]), y[e]);
        };
        f32x4 dot = {}, sum = {};
#pragma unroll
        for (int d = 0; d < 4; ++d) {
          const u32x4 b = expand<T>(v[d]);
          const int block = WHOLE ? quarter * 4 + d : d * 4 + quarter;
#pragma unroll
          for (int part = 0; part < kParts; ++part) {
            const u32x4 xa = x[(part * 16 + block) * tokens];
            dot = mfma<T>(xa, b, dot);
            sum = mfma<T>(xa, ones, sum);
          }
          if constexpr (!WHOLE) {
            scaled(dot, sum, unit * kUnit + d * 32);
            dot = sum = f32x4{};
          }
        }
        if constexpr (WHOLE) scaled(dot, sum, unit * kUnit);
      }
      w[k] = weights(i + kAhead);
    }
  }

  // join the slices
  if constexpr (CW > 1) {
    __syncthreads();
    f32x4* join = reinterpret_cast<f32x4*>(xs);
    if (cw > 0) join[(rw * CW + cw) * 64 + lane] = y;
    __syncthreads();
    if (cw > 0) return;
#pragma unroll
    for (int c = 1; c < CW; ++c) y += join[(rw * CW + c) * 64 + lane];
  }
  if (!live) return;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int m = quarter * 4 + e;
    if (m < tokens) static_cast<T*>(p.y)[(m0 + m) * p.ldy + row] = (T)y[e];
  }
}

template <typename T, int RW, int CW>
int launch_w4_as(W4Args a, void* stream, std::string* err) {
  const mg3m_w4& p = a.p;
  const long long groups = (long long)((p.K + 16 * RW - 1) / (16 * RW)) * ((p.M + 15) / 16);
  if (groups > 0x7fffffffLL) {
    *err = "4-bit product: too many rows for one launch";
    return MG3M_ERR_TOO_LARGE;
  }
  // x in LDS: all of it, or slabs that leave room for a second work-group
  const int unit_bytes = std::min(p.M, 16) * kUnit * 2 * W4Type<T>::kParts;
  const int units = (p.C + kUnit - 1) / kUnit;
  static_assert((CW & (CW - 1)) == 0, "slabs are a power of two");
  while (1 << a.slab_log2 < CW) ++a.slab_log2;
  while (1 << a.slab_log2 < units && (2 * unit_bytes) << a.slab_log2 <= 65536) ++a.slab_log2;
  const size_t lds = std::max<size_t>((size_t)unit_bytes << a.slab_log2, CW > 1 ? 8 * 64 * sizeof(f32x4) : 0);
  const bool whole = p.group % kUnit == 0;
  auto* kernel = whole ? matvec_w4<T, RW, CW, true> : matvec_w4<T, RW, CW, false>;
  kernel<<<(unsigned)groups, 512, lds, static_cast<hipStream_t>(stream)>>>(a);
  return launched("4-bit product", err);
}

}  // namespace

int launch_w4(const mg3m_w4& p, void* stream, std::string* err) {
  return with_dtype(p.dtype, [&](auto t) {
    using T = decltype(t);
    W4Args a{};
    a.p = p;
    a.vec = reinterpret_cast<uintptr_t>(p.x) % 16 == 0 && (p.ldx * sizeof(T)) % 16 == 0;
    // wide products share x between four tiles of rows
    const long long tiles = (long long)((p.K + 15) / 16) * ((p.M + 15) / 16);
    return tiles >= 1024 ? launch_w4_as<T, 4, 2>(a, stream, err) : launch_w4_as<T, 1, 8>(a, stream, err);
  });
}

}  // namespace mg3m
