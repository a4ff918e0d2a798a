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
// token together, permuted as the weights come out of a dword, and the rows'
// scales, as s and s (16 + zero); long rows in slabs.  A wave has four blocks
// of 128 channels of weights under way.
#include <type_traits>

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
  unsigned per_group;      // ceil(2^31 / (group / 32))

  // The group of a block of 32 channels: exact for block * (group / 32) below 2^31.
  __device__ __forceinline__ int group_of(int block) const { return (int)__umulhi(2u * block, per_group); }
};
constexpr int kMaxChannels = 1 << 20;

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
// consecutive channels, which lie in one group.  MT: tokens that LDS has room
// for, so that its addresses differ by constants.
template <typename T, int MT, int RW, int CW, bool WHOLE>
__global__ __launch_bounds__(512) void matvec_w4(W4Args a) {
  constexpr int kParts = W4Type<T>::kParts, kRows = 16 * RW;
  extern __shared__ u32x4 xs[];                  // [unit][part][16 blocks of 8 channels][MT], then ss
  const mg3m_w4& p = a.p;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int rw = wave / CW, cw = wave - rw * CW;
  const int col = lane & 15, quarter = lane >> 4;
  const int row_blocks = (p.K + kRows - 1) / kRows;
  const int mb = blockIdx.x / row_blocks, row0 = (int)(blockIdx.x - mb * row_blocks) * kRows;
  const int m0 = mb * 16, tokens = min(16, p.M - m0);
  const int row = row0 + rw * 16 + col;
  const int units = (p.C + kUnit - 1) / kUnit, groups = p.C / p.group;
  const unsigned char* q = p.q + (long long)min(row, p.K - 1) * (p.C / 2);
  const int token = min(col, tokens - 1);        // columns behind the last token repeat it
  const int slab = 1 << a.slab_log2, per_slab = slab / CW;      // per_slab: a multiple of kAhead
  float2* ss = reinterpret_cast<float2*>(xs + (kParts * 16 * MT << a.slab_log2));     // [group][row]

  // Four units of this wave from unit i of a slab; behind the end the row's
  // first bytes, against x = 0.
  auto load = [&](int unit0, int i, u32x4 (&w)[kAhead]) {
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int c = (unit0 + (i + k) * CW + cw) * kUnit + quarter * 32;
      w[k] = *reinterpret_cast<const u32x4*>(q + (c < p.C ? c / 2 : 0));
    }
  };

  // Four loads at a time; those behind the end repeat an element.
  auto stage_scales = [&](int group0, int here) {
    constexpr int kPer = 512 / kRows;            // threads on a row's scales
    const int k = threadIdx.x / kPer;
    const long long at = (long long)min(row0 + k, p.K - 1) * groups + group0;
    const unsigned char* zero = p.zero != nullptr ? p.zero : p.q;     // q: read, not used
    for (int g0 = threadIdx.x % kPer; g0 < here; g0 += 4 * kPer) {
      float s[4], z[4];
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        const int g = min(g0 + n * kPer, here - 1);
        s[n] = (float)static_cast<const T*>(p.scale)[at + g];
        z[n] = (float)zero[at + g];
      }
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        const float z16 = 16.0f + (p.zero != nullptr ? z[n] : 8.0f);
        if (g0 + n * kPer < here) ss[(g0 + n * kPer) * kRows + k] = float2{s[n], s[n] * z16};
      }
    }
  };
  // Channels behind the last one are zeros, to the slab's end.
  auto stage_x = [&](int unit0, auto vec) {
    const int row_log2 = a.slab_log2 + 4;
    for (int i0 = threadIdx.x; i0 < tokens << row_log2; i0 += 4 * 512) {
      T v[4][8];
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        const int i = i0 + n * 512, b = i & ((1 << row_log2) - 1);
        const int m = min(i >> row_log2, tokens - 1), c = min(unit0 * kUnit + b * 8, p.C - 8);
        const T* x = static_cast<const T*>(p.x) + (m0 + m) * p.ldx + c;
        if constexpr (decltype(vec)::value) {
#pragma unroll
          for (int k = 0; k < (int)sizeof(T) / 2; ++k)
            *reinterpret_cast<u32x4*>(v[n] + k * 16 / sizeof(T)) = reinterpret_cast<const u32x4*>(x)[k];
        } else {
#pragma unroll
          for (int k = 0; k < 8; ++k) v[n][k] = x[k];
        }
      }
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        const int i = i0 + n * 512, m = i >> row_log2, b = i & ((1 << row_log2) - 1);
        if (m >= tokens) continue;
        u32x4 o[kParts];
        arrange(v[n], o);
        const bool in = unit0 * kUnit + b * 8 < p.C;
#pragma unroll
        for (int part = 0; part < kParts; ++part)
          xs[((b / 16 * kParts + part) * 16 + b % 16) * MT + m] = in ? o[part] : u32x4{};
      }
    }
  };

  const u32x4 ones = {W4Type<T>::kOnes, W4Type<T>::kOnes, W4Type<T>::kOnes, W4Type<T>::kOnes};
  f32x4 y = {};
  int group0 = 0;                                // the slab's first group
  auto product = [&](int unit0, int in_slab, u32x4 v) {
    const u32x4* x = xs + in_slab * (kParts * 16 * MT) + quarter * (WHOLE ? 4 * MT : MT) + token;
    u32x4 xa[4][kParts];
    float2 s[WHOLE ? 1 : 4];
#pragma unroll
    for (int d = 0; d < 4; ++d) {
#pragma unroll
      for (int part = 0; part < kParts; ++part) xa[d][part] = x[(part * 16 + (WHOLE ? d : 4 * d)) * MT];
    }
#pragma unroll
    for (int d = 0; d < (WHOLE ? 1 : 4); ++d) {
      const int g = a.group_of(min((unit0 + in_slab) * 4 + d, p.C / 32 - 1)) - group0;
      s[d] = ss[g * kRows + rw * 16 + col];
    }
    if constexpr (!WHOLE) {
      const auto s02 = __builtin_amdgcn_permlane32_swap(v[0], v[2], false, false);
      const auto s13 = __builtin_amdgcn_permlane32_swap(v[1], v[3], false, false);
      const auto s01 = __builtin_amdgcn_permlane16_swap(s02[0], s13[0], false, false);
      const auto s23 = __builtin_amdgcn_permlane16_swap(s02[1], s13[1], false, false);
      v = u32x4{s01[0], s01[1], s23[0], s23[1]};
    }
    f32x4 dot = {}, sum = {};
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      const u32x4 b = expand<T>(v[d]);
#pragma unroll
      for (int part = 0; part < kParts; ++part) {
        dot = mfma<T>(xa[d][part], b, dot);
        sum = mfma<T>(xa[d][part], ones, sum);
      }
      if (!WHOLE || d == 3) {
        const float2 f = s[WHOLE ? 0 : d];
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = fmaf(f.x, dot[e], fmaf(-f.y, sum[e], y[e]));
        dot = sum = f32x4{};
      }
    }
  };
  for (int unit0 = 0; unit0 < units; unit0 += slab) {
    u32x4 w0[kAhead], w1[kAhead];
    load(unit0, 0, w0);
    group0 = a.group_of(unit0 * (kUnit / 32));
    const int end = min((min(unit0 + slab, units)) * kUnit, p.C);
    if (unit0 > 0) __syncthreads();
    stage_scales(group0, a.group_of(end / 32 - 1) - group0 + 1);
    if (a.vec) stage_x(unit0, std::true_type{});
    else stage_x(unit0, std::false_type{});
    __syncthreads();
    // this wave's units of the slab, with those of zeros that fill the last four
    const int mine = min(per_slab, (units - unit0 + CW - 1) / CW);
    for (int i = 0; i < mine; i += 2 * kAhead) {
      if (i + kAhead < mine) load(unit0, i + kAhead, w1);
#pragma unroll
      for (int k = 0; k < kAhead; ++k) product(unit0, (i + k) * CW + cw, w0[k]);
      if (i + kAhead >= mine) break;
      if (i + 2 * kAhead < mine) load(unit0, i + 2 * kAhead, w0);
#pragma unroll
      for (int k = 0; k < kAhead; ++k) product(unit0, (i + kAhead + k) * CW + cw, w1[k]);
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
  if (row >= p.K) return;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int m = quarter * 4 + e;
    if (m < tokens) static_cast<T*>(p.y)[(m0 + m) * p.ldy + row] = (T)y[e];
  }
}

template <typename T, int MT, int RW, int CW>
int launch_w4_as(W4Args a, void* stream, std::string* err) {
  const mg3m_w4& p = a.p;
  const long long groups = (long long)((p.K + 16 * RW - 1) / (16 * RW)) * ((p.M + 15) / 16);
  if (groups > 0x7fffffffLL) {
    *err = "4-bit product: too many rows for one launch";
    return MG3M_ERR_TOO_LARGE;
  }
  // x and scales in LDS: all of them, or slabs that leave room for a second work-group
  const int x_unit = MT * kUnit * 2 * W4Type<T>::kParts;
  const int units = (p.C + kUnit - 1) / kUnit;
  const auto bytes = [&](int log2) {
    return ((size_t)x_unit << log2) + (((size_t)kUnit << log2) / p.group + 2) * 16 * RW * sizeof(float2);
  };
  while (1 << a.slab_log2 < CW * kAhead) ++a.slab_log2;
  while (1 << a.slab_log2 < units && bytes(a.slab_log2 + 1) <= 65536) ++a.slab_log2;
  const size_t lds = std::max<size_t>(bytes(a.slab_log2), CW > 1 ? 8 * 64 * sizeof(f32x4) : 0);
  auto* kernel = p.group % kUnit == 0 ? matvec_w4<T, MT, RW, CW, true> : matvec_w4<T, MT, RW, CW, false>;
  kernel<<<(unsigned)groups, 512, lds, static_cast<hipStream_t>(stream)>>>(a);
  return launched("4-bit product", err);
}

template <typename T, int MT>
int launch_w4_mt(const W4Args& a, long long tiles, void* stream, std::string* err) {
  if (tiles >= 1024 || MT * W4Type<T>::kParts > 16) return launch_w4_as<T, MT, 4, 2>(a, stream, err);
  return launch_w4_as<T, MT, 1, 8>(a, stream, err);
}

}  // namespace

int launch_w4(const mg3m_w4& p, void* stream, std::string* err) {
  if (p.C > kMaxChannels) {
    *err = "4-bit product: more than 2^20 channels";
    return MG3M_ERR_TOO_LARGE;
  }
  return with_dtype(p.dtype, [&](auto t) {
    using T = decltype(t);
    W4Args a{};
    a.p = p;
    a.vec = reinterpret_cast<uintptr_t>(p.x) % 16 == 0 && (p.ldx * sizeof(T)) % 16 == 0;
    const unsigned blocks = p.group / 32;
    a.per_group = ((1u << 31) + blocks - 1) / blocks;
    // wide products share x between four tiles of rows
    const long long tiles = (long long)((p.K + 15) / 16) * ((p.M + 15) / 16);
    return p.M == 1 ? launch_w4_mt<T, 1>(a, tiles, stream, err)
           : p.M <= 4 ? launch_w4_mt<T, 4>(a, tiles, stream, err) : launch_w4_mt<T, 16>(a, tiles, stream, err);
  });
}

}  // namespace mg3m
