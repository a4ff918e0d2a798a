// Products of few tokens with 4-bit weights (include/mg3m_seq.h).
//
// Bound by the weights' bytes: with one token each weight is used once, with
// 16 still only 16 times.  What has to be cheap is a weight's way from four
// bits to a product.  Shifted so that a nibble is the top of a 16-bit float's
// mantissa under the exponent of 16, w & mask | exponent is the pair of numbers
// 16 + q, exact in bf16 and in fp16: two instructions for two weights.  The 16
// and the zero point leave the sum through a second one, of the tokens alone,
//   sum x (q - zero) = sum x (16 + q) - (16 + zero) sum x,
// whose terms are up to 31/8 the size of the result's.  That takes two of fp32's
// 24 bits, far below the 8 or 11 that a 16-bit result keeps.  fp32 tokens, whose
// result would show it, meet q - zero.
#include <type_traits>

#include "seq_device.h"

namespace mg3m {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr int kUnit = 128;          // channels per wave and step: 16 bytes of weights per lane

struct W4Args {
  mg3m_w4 p;
  int slab_log2;           // units of x in LDS
  int vec;                 // x rows are 16-byte aligned
  unsigned per_group;      // ceil(2^31 / (group / 32))

  // The group of a block of 32 channels: exact for block * (group / 32) below 2^31.
  __device__ __forceinline__ int group_of(int block) const { return (int)__umulhi(2u * block, per_group); }
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

// The eight weights of a dword as 16 + q, in the order 0 4 1 5 2 6 3 7.  mask
// and sixteen come in registers: with two literals the compiler takes an
// instruction more for each pair.
template <typename T>
__device__ __forceinline__ u32x4 expand(unsigned w, unsigned mask, unsigned sixteen) {
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int by = 4 * i - W4Type<T>::kShift;
    r[i] = ((by < 0 ? w << -by : w >> by) & mask) | sixteen;
  }
  return r;
}

// The eight weights as q - zero, exact in bf16, in the same order.
__device__ __forceinline__ u32x4 expand_exact(unsigned w, float zero) {
  const unsigned even = w & 0x0f0f0f0fu, odd = (w >> 4) & 0x0f0f0f0fu;
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const unsigned bytes = i % 2 == 0 ? even : odd;
    const unsigned lo = __builtin_bit_cast(unsigned, (float)((bytes >> (8 * (i / 2))) & 255u) - zero);
    const unsigned hi = __builtin_bit_cast(unsigned, (float)((bytes >> (8 * (i / 2) + 16)) & 255u) - zero);
    r[i] = lo >> 16 | (hi & 0xffff0000u);
  }
  return r;
}

// Lanes of a wave that exchange values through LDS: the wave's LDS accesses
// are carried out in order, and the compiler keeps theirs.
__device__ __forceinline__ void wave_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_sched_barrier(0);
}

__device__ __forceinline__ unsigned pack2(unsigned short lo, unsigned short hi) { return lo | (unsigned)hi << 16; }

// Eight channels of a token as the MFMA takes them, in `parts` registers sets:
// fp32 as three bf16 parts, the upper 16 bits of what is left each time (exact,
// as in conv_b3.h).
template <typename T>
__device__ __forceinline__ void arrange(const T (&v)[8], u32x4 (&out)[W4Type<T>::kParts]) {
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      out[0][i] = pack2(__builtin_bit_cast(unsigned short, v[i]), __builtin_bit_cast(unsigned short, v[i + 4]));
  } else {
    float r[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = v[i];
#pragma unroll
    for (int q = 0; q < 3; ++q) {
      unsigned top[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        top[i] = __builtin_bit_cast(unsigned, r[i]) & 0xffff0000u;
        r[i] -= __builtin_bit_cast(float, top[i]);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) out[q][i] = top[i] >> 16 | top[i + 4];
    }
  }
}

// More tokens, on the matrix cores.  v_mfma_f32_16x16x32 takes 16
// tokens (rows) times 16 weight rows (columns); a lane holds eight consecutive
// channels of a row, which is one dword of weights.
//
// A wave takes a tile of 16 rows and four units of 128 channels at a time, 256
// bytes of each row.  It loads them row by row, whole cache lines, and turns
// them through LDS of its own: loaded as the MFMA takes them, 64 bytes of 16
// rows at once, they came from one channel of the L2 cache wherever rows are a
// multiple of 4 KB apart (13 tokens, 8192 to 24576 channels: 54 us).
//
// A work-group has RW times CW waves: tiles of rows and slices of the channels,
// which are joined through LDS in a fixed order.  It keeps x in LDS
// as the MFMA takes it, and the rows' scales, as s and s (16 + zero); long rows
// in slabs.  fp32 tokens, whose three parts keep the matrix cores busier than
// the ALU, meet q - zero itself: no second product, and none of the bits that
// the 16 costs (relative error at 4096 channels: 1.5e-7 for 1.5e-6).  WHOLE: a group covers whole units.  Otherwise the lanes' dwords
// are transposed (lane quarter against dword), after which an MFMA covers 32
// consecutive channels, which lie in one group.
template <typename T, int RW, int CW, bool WHOLE>
__global__ __launch_bounds__(64 * RW * CW, sizeof(T) == 2 && RW == 4 ? 4 : 1) void matvec_w4(W4Args a) {
  constexpr int MT = 16;                         // tokens of an MFMA
  constexpr int kParts = W4Type<T>::kParts, kRows = 16 * RW, kWaves = RW * CW, kThreads = 64 * kWaves;
  constexpr bool kExact = kParts == 3;           // q - zero itself
  // Work-groups with a unit to themselves and registers to spare load x's first
  // round of a slab (and with eight waves the scales') a slab ahead: 12288 rows of
  // 8192 channels, 16 bf16 tokens: 21.4 us to 19.2; 8192 rows: 17.5 to 15.5.
  constexpr bool kAlone = kParts == 1 && RW != 4;
  constexpr int kAhead = kAlone ? 1 : 0, kScalesAhead = kAlone && kWaves == 8 ? 1 : 0;
  extern __shared__ u32x4 lds[];
  const mg3m_w4& p = a.p;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int rw = wave / CW, cw = wave - rw * CW;
  const int col = lane & 15, quarter = lane >> 4;
  const int row_blocks = (p.K + kRows - 1) / kRows;
  const int mb = blockIdx.x / row_blocks, row0 = (int)(blockIdx.x - mb * row_blocks) * kRows;
  const int m0 = mb * 16, tokens = min(MT, p.M - m0);
  const int row = row0 + rw * 16 + col;
  const int units = (p.C + kUnit - 1) / kUnit, groups = p.C / p.group;
  const int token = min(col, tokens - 1);        // columns behind the last token repeat it
  const int slab = 1 << a.slab_log2;             // units, a multiple of 4 CW
  // Token m of block b lies at place m ^ b: lanes that write one token's blocks
  // and lanes that read one block's tokens both reach all banks.
  int x_lane[4];
#pragma unroll
  for (int d = 0; d < 4; ++d) {
    const int b = WHOLE ? quarter * 4 + d : d * 4 + quarter;
    x_lane[d] = b * MT + (token ^ b);
  }
  u32x4* wt = lds + wave * 256;                  // [row][16 pieces of 16 bytes]
  u32x4* xs = lds + kWaves * 256;                     // [unit][part][16 blocks of 8 channels][MT]
  float2* ss = reinterpret_cast<float2*>(xs + (kParts * 16 * MT << a.slab_log2));     // [group][row]

  // Four units from channel c0 on: 16 lanes on a row, four rows at a time;
  // behind the channels' end the row's last 16 bytes, against x = 0.
  const unsigned row_bytes = p.C / 2;
  const unsigned char* q = p.q + (long long)row0 * row_bytes;
  unsigned q_lane[4];                            // below 2^26
#pragma unroll
  for (int n = 0; n < 4; ++n) q_lane[n] = (min(row0 + rw * 16 + n * 4 + quarter, p.K - 1) - row0) * row_bytes;
  auto load = [&](unsigned c0, u32x4 (&w)[4]) {
    const unsigned at = min(c0 / 2 + col * 16, row_bytes - 16);
#pragma unroll
    for (int n = 0; n < 4; ++n) w[n] = *reinterpret_cast<const u32x4*>(q + (q_lane[n] + at));
  };

  // Scales and x go to LDS in rounds of four loads by every thread; those
  // behind the end repeat an element.
  constexpr int kPer = kThreads / kRows;         // threads on a row's scales
  const unsigned char* zero = p.zero != nullptr ? p.zero : p.q;       // q: read, not used
  const auto load_scales = [&](int group0, int here, int g0, T (&s)[4], unsigned char (&z)[4]) {
    const long long at = (long long)min(row0 + (int)threadIdx.x / kPer, p.K - 1) * groups + group0;
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const int g = min(g0 + n * kPer, here - 1);
      s[n] = static_cast<const T*>(p.scale)[at + g];
      z[n] = zero[at + g];
    }
  };
  const auto put_scales = [&](int here, int g0, const T (&s)[4], const unsigned char (&z)[4]) {
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const float sr = (float)s[n], zr = p.zero != nullptr ? (float)z[n] : 8.0f;
      if (g0 + n * kPer < here)
        ss[(g0 + n * kPer) * kRows + threadIdx.x / kPer] = float2{sr, kExact ? zr : sr * (16.0f + zr)};
    }
  };
  const int row_log2 = a.slab_log2 + 4, items = tokens << row_log2;
  constexpr int kRaw = sizeof(T) / 2;            // 16 bytes each of eight channels
  const auto load_x = [&](int unit0, int i0, u32x4 (&v)[4][kRaw]) {
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const int i = i0 + n * kThreads, b = i & ((1 << row_log2) - 1);
      const int m = min(i >> row_log2, tokens - 1), c = min(unit0 * kUnit + b * 8, p.C - 8);
      const T* x = static_cast<const T*>(p.x) + (m0 + m) * p.ldx + c;
#pragma unroll
      for (int k = 0; k < kRaw; ++k) {
        const T* at = x + k * 16 / sizeof(T);
        if (a.vec) v[n][k] = *reinterpret_cast<const u32x4*>(at);
        else __builtin_memcpy(&v[n][k], at, 16);
      }
    }
  };
  // Channels behind the last one are zeros, to the slab's end.
  const auto put_x = [&](int unit0, int i0, const u32x4 (&raw)[4][kRaw]) {
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const int i = i0 + n * kThreads, m = i >> row_log2, b = i & ((1 << row_log2) - 1);
      if (m >= tokens) continue;
      T v[8];
      __builtin_memcpy(v, raw[n], sizeof(v));
      u32x4 o[kParts];
      arrange(v, o);
      const bool in = unit0 * kUnit + b * 8 < p.C;
#pragma unroll
      for (int part = 0; part < kParts; ++part)
        xs[((b / 16 * kParts + part) * 16 + b % 16) * MT + (m ^ b % 16)] = in ? o[part] : u32x4{};
    }
  };

  unsigned mask = 0x000f000fu << W4Type<T>::kShift, sixteen = W4Type<T>::kSixteen;
  asm("" : "+s"(mask));
  asm("" : "+v"(sixteen));
  const u32x4 ones = {W4Type<T>::kOnes, W4Type<T>::kOnes, W4Type<T>::kOnes, W4Type<T>::kOnes};
  f32x4 y = {};
  int group0 = 0;                                // the slab's first group
  // Two units side by side: an MFMA's result is there for the next one of its
  // sum when the other three sums have had theirs.
  auto product = [&](int unit0, int in_slab, int piece) {
    u32x4 xa[2][4][kParts], v[2];
    float2 s[2][WHOLE ? 1 : 4];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      v[u] = wt[col * 16 + ((piece + u * 4 + quarter) ^ col)];
      const u32x4* x = xs + (in_slab + u) * (kParts * 16 * MT);
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int part = 0; part < kParts; ++part) xa[u][d][part] = x[part * 16 * MT + x_lane[d]];
#pragma unroll
      for (int d = 0; d < (WHOLE ? 1 : 4); ++d) {
        const int g = a.group_of(min((unit0 + in_slab + u) * 4 + d, p.C / 32 - 1)) - group0;
        s[u][d] = ss[g * kRows + rw * 16 + col];
      }
    }
    __builtin_amdgcn_sched_barrier(0);           // the reads first
    if constexpr (!WHOLE) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const auto s02 = __builtin_amdgcn_permlane32_swap(v[u][0], v[u][2], false, false);
        const auto s13 = __builtin_amdgcn_permlane32_swap(v[u][1], v[u][3], false, false);
        const auto s01 = __builtin_amdgcn_permlane16_swap(s02[0], s13[0], false, false);
        const auto s23 = __builtin_amdgcn_permlane16_swap(s02[1], s13[1], false, false);
        v[u] = u32x4{s01[0], s01[1], s23[0], s23[1]};
      }
    }
    f32x4 dot[2] = {}, sum[2] = {};
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      u32x4 b[2];
#pragma unroll
      for (int u = 0; u < 2; ++u)
        b[u] = kExact ? expand_exact(v[u][d], s[u][WHOLE ? 0 : d].y) : expand<T>(v[u][d], mask, sixteen);
#pragma unroll
      for (int part = 0; part < kParts; ++part)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          dot[u] = mfma<T>(xa[u][d][part], b[u], dot[u]);
          if constexpr (!kExact) sum[u] = mfma<T>(xa[u][d][part], ones, sum[u]);
        }
      if (!WHOLE || d == 3) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const float2 f = s[u][WHOLE ? 0 : d];
#pragma unroll
          for (int e = 0; e < 4; ++e)
            y[e] = kExact ? fmaf(f.x, dot[u][e], y[e]) : fmaf(f.x, dot[u][e], fmaf(-f.y, sum[u][e], y[e]));
          dot[u] = sum[u] = f32x4{};
        }
      }
    }
  };
  u32x4 x_next[4][kRaw];
  T s_next[4];
  unsigned char z_next[4];
  const auto ahead = [&](int unit0) {
    const int first = a.group_of(unit0 * (kUnit / 32)), end = min(min(unit0 + slab, units) * kUnit, p.C);
    if (kScalesAhead > 0) load_scales(first, a.group_of(end / 32 - 1) - first + 1, threadIdx.x % kPer, s_next, z_next);
    load_x(unit0, threadIdx.x, x_next);
  };
  if (kAhead > 0) ahead(0);
  for (int unit0 = 0; unit0 < units; unit0 += slab) {
    // this wave's fours of units in the slab: i * CW + cw
    const int fours = (min(slab, units - unit0) + 4 * CW - 1) / (4 * CW);
    auto first = [&](int i) { return (unsigned)(unit0 + (i * CW + cw) * 4) * kUnit; };
    u32x4 w[4];
    load(first(0), w);
    group0 = a.group_of(unit0 * (kUnit / 32));
    const int end = min((min(unit0 + slab, units)) * kUnit, p.C);
    const int here = a.group_of(end / 32 - 1) - group0 + 1, g0 = threadIdx.x % kPer, t0 = threadIdx.x;
    if (unit0 > 0) __syncthreads();
    if (kScalesAhead > 0) put_scales(here, g0, s_next, z_next);
    if (kAhead > 0) put_x(unit0, t0, x_next);
    for (int g = g0 + kScalesAhead * 4 * kPer; g < here; g += 4 * kPer) {
      T s[4];
      unsigned char z[4];
      load_scales(group0, here, g, s, z);
      put_scales(here, g, s, z);
    }
    for (int i = t0 + kAhead * 4 * kThreads; i < items; i += 4 * kThreads) {
      u32x4 v[4][kRaw];
      load_x(unit0, i, v);
      put_x(unit0, i, v);
    }
    __syncthreads();
    if (kAhead > 0 && unit0 + slab < units) ahead(unit0 + slab);
    for (int i = 0; i < fours; ++i) {
#pragma unroll
      for (int n = 0; n < 4; ++n) wt[(n * 4 + quarter) * 16 + (col ^ (n * 4 + quarter))] = w[n];
      wave_order();
      load(first(min(i + 1, fours - 1)), w);     // the last one again: not under a condition
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int k = 0; k < 4; k += 2) product(unit0, (i * CW + cw) * 4 + k, k * 4);
      wave_order();                              // the next four's writes after these reads
    }
  }

  if constexpr (CW > 1) {
    __syncthreads();
    f32x4* join = reinterpret_cast<f32x4*>(lds);
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

template <typename T, int RW, int CW>
int launch_w4_many(W4Args a, void* stream, std::string* err) {
  const mg3m_w4& p = a.p;
  const long long groups = (long long)((p.K + 16 * RW - 1) / (16 * RW)) * ((p.M + 15) / 16);
  if (!fits_launch(groups, 64 * RW * CW)) {
    *err = "4-bit product: too many rows for one launch";
    return MG3M_ERR_TOO_LARGE;
  }
  // LDS: the waves' weights (4 KB each), x and scales, all or slabs: of up to 48
  // KB, so that two work-groups fit, or of all there is where one has the unit
  // (24576 rows of 8192 channels, 13 bf16 tokens: 34 us to 28), and at least
  // what CW slices take (145 KB at most: 16 bits, 4 tiles of 4 slices, groups of
  // 64; fp32, groups of 32)
  const int units = (p.C + kUnit - 1) / kUnit;
  const auto bytes = [&](int log2) {
    return ((size_t)(16 * kUnit * 2 * W4Type<T>::kParts) << log2) +
           (((size_t)kUnit << log2) / p.group + 2) * 16 * RW * sizeof(float2);
  };
  while (1 << a.slab_log2 < 4 * CW) ++a.slab_log2;
  const size_t most = RW * CW > 8 ? 163840 - 4096 * RW * CW : 49152;
  while (1 << a.slab_log2 < units && bytes(a.slab_log2 + 1) <= most) ++a.slab_log2;
  auto* kernel = p.group % kUnit == 0 ? matvec_w4<T, RW, CW, true> : matvec_w4<T, RW, CW, false>;
  kernel<<<(unsigned)groups, 64 * RW * CW, 4096 * RW * CW + bytes(a.slab_log2), static_cast<hipStream_t>(stream)>>>(a);
  return launched("4-bit product", err);
}

// Few tokens, or few rows, on the vector ALU: no x in LDS and no barrier, which
// for these cost more than the products.  M tokens to a wave; a row's blocks of 32 channels (16
// bytes) go to consecutive lanes, so loads are whole cache lines; a lane keeps
// its channels of the tokens for kRowsPer rows.  16-bit tokens multiply the
// pairs 16 + q with a two-element dot product (12 instructions for 8 weights
// and a token, 4 for each further token).  fp32 ones multiply q - zero itself,
// so that what leaves the sum does not round in it: bits 4 i .. 4 i + 3 of an
// fp32 mantissa under the exponent of 2^(23 - 4 i) are that power plus q, and
// the power plus zero, exact as well, is taken off (one token, 24576 rows of 8192
// channels: 34.8 us; q out of a byte, the zero taken off the sum: 37.5; relative
// error at 4096 channels 1.2e-7 for 4.9e-7).
constexpr int kRowsPer = 4;

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

template <typename T>
__device__ __forceinline__ float dot2(unsigned a, unsigned b, float c) {
  if constexpr (W4Type<T>::kShift == 6)
    return __builtin_amdgcn_fdot2(__builtin_bit_cast(f16x2, a), __builtin_bit_cast(f16x2, b), c, false);
  else
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, a), __builtin_bit_cast(bf16x2, b), c, false);
}

template <typename T, int M>
__global__ __launch_bounds__(256) void matvec_w4_few(W4Args a, int lanes_log2) {
  constexpr bool kHalf = sizeof(T) == 2;
  const mg3m_w4& p = a.p;
  const int lanes = 1 << lanes_log2;             // on a row
  const int lane = threadIdx.x & (lanes - 1);
  const int row0 = (int)((blockIdx.x * 256u + threadIdx.x) >> lanes_log2) * kRowsPer;
  const int m0 = blockIdx.y * M, last = p.M - 1 - m0;
  const T* tokens = static_cast<const T*>(p.x) + m0 * p.ldx;
  const int blocks = p.C / 32, groups = p.C / p.group;
  const unsigned char* zero = p.zero != nullptr ? p.zero : p.q;      // q: read, not used
  unsigned mask = 0x000f000fu << W4Type<T>::kShift, sixteen = W4Type<T>::kSixteen;
  asm("" : "+s"(mask));
  asm("" : "+v"(sixteen));
  unsigned place[4], high[4];                    // of fp32 tokens' weights, in registers as above
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    place[i] = 15u << (4 * i);
    high[i] = (127u + 23 - 4 * i) << 23;
    asm("" : "+s"(place[i]));
    asm("" : "+v"(high[i]));
  }
  float y[kRowsPer][M] = {};
  for (int b = lane; b < blocks; b += lanes) {
    u32x4 w[kRowsPer];
    float s[kRowsPer], z[kRowsPer];
    const int g = a.group_of(b);
#pragma unroll
    for (int r = 0; r < kRowsPer; ++r) {
      const long long row = min(row0 + r, p.K - 1);
      w[r] = reinterpret_cast<const u32x4*>(p.q + row * (p.C / 2))[b];
      s[r] = (float)static_cast<const T*>(p.scale)[row * groups + g];
      z[r] = (float)zero[row * groups + g];
    }
#pragma unroll
    for (int m = 0; m < M; ++m) {
      const T* x = tokens + min(m, last) * p.ldx + b * 32;
      T v[32];
      if (a.vec) {
#pragma unroll
        for (int k = 0; k < 2 * (int)sizeof(T); ++k)
          *reinterpret_cast<u32x4*>(v + k * 16 / sizeof(T)) = reinterpret_cast<const u32x4*>(x)[k];
      } else {
#pragma unroll
        for (int k = 0; k < 32; ++k) v[k] = x[k];
      }
      if constexpr (kHalf) {
        float sum = 0.0f;
        unsigned pair[16];
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            pair[d * 4 + i] = pack2(__builtin_bit_cast(unsigned short, v[d * 8 + i]),
                                    __builtin_bit_cast(unsigned short, v[d * 8 + i + 4]));
            sum = dot2<T>(pair[d * 4 + i], W4Type<T>::kOnes, sum);
          }
#pragma unroll
        for (int r = 0; r < kRowsPer; ++r) {
          float dot = 0.0f;
#pragma unroll
          for (int d = 0; d < 4; ++d) {
            const u32x4 e = expand<T>(w[r][d], mask, sixteen);
#pragma unroll
            for (int i = 0; i < 4; ++i) dot = dot2<T>(pair[d * 4 + i], e[i], dot);
          }
          const float z16 = 16.0f + (p.zero != nullptr ? z[r] : 8.0f);
          y[r][m] = fmaf(s[r], fmaf(-z16, sum, dot), y[r][m]);
        }
      } else {
#pragma unroll
        for (int r = 0; r < kRowsPer; ++r) {
          const float zr = p.zero != nullptr ? z[r] : 8.0f;
          float dot = 0.0f;
#pragma unroll
          for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const unsigned bits = ((i < 4 ? w[r][d] : w[r][d] >> 16) & place[i & 3]) | high[i & 3];
              const float off = zr + (float)(1 << (23 - 4 * (i & 3)));
              dot = fmaf(v[d * 8 + i], __builtin_bit_cast(float, bits) - off, dot);
            }
          y[r][m] = fmaf(s[r], dot, y[r][m]);
        }
      }
    }
  }
  for (int o = 1; o < lanes; o *= 2)
#pragma unroll
    for (int r = 0; r < kRowsPer; ++r)
#pragma unroll
      for (int m = 0; m < M; ++m) y[r][m] += __shfl_xor(y[r][m], o);
  if (lane != 0) return;
#pragma unroll
  for (int r = 0; r < kRowsPer; ++r)
#pragma unroll
    for (int m = 0; m < M; ++m)
      if (row0 + r < p.K && m <= last) static_cast<T*>(p.y)[(m0 + m) * p.ldy + row0 + r] = (T)y[r][m];
}

template <typename T, int M>
int launch_w4_few(const W4Args& a, void* stream, std::string* err) {
  const mg3m_w4& p = a.p;
  int lanes_log2 = 0;
  while (lanes_log2 < 6 && 32 << lanes_log2 < p.C) ++lanes_log2;
  const long long groups = (((long long)((p.K + kRowsPer - 1) / kRowsPer) << lanes_log2) + 255) / 256;
  if (!fits_launch(groups, 256)) {
    *err = "4-bit product: too many rows for one launch";
    return MG3M_ERR_TOO_LARGE;
  }
  const dim3 grid((unsigned)groups, (unsigned)((p.M + M - 1) / M));
  matvec_w4_few<T, M><<<grid, 256, 0, static_cast<hipStream_t>(stream)>>>(a, lanes_log2);
  return launched("4-bit product", err);
}

}  // namespace

int launch_w4(const mg3m_w4& p, void* stream, std::string* err) {
  return with_dtype(p.dtype, [&](auto t) {
    using T = decltype(t);
    W4Args a{};
    a.p = p;
    a.vec = reinterpret_cast<uintptr_t>(p.x) % 16 == 0 && (p.ldx * sizeof(T)) % 16 == 0;
    const unsigned blocks = p.group / 32;
    a.per_group = ((1u << 31) + blocks - 1) / blocks;
    // Tokens by the vector ALU or the matrix cores: 2 of bf16, 8192 to 24576
    // channels: 32 us against 35.  More of them while each wave of four rows and
    // four tokens has a SIMD of its own and rows are long, so that what counts is
    // how long one takes: 4096 to 1024 channels, 16 tokens of bf16: 7.9 us
    // against 9.7, of fp32 (three parts): 13 against 22.  Past either: 4096 to
    // 2048, 16 of bf16: 10.5 against 9.8; 2048 to 1024, 4 of bf16: 5.5 against
    // 5.2; 512 to 64, 8 of fp32: 7.6 against 6.4.
    if (p.M == 1) return launch_w4_few<T, 1>(a, stream, err);
    if (p.M == 2) return launch_w4_few<T, 2>(a, stream, err);
    const long long waves = (long long)((p.K + kRowsPer - 1) / kRowsPer) * ((p.M + 3) / 4);
    if (waves <= 1024 && p.C * sizeof(T) >= 8192) return launch_w4_few<T, 4>(a, stream, err);
    // One work-group to each of the 256 compute units, with the fewest rows that
    // do: all of them run the same time and x is staged once per unit (12288
    // rows of 4096 channels, 13 bf16 tokens: 3 tiles 9.9 us, 2: 17.2; 16384 of
    // 8192, 16: 4 tiles of four slices 24.0, of two 27.5; 24576, 13: 6 tiles 27,
    // 4: 39).  Beyond, four tiles, two work-groups to a unit (32768, 16: 42 us,
    // 6 tiles: 60).  Rows too short for four slices: two (1024 channels, 4096
    // rows: 5.0 us against 5.7; 1536, 12288: 7.5 against 6.6).  LDS holds neither
    // the parts of fp32 tokens for four slices or six tiles nor sixteen waves'
    // weights beside scales of 32.
    if constexpr (sizeof(T) == 2) {
      const auto one_each = [&](int rw) {
        return (long long)((p.K + 16 * rw - 1) / (16 * rw)) * ((p.M + 15) / 16) <= 256;
      };
      if (p.C > 11 * kUnit) {
        if (one_each(2)) return launch_w4_many<T, 2, 4>(a, stream, err);
        if (one_each(3)) return launch_w4_many<T, 3, 4>(a, stream, err);
        if (one_each(4) && p.group > 32) return launch_w4_many<T, 4, 4>(a, stream, err);
        if (!one_each(4) && one_each(6)) return launch_w4_many<T, 6, 2>(a, stream, err);
      }
    }
    return launch_w4_many<T, 4, 2>(a, stream, err);
  });
}

}  // namespace mg3m
