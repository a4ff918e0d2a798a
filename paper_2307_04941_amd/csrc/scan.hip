// Selective state space scan (include/mg3m_seq.h): how a prompt is dealt out,
// the small kernels around scan_pieces (scan_kernel.h), single tokens.
#include "scan.h"

namespace mg3m {
namespace {

struct ScanPlan {
  int P, F;      // states per wave, waves
  int W;         // tokens per piece, 0: whole sequences
};

constexpr int pow2_at_least(int v) {
  int p = 1;
  while (p < v) p *= 2;
  return p;
}

// How many states a wave takes, and whether sequences are cut.
//
// Two states per wave and eight waves fill the registers least and share the
// per-channel work best up to S = 16; more states go to more waves, sixteen at
// most.  Where there are more than two work-groups to a compute unit anyway,
// four states per wave cost less in shared work if that leaves four waves (16
// sequences of 512, S = 16, 256 to 512 work-groups: 59 to 80 us with two states,
// 71 to 84 with four; 768: 116, 111; 2048: 284, 267; but S = 8, 2048: 200, 239).
// The same holds for pieces (two and four states, S = 16, by work-groups: one
// sequence of 2000, D = 2048, 500: 49 and 52 us; of 2300, 575: 66, 65; four ragged
// ones of 2000 together, 500: 52, 53; of 2300, 575: 65, 63), but for few ragged
// ones in pieces of 256 (2300, D = 4096, 575: 98, 107; 4100, 1025: 145, 151).
//
// A work-group walks a whole sequence if that gives nearly every compute unit
// one (4 of 4096, D = 4096: 397 us whole, 469 cut, though the cut one computes
// nearly all decays twice).  Else sequences are cut into about two pieces per
// compute unit: not under 32 tokens, where the kernels' start counts, nor over
// 256, nor, up to 32768 tokens, into more than 128 pieces, which are joined one
// after the other (1 of 2048, D = 2048: 49 us in pieces of 128, 54 of 64 or of
// 256, 280 whole; 1 of 8192, D = 64: 35 in pieces of 64, 43 of 32, 39 of 128; 1 of
// 70000, 274 pieces: 111, 30 of them the join).  Where the host does not know
// the lengths, the longest sequence may be several times the average, so more
// sequences and channels are cut (12 to 19 sequences of 470 to 900 on average,
// 230 to 340 work-groups whole: 140 to 206 us whole, 115 to 142 cut; 392 against
// 158 with 1800 on average; 8 that are equal, 256 work-groups, lose: 99 against
// 131; and 416: 147 against 170).
ScanPlan scan_plan(int T, int D, int G, int S, int N, bool equal) {
  const double blocks = (double)G * ((D / G + 63) / 64), groups = N * blocks;
  // the longest sequence; unknown lengths: four times the average
  const double longest = equal ? T / N : std::min<double>(T, 4.0 * T / N + 1);
  ScanPlan s{};
  double all = groups;                 // work-groups that have something to do
  if (groups < (equal ? 224 : 352)) {
    s.W = 32;
    while (s.W < 256 && (s.W < T * blocks / 600 || s.W < longest / 128)) s.W *= 2;
    if (s.W >= longest) s.W = 0;
    else all = T * blocks / s.W;
  }
  s.P = S <= 8 ? 2 : S <= 16 ? (all > 512 ? 4 : 2) : S <= 32 ? 4 : S <= 128 ? 8 : 16;
  s.F = std::max(2, pow2_at_least((S + s.P - 1) / s.P));
  return s;
}

size_t round16(size_t v) { return (v + 255) / 256 * 256; }

struct ScanSpace {
  size_t bc, slots, sums;      // bytes
  size_t total() const { return bc + slots + sums; }
};
ScanSpace scan_space(const ScanPlan& s, int T, int D, int G, int S, int N, bool equal) {
  const int some = 0;
  ScanSpace m{};
  m.bc = round16(8ull * G * s.F * s.P * T + 128);     // the last tile reads 128 bytes ahead
  if (s.W != 0) {
    const size_t ids = (size_t)piece_count(equal ? nullptr : &some, N, T, s.W);
    m.slots = round16(4ull * ids * D * S);
    m.sums = round16(4ull * ids * D);
  }
  return m;
}

// bc[g][f][t][2][P] = B, C of the states f * P .. in fp32, zeros behind S: a
// state behind S stays zero and adds zero.
template <typename T>
__global__ __launch_bounds__(256) void scan_pack(ScanArgs a, float* bc, int P, int F) {
  const long long all = 2ll * P * a.p.T * a.p.G * F;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < all; i += (long long)gridDim.x * 256) {
    const int w = (int)(i % (2 * P));
    const long long row = i / (2 * P);
    const int t = (int)(row % a.p.T);
    const int gf = (int)(row / a.p.T);
    const int g = gf / F, s = (gf - g * F) * P + (w < P ? w : w - P);
    float v = 0.0f;
    if (s < a.p.S)
      v = w < P ? (float)static_cast<const T*>(a.p.B)[t * a.p.ldb + g * a.p.S + s]
                : (float)static_cast<const T*>(a.p.C)[t * a.p.ldc + g * a.p.S + s];
    bc[i] = v;
  }
}

// The states that a sequence's pieces start from: the first one's is the
// sequence's, the next one's the piece's end state with what is left of its
// start, exp(A * sum of its step sizes).  slots: end states in, start states
// out.
__global__ __launch_bounds__(256) void scan_join(ScanArgs a) {
  const mg3m_scan& p = a.p;
  const int i = blockIdx.x * 256 + threadIdx.x, n = blockIdx.y;
  if (i >= p.D * p.S) return;
  const int s = i / p.D, d = i - s * p.D;
  const SeqRange r = seq_range(p.begin, p.end, n, p.N, p.T);
  const int pieces = max(1, ceil_div(r.e - r.b, a.W));
  const long long id0 = p.begin == nullptr ? (long long)n * pieces : piece_base(p.begin, n, p.T, a.W);
  const float A = p.A[(long long)d * p.S + s] * kLog2e;
  float h = p.load_state ? p.state[((long long)n * p.D + d) * p.S + s] : 0.0f;
  float* slot = a.slots + (id0 * p.S + s) * p.D + d;
  const float* sum = a.sums + id0 * p.D + d;
  const long long step = (long long)p.S * p.D;
  // Eight pieces' loads at once (16 pieces one after the other: 7.3 us, so:
  // 4.2); those behind the last repeat it and are not used.
  constexpr int kAt = 8;
  for (int k0 = 0; k0 < pieces; k0 += kAt) {
    float end[kAt], left[kAt];
#pragma unroll
    for (int j = 0; j < kAt; ++j) {
      const int k = min(k0 + j, pieces - 1);
      end[j] = slot[k * step];
      left[j] = sum[(long long)k * p.D];
    }
#pragma unroll
    for (int j = 0; j < kAt; ++j) {
      if (k0 + j < pieces) slot[(k0 + j) * step] = h;
      // A piece's factor may leave fp32's range, at either end, where the state
      // does not: its whole powers of two are applied by themselves, as many as
      // lead from any number past any other.  (Factors that are NaN or infinite
      // by an input reach end[j] as well.)
      const float x = fminf(fmaxf(A * left[j], -400.0f), 400.0f), whole = rintf(x);
      h = ldexpf(__builtin_amdgcn_exp2f(x - whole) * h, (int)whole) + end[j];
    }
  }
}

ScanFn kernel_of(int dtype, const ScanPlan& s, bool ends) {
  switch (dtype) {
    case MG3M_F32: return scan_kernel_f32(s.P, s.F, ends);
    case MG3M_BF16: return scan_kernel_bf16(s.P, s.F, ends);
    default: return scan_kernel_f16(s.P, s.F, ends);
  }
}

template <typename T>
struct alignas(4 * sizeof(T)) Four {
  T v[4];
};

// Single tokens: a lane holds four states of a channel, so a channel takes
// the next power of two of S / 4 lanes, which then sum its output.  Bound by
// the states' bytes; of one token, by how many loads follow one another, so all
// of them come first, those without a tensor of their own from another one.
// VEC: states and rates in 16 bytes; BC: B and C by fours, too (256 sequences, D
// = 5120: 46 us without either, 38).
template <typename T, bool VEC, bool BC>
__global__ __launch_bounds__(256) void scan_token(mg3m_scan p, int lanes_log2, int blocks) {
  const int n = blockIdx.x / blocks;                // the same for all lanes
  const int i = (int)(blockIdx.x - n * blocks) * 256 + threadIdx.x;
  const int lanes = 1 << lanes_log2, q = i & (lanes - 1);
  const bool live = i >> lanes_log2 < p.D;
  const int d = min(i >> lanes_log2, p.D - 1), s0 = 4 * q;
  const int g = p.G == 1 ? 0 : d / (p.D / p.G);
  const long long row = (long long)n * p.D + d;
  float* state = p.state + row * p.S + s0;
  const float* rate = p.A + (long long)d * p.S + s0;
  const T* B = static_cast<const T*>(p.B) + n * p.ldb + g * p.S + s0;
  const T* C = static_cast<const T*>(p.C) + n * p.ldc + g * p.S + s0;
  const T* us = static_cast<const T*>(p.u) + n * p.ldu;
  const T* zs = p.z != nullptr ? static_cast<const T*>(p.z) + n * p.ldz : us;
  const T uv = us[d], dv = static_cast<const T*>(p.dt)[n * p.lddt + d], zv = zs[d];
  const float bias = (p.dt_bias != nullptr ? p.dt_bias : p.A)[d], skip = (p.D_skip != nullptr ? p.D_skip : p.A)[d];
  float4 h{}, A{};
  Four<T> b{}, c{};
  if constexpr (VEC) {
    if (s0 < p.S) {
      h = *reinterpret_cast<const float4*>(state);
      A = *reinterpret_cast<const float4*>(rate);
      if constexpr (BC) {
        b = *reinterpret_cast<const Four<T>*>(B);
        c = *reinterpret_cast<const Four<T>*>(C);
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          b.v[k] = B[k];
          c.v[k] = C[k];
        }
      }
    }
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (s0 + k < p.S) {
        (&h.x)[k] = state[k];
        (&A.x)[k] = rate[k];
        b.v[k] = B[k];
        c.v[k] = C[k];
      }
  }
  const float u = (float)uv;
  float delta = (float)dv;
  if (p.dt_bias != nullptr) delta += bias;
  if (p.softplus) delta = softplus(delta);
  const float du = delta * u;
  float out = 0.0f;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float next = fmaf(__builtin_amdgcn_exp2f(delta * ((&A.x)[k] * kLog2e)), (&h.x)[k], du * (float)b.v[k]);
    (&h.x)[k] = next;
    if (s0 + k < p.S) out = fmaf((float)c.v[k], next, out);
  }
  for (int o = 1; o < lanes; o *= 2) out += __shfl_xor(out, o);
  if (!live) return;
  if constexpr (VEC) {
    if (s0 < p.S) *reinterpret_cast<float4*>(state) = h;
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (s0 + k < p.S) state[k] = (&h.x)[k];
  }
  if (q == 0) {
    if (p.D_skip != nullptr) out = fmaf(skip, u, out);
    const float z = (float)zv;
    if (p.z != nullptr) out *= z * sigmoid(z);
    static_cast<T*>(p.y)[n * p.ldy + d] = (T)out;
  }
}

int token_lanes_log2(int S) {
  int v = 0;
  while (4 << v < S) ++v;
  return v;
}
long long token_blocks(const mg3m_scan& p) { return (((long long)p.D << token_lanes_log2(p.S)) + 255) / 256; }

// Work-groups of scan_pieces.
long long scan_groups(const mg3m_scan& p, const ScanPlan& s) {
  return piece_count(p.begin, p.N, p.T, s.W) * p.G * ((p.D / p.G + 63) / 64);
}

bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

}  // namespace

bool scan_fits(const mg3m_scan& p, bool step) {
  if (step) return fits_launch(token_blocks(p) * p.N, 256);
  const ScanPlan s = scan_plan(p.T, p.D, p.G, p.S, p.N, p.begin == nullptr);
  return fits_launch(scan_groups(p, s), 64 * s.F);
}

size_t scan_workspace_bytes(int T, int D, int G, int S, int N) {
  // for equal parts and for given rows, whichever takes more
  size_t most = 0;
  for (bool equal : {true, false})
    most = std::max(most, scan_space(scan_plan(T, D, G, S, N, equal), T, D, G, S, N, equal).total());
  return most;
}

int launch_scan(const mg3m_scan& p, void* ws, void* stream, std::string* err) {
  hipStream_t st = static_cast<hipStream_t>(stream);
  const bool equal = p.begin == nullptr;
  const ScanPlan s = scan_plan(p.T, p.D, p.G, p.S, p.N, equal);
  const ScanSpace m = scan_space(s, p.T, p.D, p.G, p.S, p.N, equal);
  ScanArgs a{};
  a.p = p;
  char* at = static_cast<char*>(ws);
  float* bc = reinterpret_cast<float*>(at);
  a.bc = bc;
  a.slots = reinterpret_cast<float*>(at + m.bc);
  a.sums = reinterpret_cast<float*>(at + m.bc + m.slots);
  a.W = s.W;
  a.blocks = (p.D / p.G + 63) / 64;
  const long long groups = scan_groups(p, s);
  const long long pack = std::min(((long long)p.G * s.F * p.T * 2 * s.P + 255) / 256, 1LL << 20);
  const ScanFn ends = kernel_of(p.dtype, s, true), whole = kernel_of(p.dtype, s, false);
  if (ends == nullptr || whole == nullptr) {
    *err = "selective scan: no kernel for this plan";
    return MG3M_ERR_PLAN;
  }
  if (pack > 0) {
    with_dtype(p.dtype, [&](auto t) {
      scan_pack<decltype(t)><<<(unsigned)pack, 256, 0, st>>>(a, bc, s.P, s.F);
      return 0;
    });
  }
  if (s.W != 0) {
    ends<<<(unsigned)groups, 64 * s.F, 0, st>>>(a);
    // N is below 352 here (scan_plan), far below the 65535 of a grid's second dimension
    scan_join<<<dim3((p.D * p.S + 255) / 256, p.N), 256, 0, st>>>(a);
  }
  whole<<<(unsigned)groups, 64 * s.F, 0, st>>>(a);
  return launched("selective scan", err);
}

int launch_scan_step(const mg3m_scan& p, void* stream, std::string* err) {
  const int lanes_log2 = token_lanes_log2(p.S);
  const long long blocks = token_blocks(p), groups = blocks * p.N;
  const bool vec = p.S % 4 == 0 && aligned16(p.state) && aligned16(p.A);
  return with_dtype(p.dtype, [&](auto t) {
    using T = decltype(t);
    const auto fours = [](const void* x, long long ld) {
      return reinterpret_cast<uintptr_t>(x) % (4 * sizeof(T)) == 0 && ld % 4 == 0;
    };
    const bool bc = vec && fours(p.B, p.ldb) && fours(p.C, p.ldc);
    auto* kernel = bc ? scan_token<T, true, true> : vec ? scan_token<T, true, false> : scan_token<T, false, false>;
    kernel<<<(unsigned)groups, 256, 0, static_cast<hipStream_t>(stream)>>>(p, lanes_log2, (int)blocks);
    return launched("selective scan", err);
  });
}

}  // namespace mg3m
