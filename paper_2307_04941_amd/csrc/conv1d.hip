// Causal depthwise convolution along tokens (include/mg3m_seq.h).
//
// 2 R flops per element: bound by the bytes of x and y.  A thread takes V
// neighbouring channels (16 bytes, or one where rows are not 16-byte aligned)
// through a piece of a sequence, the last R inputs of each in registers, so
// that x is read once but for the R - 1 rows before a piece.
#include "seq_device.h"

namespace mg3m {
namespace {

constexpr int kStep = 4;             // tokens whose loads are issued together

struct ConvArgs {
  mg3m_conv1d p;
  int W;               // tokens of a piece, a multiple of kStep
  int vecs;            // groups of V channels
  unsigned items;      // pieces times vecs
};

template <typename T, int V>
struct alignas(V * sizeof(T)) Pack {
  T v[V];
};

template <typename T, int V, int R>
__global__ __launch_bounds__(256) void conv1d_pieces(ConvArgs a) {
  const mg3m_conv1d& p = a.p;
  const unsigned item = blockIdx.x * 256u + threadIdx.x;
  if (item >= a.items) return;
  const int id = item / a.vecs, c = (int)(item - id * (unsigned)a.vecs) * V;
  const Piece pc = find_piece(p.begin, p.end, p.N, p.T, a.W, id);
  if (pc.n < 0) return;

  using P = Pack<T, V>;
  const T* x = static_cast<const T*>(p.x) + c;
  T* y = static_cast<T*>(p.y) + c;
  T* state = R > 1 && p.state != nullptr ? static_cast<T*>(p.state) + (long long)pc.n * (R - 1) * p.C + c : nullptr;
  auto row = [&](int t) { return *reinterpret_cast<const P*>(x + (unsigned long long)(unsigned)t * (unsigned)p.ldx); };
  const int first = pc.b - pc.k * a.W;           // the sequence's first row

  float w[R][V], h[R][V], bias[V];               // h[i]: the input i + 1 - R rows before
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const P r = *reinterpret_cast<const P*>(static_cast<const T*>(p.w) + (long long)i * p.C + c);
#pragma unroll
    for (int k = 0; k < V; ++k) w[i][k] = (float)r.v[k];
  }
  {
    P r{};
    if (p.bias != nullptr) r = *reinterpret_cast<const P*>(static_cast<const T*>(p.bias) + c);
#pragma unroll
    for (int k = 0; k < V; ++k) bias[k] = (float)r.v[k];
  }
  // the R - 1 rows before this piece: x's, or at the sequence's start its state's
  const bool kept = state != nullptr && p.load_state;
  {
    // loads without conditions, from rows that are there: all under way at once
    P r[R];
#pragma unroll
    for (int i = 1; i < R; ++i) {
      const int t = pc.b - R + i;
      const T* at = t >= first ? x + (unsigned long long)(unsigned)t * (unsigned)p.ldx
                               : kept ? state + (long long)(t - first + R - 1) * p.C : static_cast<const T*>(p.w) + c;
      r[i] = *reinterpret_cast<const P*>(at);
    }
#pragma unroll
    for (int i = 1; i < R; ++i)
#pragma unroll
      for (int k = 0; k < V; ++k) h[i][k] = pc.b - R + i >= first || kept ? (float)r[i].v[k] : 0.0f;
  }
  // The thread of the first piece has read the sequence's state, so it writes
  // the one after: rows end - R + 1 .. of state and x together.
  if (state != nullptr && pc.k == 0) {
    const SeqRange s = seq_range(p.begin, p.end, pc.n, p.N, p.T);
#pragma unroll
    for (int i = 1; i < R; ++i) {
      const int t = s.e - R + i;
      P r{};
      if (t >= first) {
        r = row(t);
      } else {
        const int from = t - first + R;          // h's row: at least i, as the sequence has no rows below 0
#pragma unroll
        for (int j = 1; j < R; ++j)
          if (j == from)
#pragma unroll
            for (int k = 0; k < V; ++k) r.v[k] = (T)h[j][k];
      }
      *reinterpret_cast<P*>(state + (long long)(i - 1) * p.C) = r;
    }
  }

  auto output = [&](int t, const P& in) {
#pragma unroll
    for (int i = 0; i + 1 < R; ++i)
#pragma unroll
      for (int k = 0; k < V; ++k) h[i][k] = h[i + 1][k];
    P out;
#pragma unroll
    for (int k = 0; k < V; ++k) {
      h[R - 1][k] = (float)in.v[k];
      float s = bias[k];
#pragma unroll
      for (int i = 0; i < R; ++i) s = fmaf(w[i][k], h[i][k], s);
      const float act = s * sigmoid(s);
      out.v[k] = (T)(p.silu ? act : s);
    }
    *reinterpret_cast<P*>(y + (unsigned long long)(unsigned)t * (unsigned)p.ldy) = out;
  };
  // h moves up with each token: its first row is the oldest
#pragma unroll
  for (int k = 0; k < V; ++k) h[0][k] = 0.0f;
  int t = pc.b;
  for (; t + kStep <= pc.e; t += kStep) {
    P in[kStep];
#pragma unroll
    for (int j = 0; j < kStep; ++j) in[j] = row(t + j);
#pragma unroll
    for (int j = 0; j < kStep; ++j) output(t + j, in[j]);
  }
  for (; t < pc.e; ++t) output(t, row(t));
}

// Single tokens: everything is loaded at once, for what counts is how many
// loads follow one another.
template <typename T, int V, int R>
__global__ __launch_bounds__(256) void conv1d_token(ConvArgs a) {
  const mg3m_conv1d& p = a.p;
  const unsigned item = blockIdx.x * 256u + threadIdx.x;
  if (item >= a.items) return;
  const int n = item / a.vecs, c = (int)(item - n * (unsigned)a.vecs) * V;
  using P = Pack<T, V>;
  T* state = static_cast<T*>(p.state) + (long long)n * (R - 1) * p.C + c;
  P h[R], w[R], bias{};
#pragma unroll
  for (int i = 0; i + 1 < R; ++i) h[i] = *reinterpret_cast<const P*>(state + (long long)i * p.C);
  h[R - 1] = *reinterpret_cast<const P*>(static_cast<const T*>(p.x) + n * p.ldx + c);
#pragma unroll
  for (int i = 0; i < R; ++i) w[i] = *reinterpret_cast<const P*>(static_cast<const T*>(p.w) + (long long)i * p.C + c);
  if (p.bias != nullptr) bias = *reinterpret_cast<const P*>(static_cast<const T*>(p.bias) + c);
  P out;
#pragma unroll
  for (int k = 0; k < V; ++k) {
    float s = (float)bias.v[k];
#pragma unroll
    for (int i = 0; i < R; ++i) s = fmaf((float)w[i].v[k], (float)h[i].v[k], s);
    const float act = s * sigmoid(s);
    out.v[k] = (T)(p.silu ? act : s);
  }
#pragma unroll
  for (int i = 0; i + 1 < R; ++i) *reinterpret_cast<P*>(state + (long long)i * p.C) = h[i + 1];
  *reinterpret_cast<P*>(static_cast<T*>(p.y) + n * p.ldy + c) = out;
}

template <typename T, int V, int R>
void launch_as(const ConvArgs& a, bool token, void* stream) {
  auto* kernel = token ? conv1d_token<T, V, R> : conv1d_pieces<T, V, R>;
  kernel<<<(a.items + 255) / 256, 256, 0, static_cast<hipStream_t>(stream)>>>(a);
}

template <typename T, int V>
void launch_taps(const ConvArgs& a, bool token, void* stream) {
  switch (a.p.R) {
    case 1: launch_as<T, V, 1>(a, token, stream); break;
    case 2: launch_as<T, V, 2>(a, token, stream); break;
    case 3: launch_as<T, V, 3>(a, token, stream); break;
    case 4: launch_as<T, V, 4>(a, token, stream); break;
    case 5: launch_as<T, V, 5>(a, token, stream); break;
    case 6: launch_as<T, V, 6>(a, token, stream); break;
    case 7: launch_as<T, V, 7>(a, token, stream); break;
    default: launch_as<T, V, 8>(a, token, stream); break;
  }
}

bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

int launch(const mg3m_conv1d& p, bool token, void* stream, std::string* err) {
  return with_dtype(p.dtype, [&](auto t) {
    using T = decltype(t);
    constexpr int V = 16 / sizeof(T);
    const bool vec = p.C % V == 0 && p.ldx % V == 0 && p.ldy % V == 0 && aligned16(p.x) && aligned16(p.y) &&
                     aligned16(p.w) && aligned16(p.bias) && aligned16(p.state);
    ConvArgs a{};
    a.p = p;
    a.vecs = vec ? p.C / V : p.C;
    // Pieces as long as they may be with threads enough to fill the chip: each
    // piece reads R - 1 rows again.  Not under R - 1 tokens: only a sequence's
    // first piece may read its state, which the same thread overwrites.
    const int least = p.R - 1 <= kStep ? kStep : 2 * kStep;
    static_assert(2 * kStep >= 7, "R is at most 8");
    long long pieces = p.N, items = pieces * a.vecs;
    const auto cut = [&] {
      pieces = piece_count(p.begin, p.N, p.T, a.W);
      items = pieces * a.vecs;
    };
    const auto fits = [&] { return pieces <= 0x7fffffffLL && fits_launch((items + 255) / 256, 256); };
    if (!token) {
      for (a.W = 32;; a.W /= 2) {
        cut();
        if (a.W == least || items >= 256 * 2048) break;
      }
      while (!fits() && a.W < (1 << 20)) {
        a.W *= 2;
        cut();
      }
    }
    if (!fits()) {
      *err = "causal convolution: too many sequences and channels for one launch";
      return (int)MG3M_ERR_TOO_LARGE;
    }
    a.items = (unsigned)items;
    if (vec) launch_taps<T, V>(a, token, stream);
    else launch_taps<T, 1>(a, token, stream);
    return launched("causal convolution", err);
  });
}

}  // namespace

int launch_conv1d(const mg3m_conv1d& p, void* stream, std::string* err) { return launch(p, false, stream, err); }

int launch_conv1d_step(const mg3m_conv1d& p, void* stream, std::string* err) { return launch(p, true, stream, err); }

}  // namespace mg3m
