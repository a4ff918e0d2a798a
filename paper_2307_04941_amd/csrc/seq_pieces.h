// Sequences as row ranges, and their cut into pieces (include/mg3m_seq.h).
// Plain integer arithmetic: tests/seq_pieces.cpp checks it on the host.
#pragma once

#include <algorithm>

namespace mg3m {

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

// a / b rounded up, for any a >= 0
__device__ __forceinline__ int ceil_div(int a, int b) { return a / b + (a % b != 0); }

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
  if (begin == nullptr) return (long long)N * std::max(1, T / N / W + (T / N % W != 0));
  return (long long)T / W + N;
}
__device__ __forceinline__ int piece_base(const int* begin, int n, int T, int W) {
  return (int)((unsigned)min(max(begin[n], 0), T) / (unsigned)W) + n;
}
__device__ __forceinline__ Piece find_piece(const int* begin, const int* end, int N, int T, int W, int id) {
  Piece p{id, 0, 0, 0, true};
  if (W != 0) {
    if (begin == nullptr) {
      const int per = max(1, ceil_div(T / N, W));
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

}  // namespace mg3m
