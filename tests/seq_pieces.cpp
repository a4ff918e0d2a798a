// The cut of sequences into pieces (paper_2307_04941_amd/csrc/seq_pieces.h) on
// the host: for valid ranges every row is in exactly one piece of its
// sequence; for any values at all, every piece and every number derived from
// one stays inside the tensors and the workspace.
#include <algorithm>
#include <climits>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#define __device__
#define __forceinline__ inline
using std::max;
using std::min;
#include "seq_pieces.h"

using namespace mg3m;

static void require(bool ok, const char* what) {
  if (!ok) {
    std::printf("failed: %s\n", what);
    std::exit(1);
  }
}

// Every piece of a call; rows counted if `seen` is given.
static void walk(const int* b, const int* e, int N, int T, int W, std::vector<int>* seen) {
  const long long ids = piece_count(b, N, T, W);
  std::vector<int> first(N, 0), lasts(N, 0);
  for (long long id = 0; id < ids; ++id) {
    const Piece p = find_piece(b, e, N, T, W, (int)id);
    if (p.n < 0) continue;
    require(p.n < N && p.k >= 0, "sequence and piece");
    require(0 <= p.b && p.b <= p.e && p.e <= T, "rows inside the tensor");
    require(W == 0 || p.e - p.b <= W, "a piece's length");
    require(p.b - (long long)p.k * W >= 0, "the sequence's first row");
    if (seen == nullptr) continue;
    const SeqRange r = seq_range(b, e, p.n, N, T);
    require(p.b >= r.b && p.e <= r.e && p.b == r.b + (long long)p.k * W, "rows inside the sequence");
    require(p.last == (p.e == r.e), "the last piece");
    first[p.n] += p.k == 0;
    lasts[p.n] += p.last;
    for (int t = p.b; t < p.e; ++t) ++(*seen)[t];
  }
  if (W != 0 && b != nullptr)
    for (int n = 0; n < N; ++n) {
      // the numbers that the joining kernel derives itself
      const SeqRange r = seq_range(b, e, n, N, T);
      const long long id0 = piece_base(b, n, T, W);
      require(id0 >= 0 && id0 + std::max(1, ceil_div(r.e - r.b, W)) <= ids, "joined pieces");
    }
  if (seen != nullptr)
    for (int n = 0; n < N; ++n) require(first[n] == 1 && lasts[n] == 1, "one first and one last piece");
}

int main() {
  std::mt19937 rng(7);
  auto to = [&](int a, int b) { return (int)(a + rng() % (unsigned)(b - a + 1)); };
  for (int trial = 0; trial < 4000; ++trial) {
    const int N = to(1, 12), W = to(0, 4) == 0 ? 0 : 1 << to(0, 6);
    std::vector<int> b(N), e(N);
    int at = to(0, 3);
    for (int n = 0; n < N; ++n) {
      b[n] = at + (to(0, 2) == 0 ? to(0, 9) : 0);
      e[n] = b[n] + (to(0, 3) == 0 ? 0 : to(0, 90));
      at = e[n];
    }
    const int T = at + to(0, 5);
    std::vector<int> seen(T, 0);
    walk(b.data(), e.data(), N, T, W, &seen);
    for (int t = 0; t < T; ++t) {
      int in = 0;
      for (int n = 0; n < N; ++n) in += b[n] <= t && t < e[n];
      require(seen[t] == in, "every row once");
    }
    const int L = to(0, 70);
    std::vector<int> all(N * L, 0);
    walk(nullptr, nullptr, N, N * L, W, &all);
    for (int v : all) require(v == 1, "every row of equal parts once");
    // anything
    for (int n = 0; n < N; ++n) {
      b[n] = to(0, 3) == 0 ? (int)rng() : to(-20, T + 20);
      e[n] = to(0, 3) == 0 ? (int)rng() : to(-20, T + 20);
    }
    walk(b.data(), e.data(), N, T, W, nullptr);
  }
  // the largest sizes, where a sum could pass the ints
  const int T = 0x7fff0000;
  for (int W : {0, 4, 256, 1 << 20}) {
    const int b[2] = {0, INT_MAX}, e[2] = {INT_MAX, INT_MAX};
    const long long ids = piece_count(b, 2, T, W);
    for (long long id : {0LL, 1LL, ids / 2, ids - 2, ids - 1}) {
      if (id < 0 || id > INT_MAX) continue;
      const Piece p = find_piece(b, e, 2, T, W, (int)id);
      require(p.n < 0 || (0 <= p.b && p.b <= p.e && p.e <= T), "large rows inside the tensor");
    }
    require(piece_count(nullptr, 1, T, W) <= INT_MAX || W == 0, "pieces of the longest sequence");
  }
  std::printf("pieces ok\n");
  return 0;
}
