// C entry points of the sequence operators (include/mg3m_seq.h): validation
// and dispatch.  Validation finishes before anything is launched.
#include <cstdint>
#include <cstdlib>
#include <exception>
#include <initializer_list>
#include <string>

#include "seq.h"

namespace mg3m {
namespace {

// A row tensor: rows x cols elements of `size` bytes, ld elements apart.
struct Rows {
  const char* name;
  const void* p;
  long long rows, cols, ld;
  int size;
  bool out;

  uintptr_t first() const { return reinterpret_cast<uintptr_t>(p); }
  unsigned long long bytes() const {
    return rows == 0 ? 0 : ((unsigned long long)(rows - 1) * ld + cols) * size;
  }
};

// Sizes are ints and distances at most 2^30 elements, so extents fit 64 bits.
constexpr long long kMaxDistance = 1LL << 30;
// Rows, and what else the kernels count in ints, stay clear of their end.
constexpr int kMaxRows = 0x7fff0000, kMaxSize = 1 << 30;

Rows dense(const char* name, const void* p, long long n, int size, bool out = false) {
  return {name, p, 1, n, n, size, out};
}

// Whether two row tensors share an element.  Rows of one distance may lie
// between one another (columns of one wider tensor).
bool share(const Rows& a, const Rows& b) {
  if (a.bytes() == 0 || b.bytes() == 0) return false;
  if (a.first() + a.bytes() <= b.first() || b.first() + b.bytes() <= a.first()) return false;
  const unsigned long long step = (unsigned long long)a.ld * a.size;
  if (a.rows > 1 && b.rows > 1 && step == (unsigned long long)b.ld * b.size) {
    const Rows& lo = a.first() <= b.first() ? a : b;
    const Rows& hi = a.first() <= b.first() ? b : a;
    const unsigned long long off = (hi.first() - lo.first()) % step;
    return off < (unsigned long long)lo.cols * lo.size || off + (unsigned long long)hi.cols * hi.size > step;
  }
  return true;
}

int check_rows(std::initializer_list<Rows> ts) {
  for (const Rows& t : ts) {
    if (t.p == nullptr) continue;
    if (t.first() % t.size != 0)
      return set_error(MG3M_ERR_ALIGN, std::string(t.name) + " is not aligned to its " + std::to_string(t.size) +
                                           "-byte elements");
    if (t.ld < t.cols || (t.rows > 1 && t.ld > kMaxDistance))
      return set_error(MG3M_ERR_SHAPE, "the distance between rows of " + std::string(t.name) + " is " +
                                           std::to_string(t.ld) + ": " + std::to_string(t.cols) + " to 2^30 allowed");
  }
  for (const Rows& o : ts)
    for (const Rows& t : ts)
      if (o.out && o.p != nullptr && t.p != nullptr && &o != &t && share(o, t))
        return set_error(MG3M_ERR_ALIAS, std::string(o.name) + " overlaps " + t.name);
  return MG3M_OK;
}

bool flag(int v) { return v == 0 || v == 1; }

int check_type(int dtype) {
  return dtype == MG3M_F32 || dtype == MG3M_BF16 || dtype == MG3M_F16
             ? MG3M_OK
             : set_error(MG3M_ERR_ARG, "unknown dtype " + std::to_string(dtype));
}

// T rows in N sequences: begin and end, or equal parts.
int check_sequences(const int* begin, const int* end, int T, int N) {
  if (T < 0 || N < 1) return set_error(MG3M_ERR_SHAPE, "T must be >= 0 and N >= 1");
  if ((begin == nullptr) != (end == nullptr)) return set_error(MG3M_ERR_ARG, "give begin and end, or neither");
  if (T > kMaxRows) return set_error(MG3M_ERR_TOO_LARGE, "more than 2^31 - 2^16 rows");
  if (begin == nullptr && T % N != 0)
    return set_error(MG3M_ERR_SHAPE, "T must be a multiple of N when begin and end are NULL");
  if (reinterpret_cast<uintptr_t>(begin) % 4 != 0 || reinterpret_cast<uintptr_t>(end) % 4 != 0)
    return set_error(MG3M_ERR_ALIGN, "begin and end must be 4-byte aligned");
  return MG3M_OK;
}

// The test hook of conv_launch.hip, for these launches.
bool launch_failure_injected() {
  const char* v = std::getenv("MG3M_TEST_FAIL_LAUNCH");
  return v != nullptr && v[0] == '1' && v[1] == 0;
}
int injected() { return set_error(MG3M_ERR_HIP, "kernel launch: failure injected by MG3M_TEST_FAIL_LAUNCH"); }

int element_size(int dtype) { return dtype == MG3M_F32 ? 4 : 2; }

int conv1d(const mg3m_conv1d* in, bool step, void* stream) {
  clear_error();
  if (in == nullptr) return set_error(MG3M_ERR_NULL, "the arguments must be non-NULL");
  mg3m_conv1d a = *in;
  if (int rc = check_type(a.dtype)) return rc;
  if (!flag(a.load_state) || !flag(a.silu) || a.reserved != 0)
    return set_error(MG3M_ERR_ARG, "load_state and silu must be 0 or 1, reserved 0");
  if (step) {
    if (a.begin != nullptr || a.end != nullptr)
      return set_error(MG3M_ERR_ARG, "begin and end must be NULL for single tokens");
    a.T = a.N;
    a.load_state = 1;
  }
  if (int rc = check_sequences(a.begin, a.end, a.T, a.N)) return rc;
  if (a.C < 1 || a.R < 1 || a.R > 8) return set_error(MG3M_ERR_SHAPE, "C must be >= 1 and R 1..8");
  if (a.C > kMaxSize) return set_error(MG3M_ERR_TOO_LARGE, "more than 2^30 channels");
  if (a.w == nullptr || (a.T > 0 && (a.x == nullptr || a.y == nullptr)))
    return set_error(MG3M_ERR_NULL, "x, w and y must be non-NULL");
  if (a.R == 1) a.state = nullptr;
  if (step && a.R > 1 && a.state == nullptr)
    return set_error(MG3M_ERR_NULL, "state must be non-NULL for single tokens");
  if (a.load_state && !step && a.R > 1 && a.state == nullptr)
    return set_error(MG3M_ERR_NULL, "load_state without a state");
  const int e = element_size(a.dtype);
  if (int rc = check_rows({{"y", a.y, a.T, a.C, a.ldy, e, true},
                           dense("state", a.state, (long long)a.N * (a.R - 1) * a.C, e, true),
                           {"x", a.x, a.T, a.C, a.ldx, e, false},
                           dense("w", a.w, (long long)a.R * a.C, e),
                           dense("bias", a.bias, a.C, e),
                           dense("begin", a.begin, a.N, 4),
                           dense("end", a.end, a.N, 4)}))
    return rc;
  if (launch_failure_injected()) return injected();
  std::string err;
  const int rc = step ? launch_conv1d_step(a, stream, &err) : launch_conv1d(a, stream, &err);
  return rc ? set_error(rc, err) : MG3M_OK;
}

int check_scan_sizes(int T, int D, int G, int S, int N) {
  if (T < 0 || N < 1) return set_error(MG3M_ERR_SHAPE, "T must be >= 0 and N >= 1");
  if (D < 1 || G < 1 || D % G != 0 || S < 1 || S > 256)
    return set_error(MG3M_ERR_SHAPE, "D must be >= 1, G divide it, and S be 1..256");
  if ((long long)D * S > kMaxSize) return set_error(MG3M_ERR_TOO_LARGE, "D * S above 2^30");
  return MG3M_OK;
}

int scan(const mg3m_scan* in, bool step, void* stream) {
  clear_error();
  if (in == nullptr) return set_error(MG3M_ERR_NULL, "the arguments must be non-NULL");
  mg3m_scan a = *in;
  if (int rc = check_type(a.dtype)) return rc;
  if (!flag(a.load_state) || !flag(a.softplus))
    return set_error(MG3M_ERR_ARG, "load_state and softplus must be 0 or 1");
  if (step) {
    if (a.begin != nullptr || a.end != nullptr)
      return set_error(MG3M_ERR_ARG, "begin and end must be NULL for single tokens");
    a.T = a.N;
    a.load_state = 1;
  }
  if (int rc = check_scan_sizes(a.T, a.D, a.G, a.S, a.N)) return rc;
  if (int rc = check_sequences(a.begin, a.end, a.T, a.N)) return rc;
  if (a.A == nullptr || (a.T > 0 && (a.u == nullptr || a.dt == nullptr || a.B == nullptr || a.C == nullptr ||
                                     a.y == nullptr)))
    return set_error(MG3M_ERR_NULL, "u, dt, A, B, C and y must be non-NULL");
  if ((step || a.load_state) && a.state == nullptr)
    return set_error(MG3M_ERR_NULL, "state must be non-NULL to be loaded");
  const int e = element_size(a.dtype), bc = a.G * a.S;
  const size_t need = step ? 0 : scan_workspace_bytes(a.T, a.D, a.G, a.S, a.N);
  const bool own = a.workspace == nullptr;
  if (need > 0 && !own) {
    if (a.workspace_bytes < need)
      return set_error(MG3M_ERR_WORKSPACE, "the scan needs " + std::to_string(need) + " workspace bytes");
    if (reinterpret_cast<uintptr_t>(a.workspace) % 16 != 0)
      return set_error(MG3M_ERR_WORKSPACE, "workspace must be 16-byte aligned");
  }
  if (int rc = check_rows({{"y", a.y, a.T, a.D, a.ldy, e, true},
                           dense("state", a.state, (long long)a.N * a.D * a.S, 4, true),
                           dense("workspace", need > 0 && !own ? a.workspace : nullptr, (long long)need, 1, true),
                           {"u", a.u, a.T, a.D, a.ldu, e, false},
                           {"dt", a.dt, a.T, a.D, a.lddt, e, false},
                           {"B", a.B, a.T, bc, a.ldb, e, false},
                           {"C", a.C, a.T, bc, a.ldc, e, false},
                           {"z", a.z, a.T, a.D, a.ldz, e, false},
                           dense("A", a.A, (long long)a.D * a.S, 4),
                           dense("D", a.D_skip, a.D, 4),
                           dense("dt_bias", a.dt_bias, a.D, 4),
                           dense("begin", a.begin, a.N, 4),
                           dense("end", a.end, a.N, 4)}))
    return rc;
  if (!scan_fits(a, step))
    return set_error(MG3M_ERR_TOO_LARGE, "selective scan: too many rows, sequences or channels for one launch");
  if (launch_failure_injected()) return injected();
  std::string err;
  int rc = MG3M_OK;
  if (step) {
    rc = launch_scan_step(a, stream, &err);
  } else if (need == 0 || !own) {
    rc = launch_scan(a, a.workspace, stream, &err);
  } else {
    CallWorkspace w;
    rc = take_workspace(stream, need, &w, &err);
    if (rc == MG3M_OK) rc = give_workspace(stream, &w, launch_scan(a, w.ptr, stream, &err), &err);
  }
  return rc ? set_error(rc, err) : MG3M_OK;
}

int w4(const mg3m_w4* in, void* stream) {
  clear_error();
  if (in == nullptr) return set_error(MG3M_ERR_NULL, "the arguments must be non-NULL");
  const mg3m_w4& a = *in;
  if (int rc = check_type(a.dtype)) return rc;
  if (a.reserved != 0) return set_error(MG3M_ERR_ARG, "reserved must be 0");
  if (a.M < 1 || a.C < 1 || a.K < 1) return set_error(MG3M_ERR_SHAPE, "M, C and K must be >= 1");
  if (a.group < 32 || a.group % 32 != 0 || a.C % a.group != 0)
    return set_error(MG3M_ERR_SHAPE, "group must be a multiple of 32 that divides C");
  if (a.M > kMaxSize || a.K > kMaxSize || a.C > kMaxW4Channels)
    return set_error(MG3M_ERR_TOO_LARGE, "M and K are at most 2^30, C at most 2^20");
  if (a.x == nullptr || a.q == nullptr || a.scale == nullptr || a.y == nullptr)
    return set_error(MG3M_ERR_NULL, "x, q, scale and y must be non-NULL");
  if (reinterpret_cast<uintptr_t>(a.q) % 16 != 0) return set_error(MG3M_ERR_ALIGN, "q must be 16-byte aligned");
  const int e = element_size(a.dtype);
  const long long groups = a.C / a.group;
  if (int rc = check_rows({{"y", a.y, a.M, a.K, a.ldy, e, true},
                           {"x", a.x, a.M, a.C, a.ldx, e, false},
                           dense("q", a.q, (long long)a.K * (a.C / 2), 1),
                           dense("scale", a.scale, a.K * groups, e),
                           dense("zero", a.zero, a.K * groups, 1)}))
    return rc;
  if (launch_failure_injected()) return injected();
  std::string err;
  const int rc = launch_w4(a, stream, &err);
  return rc ? set_error(rc, err) : MG3M_OK;
}

template <typename F>
int guarded(F&& f) {
  try {
    return f();
  } catch (const std::exception& e) {
    return set_error(MG3M_ERR_HIP, e.what());
  } catch (...) {
    return set_error(MG3M_ERR_HIP, "unknown exception");
  }
}

}  // namespace
}  // namespace mg3m

extern "C" {

int conv1d_causal_fwd(const mg3m_conv1d* a, void* stream) {
  return mg3m::guarded([&] { return mg3m::conv1d(a, false, stream); });
}

int conv1d_causal_step(const mg3m_conv1d* a, void* stream) {
  return mg3m::guarded([&] { return mg3m::conv1d(a, true, stream); });
}

int selective_scan_fwd(const mg3m_scan* a, void* stream) {
  return mg3m::guarded([&] { return mg3m::scan(a, false, stream); });
}

int selective_scan_workspace_bytes(int T, int D, int G, int S, int N, size_t* bytes) {
  return mg3m::guarded([&]() -> int {
    mg3m::clear_error();
    if (bytes == nullptr) return mg3m::set_error(MG3M_ERR_NULL, "bytes must be non-NULL");
    if (int rc = mg3m::check_scan_sizes(T, D, G, S, N)) return rc;
    *bytes = mg3m::scan_workspace_bytes(T, D, G, S, N);
    return MG3M_OK;
  });
}

int selective_scan_step(const mg3m_scan* a, void* stream) {
  return mg3m::guarded([&] { return mg3m::scan(a, true, stream); });
}

int matvec_w4_fwd(const mg3m_w4* a, void* stream) {
  return mg3m::guarded([&] { return mg3m::w4(a, stream); });
}

}  // extern "C"
