// Sequence operators (include/mg3m_seq.h): what the entry points (seq.cpp) and
// the kernels share.  Host part without HIP headers.
#pragma once

#include <mutex>
#include <string>

#include "mg3m_internal.h"
#include "mg3m_seq.h"

namespace mg3m {

// The workspace that the library keeps for a stream (abi.cpp), for one call:
// the holder of `lock` queues its launches and then gives it back.
struct CallWorkspace {
  void* ptr = nullptr;
  void* done = nullptr;                     // event recorded when given back, or null: a pool block
  std::unique_lock<std::mutex> lock;
};
int take_workspace(void* stream, size_t bytes, CallWorkspace* w, std::string* err);
// rc: the status of the launches; returns it, or the error of giving back.
int give_workspace(void* stream, CallWorkspace* w, int rc, std::string* err);

// Channels of a 4-bit product: its kernels divide by multiplication (matvec_w4.hip).
constexpr int kMaxW4Channels = 1 << 20;

// Launchers.  Arguments are checked; each returns an mg3m_status.
int launch_conv1d(const mg3m_conv1d& a, void* stream, std::string* err);        // conv1d.hip
int launch_conv1d_step(const mg3m_conv1d& a, void* stream, std::string* err);
size_t scan_workspace_bytes(int T, int D, int G, int S, int N);                 // scan.hip
bool scan_fits(const mg3m_scan& a, bool step);       // whether the launches take this many rows, sequences and channels
int launch_scan(const mg3m_scan& a, void* ws, void* stream, std::string* err);
int launch_scan_step(const mg3m_scan& a, void* stream, std::string* err);
int launch_w4(const mg3m_w4& a, void* stream, std::string* err);                // matvec_w4.hip

}  // namespace mg3m
