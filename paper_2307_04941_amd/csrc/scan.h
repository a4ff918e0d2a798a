// The scan kernel by element type (scan_*.hip) and its launcher (scan.hip).
#pragma once

#include "seq_device.h"

namespace mg3m {

constexpr int kTile = 16;            // tokens between two barriers

struct ScanArgs {
  mg3m_scan p;
  const float* bc;       // B and C in fp32: [G][F][T][2][P], zeros behind S
  float* slots;          // cut sequences: [piece][S][D], the state a piece starts from (between the passes: ends with)
  float* sums;           // [piece][D], the sum of a piece's step sizes
  int W;                 // tokens of a piece, 0: sequences are not cut
  int blocks;            // 64-channel blocks of a group
};

using ScanFn = void (*)(ScanArgs);

ScanFn scan_kernel_f32(int P, int F, bool ends);
ScanFn scan_kernel_bf16(int P, int F, bool ends);
ScanFn scan_kernel_f16(int P, int F, bool ends);

}  // namespace mg3m
