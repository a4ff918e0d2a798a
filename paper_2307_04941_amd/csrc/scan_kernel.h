// Selective state space scan, the kernel over prompts.
//
// One work-group runs one piece of a sequence through 64 channels of a group,
// a lane per channel.  The S states of a channel are dealt out to the F waves,
// P to a wave: each wave keeps its P states and rates in registers and walks
// all tokens.  B and C are the same for all channels of a group, so a wave
// takes them from scalar registers: a first kernel (scan.hip) writes them in
// fp32, [G][F][T][2][P], which makes a wave's values of consecutive tokens
// consecutive.
//
// What is per channel and token, not per state, is done once and shared
// through LDS: token j of a tile of 16 belongs to wave j mod F, which makes
// delta and delta * u of the next tile while all waves walk this one, and
// sums the F partial outputs, adds D u, gates and stores those of the last
// one.  Both arrays have two buffers, so a tile takes one barrier.
//
// A state and token cost four full-rate instructions and one exp2 at half
// rate: 24 cycles of a SIMD for 64 channels (measured: fma 4.2, exp2 8.8 at
// four waves).
#pragma once

#include <type_traits>

#include "scan.h"

namespace mg3m {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef const __attribute__((address_space(4))) f32x16 const16;

__device__ __forceinline__ void wave_barrier_lds() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// ENDS: the first pass over cut sequences, which computes no outputs but the
// state that each piece but a sequence's last ends with, started from zero,
// and its sum of step sizes.
template <typename T, int P, int F, bool ENDS>
__global__ __launch_bounds__(64 * F) void scan_pieces(ScanArgs a) {
  constexpr int kOwn = kTile / F;              // tokens of a tile that are this wave's to prepare and finish
  constexpr int kBatch = 16 / P;               // tokens per 32 values of B and C
  __shared__ float2 dd[2][kTile][64];                                    // delta, delta * u
  __shared__ float part[ENDS ? 1 : 2][F][ENDS ? 1 : kTile][64];          // outputs of P states

  const mg3m_scan& p = a.p;
  const int lane = threadIdx.x & 63;
  const int f = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int cblocks = a.blocks * p.G;
  const int id = blockIdx.x / cblocks, cb = blockIdx.x - id * cblocks;
  const int g = cb / a.blocks, per = p.D / p.G;
  // channels d0 + l: d0 is the same for all lanes, so that addresses are a
  // scalar and the lane's offset; lanes behind the group repeat its last channel
  const int in_group = (cb - g * a.blocks) * 64, d0 = g * per + in_group;
  const bool live = in_group + lane < per;
  const unsigned l = min(lane, per - 1 - in_group), lb = l * sizeof(T);
  const int d = d0 + l;

  Piece pc = find_piece(p.begin, p.end, p.N, p.T, a.W, id);
  const int n = __builtin_amdgcn_readfirstlane(pc.n);
  const bool last = __builtin_amdgcn_readfirstlane((int)pc.last);
  if (n < 0 || (ENDS && last)) return;
  const int b = __builtin_amdgcn_readfirstlane(pc.b), e = __builtin_amdgcn_readfirstlane(pc.e);
  const int tokens = e - b, tiles = ceil_div(tokens, kTile);

  // States f * P .. + P of channel d.  Loads without conditions, from elements
  // that are there, so that they are all under way at once: each under its own
  // condition, the compiler waits for them one by one.
  float A[P], h[P];
  const float* start = a.W != 0 ? a.slots : p.load_state ? p.state : p.A;
  const long long start_at = a.W != 0 ? (long long)id * p.S * p.D + d : p.load_state ? ((long long)n * p.D + d) * p.S : 0;
  const long long start_step = a.W != 0 ? p.D : p.load_state ? 1 : 0;
  const bool started = !ENDS && (a.W != 0 || p.load_state);
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const int s = min(f * P + i, p.S - 1);
    A[i] = p.A[(long long)d * p.S + s];
    h[i] = ENDS ? 0.0f : start[start_at + s * start_step];
  }
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const bool in = f * P + i < p.S;
    A[i] = in ? A[i] * kLog2e : 0.0f;
    h[i] = in && started ? h[i] : 0.0f;
  }
  const float bias = p.dt_bias != nullptr ? p.dt_bias[d] : 0.0f;
  const float skip = !ENDS && p.D_skip != nullptr ? p.D_skip[d] : 0.0f;

  const T* u = static_cast<const T*>(p.u) + (long long)b * p.ldu + d0;
  const T* dt = static_cast<const T*>(p.dt) + (long long)b * p.lddt + d0;
  // without a gate u stands in for z and is not used: no branch per token
  const bool gate = p.z != nullptr;
  const T* z = gate ? static_cast<const T*>(p.z) + (long long)b * p.ldz + d0 : u;
  const unsigned ldu = p.ldu, lddt = p.lddt, ldz = gate ? p.ldz : p.ldu, ldy = p.ldy;
  T* y = static_cast<T*>(p.y) + (long long)b * p.ldy + d0;
  const float* bc = a.bc + (((long long)g * F + f) * p.T + b) * (2 * P);

  // rows and distances are below 2^31: one 32 x 32 bit product per address
  auto row_at = [](int row, unsigned ld) { return (unsigned long long)(unsigned)row * ld; };
  using Raw = std::conditional_t<sizeof(T) == 4, unsigned, unsigned short>;
  // this wave's tokens of a tile; those behind the end read the last token
  auto load = [&](const T* x, unsigned ld, int tile, unsigned (&v)[kOwn]) {
#pragma unroll
    for (int k = 0; k < kOwn; ++k) {
      const T* row = x + row_at(min(tile * kTile + f + k * F, tokens - 1), ld);
      v[k] = *reinterpret_cast<const Raw*>(reinterpret_cast<const char*>(row) + lb);
    }
  };
  auto step_size = [&](unsigned raw) {
    const float v = raw_value<T>(raw) + bias;
    const float s = softplus(v);
    return p.softplus ? s : v;
  };
  auto finished = [&](float out, unsigned uv, unsigned zv) {
    out = fmaf(skip, raw_value<T>(uv), out);
    const float zf = raw_value<T>(zv);
    const float gated = out * (zf * sigmoid(zf));
    return gate ? gated : out;
  };
  auto store = [&](int tile, const float (&out)[kOwn]) {
#pragma unroll
    for (int k = 0; k < kOwn; ++k) {
      const int t = tile * kTile + f + k * F;
      if (live && t < tokens) *reinterpret_cast<T*>(reinterpret_cast<char*>(y + row_at(t, ldy)) + lb) = (T)out[k];
    }
  };

  float sum = 0.0f;                            // ENDS: of the step sizes
  // One token of this wave's states; a: exp2(delta A); B and C: v(0..P), v(P..2P).
  auto walk = [&](const float (&decay)[P], float du, auto&& v) {
    float out = 0.0f;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      h[i] = fmaf(decay[i], h[i], du * v(i));
      if (!ENDS) out = i == 0 ? v(P) * h[0] : fmaf(v(P + i), h[i], out);
    }
    return out;
  };
  auto decays = [&](float delta, float (&decay)[P]) {
#pragma unroll
    for (int i = 0; i < P; ++i) decay[i] = __builtin_amdgcn_exp2f(delta * A[i]);
  };
  // A whole tile, or its first `some` tokens; get(j): delta and delta * u of
  // token j, put(j, partial output).
  f32x16 v0, v1;                               // B and C of the next tokens
  auto whole_tile = [&](int tile, auto&& get, auto&& put) {
    const const16* at = (const const16*)(bc + (long long)tile * kTile * 2 * P);
#pragma unroll(P == 16 ? 1 : P)
    for (int q = 0; q < P; ++q) {
      // the next 32 values; behind a tile's last ones those of the next tile
      const f32x16 n0 = at[2 * q + 2], n1 = at[2 * q + 3];
      // all exp2 of the batch ahead of their uses, which would wait for them one by one
      float2 x[kBatch];
      float decay[kBatch][P];
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        x[k] = get(q * kBatch + k);
        decays(x[k].x, decay[k]);
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        const float out = walk(decay[k], x[k].y, [&](int i) { const int w = k * 2 * P + i; return w < 16 ? v0[w & 15] : v1[w & 15]; });
        if (ENDS) sum += x[k].x; else put(q * kBatch + k, out);
      }
      v0 = n0;
      v1 = n1;
      __builtin_amdgcn_sched_barrier(0);       // or all batches' loads move to the front and spill
    }
  };
  auto part_tile = [&](int tile, int some, auto&& get, auto&& put) {
#pragma unroll 1
    for (int j = 0; j < some; ++j) {
      const auto* at = (const __attribute__((address_space(4))) float*)(bc + (long long)(tile * kTile + j) * 2 * P);
      const float2 x = get(j);
      float decay[P];
      decays(x.x, decay);
      const float out = walk(decay, x.y, [&](int i) { return at[i]; });
      if (ENDS) sum += x.x; else put(j, out);
    }
  };

  auto prepare = [&](int buf, const unsigned (&uv)[kOwn], const unsigned (&dv)[kOwn]) {
#pragma unroll
    for (int k = 0; k < kOwn; ++k) {
      const float v = step_size(dv[k]);
      dd[buf][k * F + f][lane] = float2{v, v * raw_value<T>(uv[k])};
    }
  };
  auto complete = [&](int tile, const unsigned (&uv)[kOwn], const unsigned (&zv)[kOwn]) {
    float o[kOwn];
#pragma unroll
    for (int k = 0; k < kOwn; ++k) {
      float out = part[tile & 1][0][k * F + f][lane];
#pragma unroll
      for (int w = 1; w < F; ++w) out += part[tile & 1][w][k * F + f][lane];
      o[k] = finished(out, uv[k], zv[k]);
    }
    store(tile, o);
  };
  // u and dt of the next tile; u of this one; u and z of the one before, for
  // its outputs.  Every load goes to the registers of values just used, so
  // that it has a tile's time to arrive and no copy waits for it.
  unsigned u0[kOwn], u1[kOwn], d1[kOwn], ub[kOwn], zb[kOwn];
  if (tiles > 0) {
    load(u, ldu, 0, u0);
    load(dt, lddt, 0, d1);
    prepare(0, u0, d1);
    load(u, ldu, 1, u1);
    load(dt, lddt, 1, d1);
    v0 = ((const const16*)bc)[0];
    v1 = ((const const16*)bc)[1];
  }
  for (int tile = 0; tile < tiles; ++tile) {
    wave_barrier_lds();
    const int buf = tile & 1;
    const int some = min(kTile, tokens - tile * kTile);
    // read ahead: a wait for LDS also waits for scalar loads
    constexpr bool kAhead = P * F < 256;       // else too few registers
    float2 x[kAhead ? kTile : 1];
    if (kAhead) {
#pragma unroll
      for (int j = 0; j < kTile; ++j) x[j] = dd[buf][j][lane];
    }
    if (!ENDS) {
      if (tile > 0) complete(tile - 1, ub, zb);
      load(z, ldz, tile, zb);
    }
    if (some == kTile) {
      // LDS is waited for here, before whole_tile's scalar loads are under way
      __builtin_amdgcn_s_waitcnt(0xc07f);      // lgkmcnt(0)
      whole_tile(tile, [&](int j) { return kAhead ? x[kAhead ? j : 0] : dd[buf][j][lane]; },
                 [&](int j, float out) { part[buf][f][j][lane] = out; });
    } else {
      part_tile(tile, some, [&](int j) { return dd[buf][j][lane]; },
                [&](int j, float out) { part[buf][f][j][lane] = out; });
    }
    prepare(buf ^ 1, u1, d1);
#pragma unroll
    for (int k = 0; k < kOwn; ++k) {
      ub[k] = u0[k];
      u0[k] = u1[k];
    }
    load(u, ldu, tile + 2, u1);
    load(dt, lddt, tile + 2, d1);
  }
  if (!ENDS && tiles > 0) {
    wave_barrier_lds();
    complete(tiles - 1, ub, zb);
  }

  if (!live) return;
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const int s = f * P + i;
    if (s >= p.S) continue;
    if (ENDS) a.slots[((long long)id * p.S + s) * p.D + d] = h[i];
    else if (last && p.state != nullptr) p.state[((long long)n * p.D + d) * p.S + s] = h[i];
  }
  if (ENDS && f == 0) a.sums[(long long)id * p.D + d] = sum;
}

// The pairs that scan_plan takes.
template <typename T, bool ENDS>
ScanFn scan_kernel_of(int P, int F) {
  switch (P * 100 + F) {
    case 202: return scan_pieces<T, 2, 2, ENDS>;
    case 204: return scan_pieces<T, 2, 4, ENDS>;
    case 208: return scan_pieces<T, 2, 8, ENDS>;
    case 404: return scan_pieces<T, 4, 4, ENDS>;
    case 408: return scan_pieces<T, 4, 8, ENDS>;
    case 808: return scan_pieces<T, 8, 8, ENDS>;
    case 816: return scan_pieces<T, 8, 16, ENDS>;
    case 1616: return scan_pieces<T, 16, 16, ENDS>;
    default: return nullptr;
  }
}
template <typename T>
ScanFn scan_kernel(int P, int F, bool ends) {
  return ends ? scan_kernel_of<T, true>(P, F) : scan_kernel_of<T, false>(P, F);
}

}  // namespace mg3m
