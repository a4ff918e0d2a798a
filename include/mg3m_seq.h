/*
 * mg3m_seq.h -- sequence operators of the MI355X (gfx950) convolution library:
 * the causal short convolution over tokens, the selective state space scan
 * behind it, and the product of single tokens with 4-bit weights.  With the
 * 1x1 convolutions of mg3m.h they make up a state space layer, for prompts
 * and for single tokens.  Inference only: there are no gradients here.
 *
 * Tensors.  Activations are rows of tokens, x[t][c] at x + t * ldx + c: the
 * channels of a token are contiguous, the distance ldx between tokens (in
 * elements, at least the channel count, at most 2^30) is free, so a tensor may be some
 * columns of a wider one.  With ldx = C this is an HWCN image of height 1,
 * width T and one image, x[1][T][C][1].  Their type (argument dtype) is fp32,
 * bf16 or fp16; sums, states and step sizes are fp32 in every type, and each
 * result is rounded once (to nearest, ties to even).
 *
 * Sequences.  A call over T rows holds N sequences.  Sequence n has the rows
 * begin[n] <= t < end[n] (device arrays of N ints, begin ascending, end[n] <=
 * begin[n+1]); rows between the sequences are neither read into a result nor
 * written.  A packed batch passes its N+1 offsets as begin = offsets, end =
 * offsets + 1; a padded one begin[n] = n * L, end[n] = n * L + length[n].  A
 * sequence may be empty.  With begin and end NULL the N sequences have T / N
 * rows each, one after the other (T a multiple of N).  Values outside
 * 0..T are taken as the nearest of them, and an end before its begin as an
 * empty sequence; begins that descend or rows in two sequences give
 * unspecified results, but no access outside the tensors.
 *
 * States are dense, one per sequence, and updated in place, so that a prompt
 * may come in pieces and single tokens may follow it.  state NULL: sequences
 * start from nothing and nothing is kept.  load_state 0: they start from
 * nothing and the state is written; 1: they start from the state.
 *
 * Everything else is as in mg3m.h: device pointers on the current device,
 * asynchronous and ordered on `stream`, an mg3m_status returned, arguments
 * checked before anything is launched, the detail in mg3m_last_error(), no
 * C++ exception across the interface, no pointer kept.  Checked beyond the
 * rules there: MG3M_ERR_ARG for an unknown dtype or a flag other than 0 and 1
 * or a begin without an end; MG3M_ERR_ALIGN for a pointer not aligned to its
 * element; MG3M_ERR_ALIAS if an output (y, state) shares an element with any
 * other tensor, where rows of one distance that interleave without sharing an
 * element are accepted; MG3M_ERR_TOO_LARGE for T above 2^31 - 2^16, C (of the
 * convolution), M, K or D * S above 2^30, C of the 4-bit product above 2^20, or
 * more threads than a launch takes (2^32).  N and M are at least 1, T may be 0.
 * Tensors may exceed 4 GiB.
 *
 * Infinities and NaN in a tensor reach the results that the formulas take them
 * to, there as either of the two, and no others; rows outside the sequences
 * may hold them.  Sums of the 4-bit product are formed before the group's scale
 * and, of 16-bit tokens, with 16 added to q, so tokens or scales above 2^112 may
 * overflow.
 */
#ifndef MG3M_SEQ_H
#define MG3M_SEQ_H

#include "mg3m.h"

#ifdef __cplusplus
extern "C" {
#endif

enum mg3m_dtype {
    MG3M_F32 = 0,
    MG3M_BF16 = 1,
    MG3M_F16 = 2
};

/* Causal convolution of every channel by itself (depthwise) along the tokens
 * of a sequence:
 *   y[t][c] = act(bias[c] + sum_{r<R} w[r][c] * x[t - (R-1) + r][c]),
 * Eq. 1 with height 1, R taps, R-1 columns of padding on the left only, one
 * input channel per output channel.  Rows before the sequence's first are
 * those of its state (the oldest first), or zeros.  act: none, or SiLU
 * (v * sigmoid(v)).  The state after is the last R-1 rows of (state, x).
 * R is 1..8; with R = 1 there is no state. */
typedef struct mg3m_conv1d {
    const void *x;            /* [T][C], distance ldx */
    const void *w;            /* [R][C], dense, the type of x */
    const void *bias;         /* [C], the type of x, or NULL */
    void *state;              /* [N][R-1][C], dense, the type of x, or NULL */
    void *y;                  /* [T][C], distance ldy, the type of x */
    const int *begin, *end;   /* [N] each, or both NULL */
    long long ldx, ldy;
    int T, C, R, N;
    int load_state, silu, dtype;
    int reserved;             /* 0 */
} mg3m_conv1d;

int conv1d_causal_fwd(const mg3m_conv1d *a, void *stream);

/* One token of each of N sequences: x and y are [N][C] (T is ignored, begin
 * and end must be NULL), state is required if R > 1 and read whatever
 * load_state says. */
int conv1d_causal_step(const mg3m_conv1d *a, void *stream);

/* Selective state space scan.  For every sequence and channel d, in the group
 * g = d / (D / G), over the tokens t, with the state h[s], s < S:
 *   delta = dt[t][d] + dt_bias[d];  softplus: delta = log(1 + exp(delta))
 *   h[s]  = exp(delta * A[d][s]) * h[s] + delta * B[t][g][s] * u[t][d]
 *   y     = sum_s C[t][g][s] * h[s] + D[d] * u[t][d]
 *   y[t][d] = z ? y * z[t][d] * sigmoid(z[t][d]) : y
 * S is 1..256, G divides D.  exp of a token's delta * A is an fp32 number:
 * infinite for exponents above 88, where states grow, and zero below -87; rates
 * are below 2^127 in size, or infinite.  Long prompts of few channels are cut along the
 * tokens: the pieces run side by side and are joined through their end states
 * (in a fixed order: results are the same from run to run).
 * workspace: selective_scan_workspace_bytes() of device memory, 16-byte
 * aligned, or NULL for the one that the library keeps for `stream`
 * (mg3m.h, conv2d_fwd_f32; mg3m_trim_workspace_pool gives it back).  Calls in
 * captured graphs that may run side by side want a workspace each. */
typedef struct mg3m_scan {
    const void *u, *dt;       /* [T][D], distances ldu, lddt */
    const float *A;           /* [D][S], dense */
    const void *B, *C;        /* [T][G][S], a row dense, distances ldb, ldc */
    const float *D_skip;      /* [D], or NULL for 0 */
    const void *z;            /* [T][D], distance ldz, or NULL */
    const float *dt_bias;     /* [D], or NULL for 0 */
    float *state;             /* [N][D][S], dense, or NULL */
    void *y;                  /* [T][D], distance ldy */
    const int *begin, *end;   /* [N] each, or both NULL */
    void *workspace;
    size_t workspace_bytes;
    long long ldu, lddt, ldb, ldc, ldz, ldy;
    int T, D, G, S, N;
    int load_state, softplus, dtype;
} mg3m_scan;

int selective_scan_fwd(const mg3m_scan *a, void *stream);

/* Bytes of workspace that selective_scan_fwd needs for these sizes, whatever
 * the sequences' lengths.  Host only. */
int selective_scan_workspace_bytes(int T, int D, int G, int S, int N, size_t *bytes);

/* One token of each of N sequences: the row tensors are [N][...] (T is
 * ignored, begin and end must be NULL), state is required and read whatever
 * load_state says.  Takes no workspace. */
int selective_scan_step(const mg3m_scan *a, void *stream);

/* Product of M tokens with 4-bit weights:
 *   y[m][k] = sum_c x[m][c] * scale[k][c / group] * (q[k][c] - zero[k][c / group])
 * q: [K][C/2] bytes, the even c in the low four bits, values 0..15 (16-byte
 * aligned); scale: [K][C/group] of the type of x; zero: [K][C/group] bytes,
 * or NULL for 8.  group is a multiple of 32 that divides C.  Made for few
 * tokens: each 16 tokens read the weights once.  fp32 channels below 2^-100
 * lose low bits. */
typedef struct mg3m_w4 {
    const void *x;            /* [M][C], distance ldx */
    const unsigned char *q;
    const void *scale;
    const unsigned char *zero;
    void *y;                  /* [M][K], distance ldy */
    long long ldx, ldy;
    int M, C, K, group, dtype;
    int reserved;             /* 0 */
} mg3m_w4;

int matvec_w4_fwd(const mg3m_w4 *a, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* MG3M_SEQ_H */
