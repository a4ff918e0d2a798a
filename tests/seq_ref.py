"""64-bit references of the sequence operators (include/mg3m_seq.h) on the
CPU, written from their formulas with plain loops over sequences and tokens,
and how far fp32 arithmetic may be from them.

Roundings are counted in units of 2^-24, half a step of fp32.  The kernels'
exp2, log2 and reciprocal are good to one step (2 units)."""
import torch

H = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
# half the smallest subnormal: what rounding to the type may add to a relative bound
TINY = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -25}


def half_step(t):
    return torch.finfo(t).eps / 2


def stored(y, tol, t):
    """The bound with the rounding of the result to type t on top."""
    return tol + (y.abs() + tol) * half_step(t) + TINY[t]


def sigmoid_units(v):
    """Relative error of sigmoid(v) = 1 / (1 + exp2(-v * log2e)): the constant
    and the product round (2 units of the exponent |v|), then exp2 (2), the sum
    (1) and the reciprocal (2)."""
    return (2 * v.abs() + 5) * H


def conv(x, w, bias, state, ranges, load, silu):
    """(y, state, bound of |error| of y before its last rounding) of the
    sequences ranges = [(begin, end)] of the rows of x; rows outside stay NaN."""
    T, C = x.shape
    R = w.shape[0]
    x, w = x.double(), w.double()
    y, tol = torch.full((T, C), float("nan"), dtype=torch.float64), torch.zeros(T, C, dtype=torch.float64)
    b0 = torch.zeros(C, dtype=torch.float64) if bias is None else bias.double()
    after = []
    for n, (b, e) in enumerate(ranges):
        past = state[n].double() if load else torch.zeros(R - 1, C, dtype=torch.float64)
        rows = torch.cat([past, x[b:e]])
        after.append(rows[len(rows) - (R - 1):])
        for t in range(b, e):
            v = rows[t - b:t - b + R]
            y[t] = b0 + (w * v).sum(0)
            # R products in a chain of fused multiply-adds: R roundings, each of at most the sum of magnitudes
            tol[t] = R * H * (b0.abs() + (w * v).abs().sum(0))
    if silu:
        # |d silu / dv| <= 1.1; the sigmoid and the product round
        v = y
        y = v * torch.sigmoid(v)
        tol = 1.1 * tol + y.abs().nan_to_num() * (sigmoid_units(v.nan_to_num()) + H)
    return y, torch.stack(after) if after else None, tol


# The largest piece that a prompt is cut into (scan.hip): its step sizes are
# summed in fp32, one rounding each.
PIECE = 512


def scan(u, dt, A, B, C, D, z, dt_bias, softplus, state, ranges, load):
    """(y, state, bound of y's error before its last rounding, bound of the state's error)."""
    T, Dn = u.shape
    G, S = B.shape[1:]
    u, dt, A, B, C = (v.double() for v in (u, dt, A, B, C))
    bias = torch.zeros(Dn, dtype=torch.float64) if dt_bias is None else dt_bias.double()
    skip = torch.zeros(Dn, dtype=torch.float64) if D is None else D.double()
    y, tol = torch.full((T, Dn), float("nan"), dtype=torch.float64), torch.zeros(T, Dn, dtype=torch.float64)
    of = torch.arange(Dn) // (Dn // G)
    after, after_tol = [], []
    for n, (b, e) in enumerate(ranges):
        h = state[n].double() if load else torch.zeros(Dn, S, dtype=torch.float64)
        err = torch.zeros_like(h)
        for t in range(b, e):
            raw = dt[t] + bias
            delta = torch.nn.functional.softplus(raw, threshold=100.0) if softplus else raw
            # the sum rounds (1 unit of |raw|, which softplus passes on to at most |raw| relative units of
            # itself); exp2's argument (2 |raw|); exp2, log2 and the reciprocal (2 each), three sums and
            # three products (1 each), and as much again for 1 + e standing in for the exact sum.  Below -150
            # the step is under 2^-216 and 0 in fp32, which 2^-126 on the state covers: no relative error counts
            rho = ((3 * raw.abs().clamp_max(150) + 24) * H if softplus else (raw.abs() / delta.abs().clamp_min(1e-300)) * H)[:, None]
            x = (delta[:, None] * A).abs()
            a = torch.exp(delta[:, None] * A)
            # exp2(delta * (A log2e)): three roundings of the exponent, and a piece's sum of step sizes; exp2: 2
            rho_a = x * (rho + (3 + PIECE) * H) + 2 * H
            term = (delta * u[t])[:, None] * B[t][of]
            err = a * err + (a * h).abs() * rho_a + term.abs() * (rho + 2 * H)
            h = a * h + term
            err = err + h.abs() * H + 2.0 ** -126
            out = (C[t][of] * h).sum(1) + skip * u[t]
            # S + 1 products and their sum, in any order: at most one rounding per term
            size = (C[t][of] * h).abs().sum(1) + (skip * u[t]).abs()
            y[t] = out
            tol[t] = (C[t][of].abs() * err).sum(1) + (S + 2) * H * size
        after.append(h)
        after_tol.append(err)
    if z is not None:
        z = z.double()
        gate = z * torch.sigmoid(z)
        # the sigmoid, z * sigmoid and the product with y round
        tol = tol * gate.abs() + (y * gate).abs().nan_to_num() * (sigmoid_units(z) + 2 * H)
        y = y * gate
    return y, torch.stack(after), tol, torch.stack(after_tol)


def w4(x, q, scale, zero, group):
    """(y, bound).  Each product is exact but for the group's scale; a sum of
    C terms, whose magnitudes are taken at 31 (weights may enter with 16
    added, which is taken out of the sum), rounds at most once per term and
    twice per group."""
    K, C = q.shape[0], x.shape[1]
    codes = torch.empty(K, C, dtype=torch.float64)
    codes[:, 0::2], codes[:, 1::2] = (q % 16).double(), (q // 16).double()
    zr = torch.full((K, C // group), 8.0, dtype=torch.float64) if zero is None else zero.double()
    s = scale.double().repeat_interleave(group, 1)
    w = (codes - zr.repeat_interleave(group, 1)) * s
    x = x.double()
    return x @ w.t(), (C + 2 * C // group + 8) * H * 31 * (x.abs() @ s.abs().t())
