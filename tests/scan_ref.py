"""64-bit reference of the selective scan (include/mg3m_seq.h), the sequences
side by side, and how far fp32 arithmetic may be from it when prompts are cut
into pieces of W tokens (0: not cut).  Units as in seq_ref.py: H is half a step
of fp32."""
import torch

from seq_ref import H, sigmoid_units

FLUSH = 2.0 ** -126          # what a product below fp32's normal range may lose


def scan(u, dt, A, B, C, D, z, dt_bias, softplus, state, ranges, load, W=0):
    """(y, state, bound of y's error before its last rounding, bound of the
    state's error), on the tensors' device; rows outside the sequences stay NaN."""
    T, Dn = u.shape
    G, S = B.shape[1:]
    N = len(ranges)
    on_device = dict(dtype=torch.float64, device=u.device)
    u, dt, A, B, C = (v.double() for v in (u, dt, A, B, C))
    bias = torch.zeros(Dn, **on_device) if dt_bias is None else dt_bias.double()
    skip = torch.zeros(Dn, **on_device) if D is None else D.double()
    y, tol = torch.full((T, Dn), float("nan"), **on_device), torch.zeros(T, Dn, **on_device)
    of = torch.arange(Dn, device=u.device) // (Dn // G)
    begin, lens = (torch.tensor(v, device=u.device) for v in ([b for b, _ in ranges], [max(0, e - b) for b, e in ranges]))
    h = state.double().clone() if load else torch.zeros(N, Dn, S, **on_device)
    err = torch.zeros_like(h)
    # of the piece so far: the state from nothing and its error, what it started
    # from and that one's error, the exponent of its factor and its error
    own, own_err, start, start_err, far, far_err = (torch.zeros_like(h) for _ in range(6))
    for t in range(int(lens.max()) if N else 0):
        on = (lens > t).nonzero()[:, 0]
        rows = begin[on] + t
        if W and t % W == 0:
            if t:
                # a piece starts from factor * start + the piece's own end: the factor's exponent
                # is a sum of W steps (a rounding each) times A log2e (three); exp2 2, two products
                # (the second a power of two, which may leave the normal range) and the sum 1 each
                f = torch.exp(far[on])
                carried = (f * start[on]).abs()
                err[on] = (f * start_err[on] + carried * (far_err[on] + 3 * H) + own_err[on] + FLUSH
                           + (f * start[on] + own[on]).abs() * H)
                h[on] = f * start[on] + own[on]
            start[on], start_err[on] = h[on], err[on]
            for v in (own, own_err, far, far_err):
                v[on] = 0.0
        raw = dt[rows] + bias
        delta = torch.nn.functional.softplus(raw, threshold=100.0) if softplus else raw
        # roundings of the step, relative to it: seq_ref.scan counts them
        rho = ((3 * raw.abs().clamp_max(150) + 24) * H if softplus
               else (raw.abs() / delta.abs().clamp_min(1e-300)) * H)[..., None]
        x = delta[..., None] * A
        a = torch.exp(x)
        rho_a = x.abs() * (rho + 3 * H) + 2 * H
        term = (delta * u[rows])[..., None] * B[rows][:, of]
        term_err = term.abs() * (rho + 2 * H) + FLUSH

        def step(v, e):
            e = a * e + (a * v).abs() * rho_a + term_err
            v = a * v + term
            return v, e + v.abs() * H
        h[on], err[on] = step(h[on], err[on])
        if W:
            own[on], own_err[on] = step(own[on], own_err[on])
            far[on] += x
            far_err[on] += x.abs() * (rho + (3 + W) * H)
        c = C[rows][:, of]
        size = (c * h[on]).abs().sum(-1) + (skip * u[rows]).abs()
        y[rows] = (c * h[on]).sum(-1) + skip * u[rows]
        tol[rows] = (c.abs() * err[on]).sum(-1) + (S + 2) * H * size + FLUSH
    if z is not None:
        z = z.double()
        gate = z * torch.sigmoid(z)
        tol = tol * gate.abs() + (y * gate).abs().nan_to_num() * (sigmoid_units(z) + 2 * H)
        y = y * gate
    return y, h, tol, err
