"""The sequence operators (include/mg3m_seq.h) on the GPU against 64-bit
references (tests/seq_ref.py), with the bounds that their fp32 arithmetic
allows, and exactly on small integers."""
import pytest
import torch

import seq_ref as ref
from paper_2307_04941_amd import mg3m

pytestmark = pytest.mark.gpu
T3 = ["f32", "bf16", "f16"]


def gen(seed):
    return torch.Generator().manual_seed(seed)


def randn(g, *shape, t=torch.float32, std=1.0):
    return (torch.randn(*shape, generator=g) * std).to(t)


def ints(g, lo, hi, *shape, t=torch.float32):
    return torch.randint(lo, hi + 1, shape, generator=g).to(t)


def dev(v):
    return None if v is None else v.cuda()


def near(got, want, tol, what=""):
    got = got.double().cpu()
    bad = ~((got - want).abs() <= tol) & ~(got.isnan() & want.isnan())
    assert not bad.any(), (f"{what}: {int(bad.sum())} of {bad.numel()} outside; first at {bad.nonzero()[0].tolist()}: "
                           f"{got[bad][0].item()!r} against {want[bad][0].item()!r} +- {tol[bad][0].item():.3g}")


def edges_of(lens):
    e = [0]
    for v in lens:
        e.append(e[-1] + v)
    return e


# ------------------------------------------------------------ convolution
LENS = {"one": [1], "long": [777], "ragged": [5, 0, 1, 130, 2, 0, 64], "few": [3, 3, 3]}


def conv_case(t, lens, C, R, seed, bias=True, integer=False, spare=0):
    g = gen(seed)
    T = sum(lens) + spare
    if integer:
        x, w, s = ints(g, -3, 3, T, C, t=t), ints(g, -2, 2, R, C, t=t), ints(g, -3, 3, len(lens), R - 1, C, t=t)
        b = ints(g, -4, 4, C, t=t) if bias else None
    else:
        x, w, s = randn(g, T, C, t=t), randn(g, R, C, t=t), randn(g, len(lens), R - 1, C, t=t)
        b = randn(g, C, t=t) if bias else None
    return x, w, b, s


@pytest.mark.parametrize("t", T3)
@pytest.mark.parametrize("lens,C,R,silu,load", [
    ("one", 1, 4, True, True), ("one", 64, 4, False, False), ("long", 96, 4, True, False), ("long", 33, 3, True, True),
    ("ragged", 200, 4, True, True), ("ragged", 7, 2, False, True), ("ragged", 1024, 4, True, False),
    ("few", 40, 8, True, True), ("few", 17, 5, False, True), ("ragged", 72, 1, True, False),
    ("ragged", 24, 6, False, True), ("long", 8, 7, True, True)])
def test_conv_prompts(t, lens, C, R, silu, load):
    tt, ls = ref.TYPES[t], LENS[lens]
    x, w, b, s = conv_case(tt, ls, C, R, 11 * C + R, bias=C % 3 != 0)
    e = edges_of(ls)
    want, after, tol = ref.conv(x, w, b, s, list(zip(e, e[1:])), load, silu)
    sd = dev(s)
    y = mg3m.conv1d_causal(dev(x), dev(w), dev(b), silu, sd if R > 1 else None, load,
                           offsets=torch.tensor(e, dtype=torch.int32).cuda())
    near(y, want, ref.stored(want, tol, tt), "y")
    if R > 1:
        assert torch.equal(sd.cpu().double(), after)          # inputs, kept as they are


@pytest.mark.parametrize("t", T3)
@pytest.mark.parametrize("C,R", [(1, 2), (65, 4), (512, 4), (2056, 3), (100, 8)])
def test_conv_integers_are_exact(t, C, R):
    tt, ls = ref.TYPES[t], [259, 1, 0, 33, 700]
    x, w, b, s = conv_case(tt, ls, C, R, C + R, integer=True)
    e = edges_of(ls)
    want, after, _ = ref.conv(x, w, b, s, list(zip(e, e[1:])), True, False)
    sd = dev(s)
    y = mg3m.conv1d_causal(dev(x), dev(w), dev(b), False, sd, True, offsets=torch.tensor(e, dtype=torch.int32).cuda())
    assert torch.equal(y.cpu().double(), want) and torch.equal(sd.cpu().double(), after)


@pytest.mark.parametrize("t", T3)
def test_conv_equal_parts_and_no_state(t):
    tt = ref.TYPES[t]
    x, w, b, s = conv_case(tt, [50] * 6, 48, 4, 3)
    want, _, tol = ref.conv(x, w, b, s, [(50 * i, 50 * i + 50) for i in range(6)], False, True)
    y = mg3m.conv1d_causal(dev(x).view(6, 50, 48), dev(w), dev(b), True)
    near(y.reshape(300, 48), want, ref.stored(want, tol, tt))
    sd = torch.full((6, 3, 48), 7.0, dtype=tt).cuda()          # not loaded: overwritten
    y2 = mg3m.conv1d_causal(dev(x).view(6, 50, 48), dev(w), dev(b), True, sd)
    assert torch.equal(y, y2) and torch.equal(sd.cpu(), x.view(6, 50, 48)[:, 47:])


@pytest.mark.parametrize("t", T3)
@pytest.mark.parametrize("C,off,ldx,ldy", [(64, 0, 96, 72), (64, 3, 131, 64), (40, 8, 64, 41), (256, 0, 512, 256)])
def test_conv_strided_rows_padded_batch_and_rows_left_alone(t, C, off, ldx, ldy):
    """Columns of wider tensors, sequences that do not fill their part of the
    batch, rows before, between and behind them."""
    tt, L = ref.TYPES[t], 37
    g = gen(C + off)
    wide, s = randn(g, 4 * L, ldx, t=tt), randn(g, 4, 3, C, t=tt)
    w, b = randn(g, 4, C, t=tt), randn(g, C, t=tt)
    begin, end = [5, L, 2 * L + 1, 3 * L], [30, L, 3 * L, 3 * L + 2]
    x = wide[:, off:off + C]
    want, after, tol = ref.conv(x, w, b, s, list(zip(begin, end)), True, True)
    out = torch.full((4 * L, ldy), float("nan"), dtype=tt).cuda()
    sd = dev(s)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32).cuda()  # noqa: E731
    mg3m.conv1d_causal(dev(wide)[:, off:off + C], dev(w), dev(b), True, sd, True, begin=i32(begin), end=i32(end),
                       out=out[:, :C])
    near(out[:, :C], want, ref.stored(want, tol, tt), "y (NaN: left alone)")
    assert out[:, C:].isnan().all() and torch.equal(sd.cpu().double(), after)


@pytest.mark.parametrize("t", T3)
@pytest.mark.parametrize("N,C,R,silu", [(1, 1, 4, True), (1, 2048, 4, True), (37, 300, 3, False), (130, 64, 2, True),
                                        (5, 77, 8, True), (3, 50, 1, False), (300, 1032, 4, True)])
def test_conv_step(t, N, C, R, silu):
    tt = ref.TYPES[t]
    x, w, b, s = conv_case(tt, [1] * N, C, R, N + C)
    want, after, tol = ref.conv(x, w, b, s, [(i, i + 1) for i in range(N)], True, silu)
    sd = dev(s)
    y = mg3m.conv1d_causal_step(dev(x), dev(w), sd if R > 1 else None, dev(b), silu)
    near(y, want, ref.stored(want, tol, tt))
    if R > 1:
        assert torch.equal(sd.cpu().double(), after)


def test_conv_special_values():
    """Infinities and NaN reach the outputs that their taps reach, and no other."""
    C, L = 8, 40
    x = torch.zeros(L, C)
    x[10, 1], x[20, 2], x[30, 3] = float("nan"), float("inf"), float("-inf")
    w = torch.ones(4, C)
    want, _, tol = ref.conv(x, w, None, None, [(0, L)], False, False)
    y = mg3m.conv1d_causal(dev(x), dev(w)).cpu().double()
    assert torch.equal(y.isnan(), want.isnan())
    assert torch.equal(y.nan_to_num(0.0, 9.0, -9.0), want.nan_to_num(0.0, 9.0, -9.0))


# ------------------------------------------------------------------- scan
def scan_case(t, T, N, D, S, G, seed, gate=True, rest=True):
    g = gen(seed)
    return dict(u=randn(g, T, D, t=t), dt=randn(g, T, D, t=t), A=-torch.rand(D, S, generator=g) * 4 - 0.01,
                B=randn(g, T, G, S, t=t), C=randn(g, T, G, S, t=t), D=randn(g, D) if rest else None,
                z=randn(g, T, D, t=t, std=2.0) if gate else None,
                dt_bias=randn(g, D) - 3 if rest else None, state=randn(g, N, D, S))


def scan_want(c, ranges, softplus, load):
    return ref.scan(c["u"], c["dt"], c["A"], c["B"], c["C"], c["D"], c["z"], c["dt_bias"], softplus, c["state"], ranges,
                    load)


def scan_run(c, state, softplus=True, load=True, **kw):
    return mg3m.selective_scan(dev(c["u"]), dev(c["dt"]), dev(c["A"]), dev(c["B"]), dev(c["C"]), dev(c["D"]),
                               dev(c["z"]), dev(c["dt_bias"]), softplus, state, load, **kw)


@pytest.mark.parametrize("t", T3)
@pytest.mark.parametrize("lens,D,S,G,gate,rest,load", [
    ([1], 1, 1, 1, False, False, False), ([300], 64, 16, 1, True, True, False), ([1100], 20, 16, 1, True, True, True),
    ([5, 0, 1, 130, 2, 0, 64], 100, 16, 1, True, True, True), ([3, 0, 257, 65], 130, 13, 2, True, True, True),
    ([70, 70], 48, 32, 3, False, True, False), ([33, 1], 66, 1, 1, True, False, True), ([40], 10, 65, 2, True, True, True),
    ([20, 9], 8, 256, 1, False, True, True), ([90], 200, 5, 4, True, True, False), ([0, 0], 16, 16, 1, True, True, True)])
def test_scan_prompts(t, lens, D, S, G, gate, rest, load):
    tt = ref.TYPES[t]
    c = scan_case(tt, sum(lens), len(lens), D, S, G, D + S, gate, rest)
    e = edges_of(lens)
    want, after, tol, atol = scan_want(c, list(zip(e, e[1:])), True, load)
    sd = dev(c["state"])
    y = scan_run(c, sd, load=load, offsets=torch.tensor(e, dtype=torch.int32).cuda())
    near(y, want, ref.stored(want, tol, tt), "y")
    near(sd, after, atol, "state")


@pytest.mark.parametrize("N,L,D,S", [(1, 4096, 64, 16), (2, 1000, 256, 16), (1, 513, 1536, 4), (40, 60, 128, 16),
                                     (3, 700, 200, 24), (1, 2000, 5, 100), (70, 3, 640, 8)])
def test_scan_of_ones_is_an_exact_sum(N, L, D, S):
    """A = 0 and delta = 1: the state is the running sum of B u, exact on
    integers however the tokens are cut."""
    g = gen(L)
    u, B, C = ints(g, -2, 2, N, L, D), ints(g, -2, 2, N, L, 1, S), ints(g, -1, 1, N, L, 1, S)
    s0 = ints(g, -5, 5, N, D, S)
    h = s0[:, None].double() + torch.cumsum(u[..., None].double() * B.double(), 1)
    want = (h * C.double()).sum(-1)
    sd = dev(s0)
    y = mg3m.selective_scan(dev(u), torch.ones(N, L, D).cuda(), torch.zeros(D, S).cuda(), dev(B), dev(C), state=sd,
                            load_state=True)
    assert torch.equal(y.cpu().double(), want)
    assert torch.equal(sd.cpu().double(), h[:, -1])


@pytest.mark.parametrize("t", T3)
@pytest.mark.parametrize("softplus", [False, True])
def test_scan_equal_parts_without_state(t, softplus):
    tt = ref.TYPES[t]
    c = scan_case(tt, 4 * 61, 4, 72, 16, 1, 5)
    if not softplus:
        c["dt"], c["dt_bias"] = (c["dt"].abs() * 0.1).to(tt), None
    want, after, tol, atol = scan_want(c, [(61 * i, 61 * i + 61) for i in range(4)], softplus, False)
    c3 = {k: v.view(4, 61, *v.shape[1:]) if k in ("u", "dt", "B", "C", "z") else v for k, v in c.items()}
    y = scan_run(c3, None, softplus, False)
    near(y.reshape(244, 72), want, ref.stored(want, tol, tt))
    sd = torch.full((4, 72, 16), 9.0).cuda()                   # not loaded: overwritten
    assert torch.equal(scan_run(c3, sd, softplus, False), y)
    near(sd, after, atol, "state")


@pytest.mark.parametrize("t", T3)
@pytest.mark.parametrize("D,S,G", [(64, 16, 1), (50, 7, 2)])
def test_scan_slices_of_one_projection_padded_batch(t, D, S, G):
    """B, C, dt and z as columns of wider tensors, y into one, sequences in a
    padded batch; rows outside them stay as they are."""
    tt, L = ref.TYPES[t], 45
    c = scan_case(tt, 3 * L, 3, D, S, G, 17)
    begin, end = [2, L, 2 * L], [L, L + 1, 3 * L - 3]
    want, after, tol, atol = scan_want(c, list(zip(begin, end)), True, True)
    proj = torch.cat([c["dt"], c["B"].flatten(1), c["C"].flatten(1), c["z"]], 1).cuda()
    d, gs = D, G * S
    buf = torch.full((3 * L, 2 * D + 3), float("nan"), dtype=tt).cuda()
    buf[:, :D] = dev(c["u"])
    i32 = lambda v: torch.tensor(v, dtype=torch.int32).cuda()  # noqa: E731
    sd = dev(c["state"])
    # u and y are columns of one tensor
    mg3m.selective_scan(buf[:, :D], proj[:, :d], dev(c["A"]), proj[:, d:d + gs].unflatten(1, (G, S)),
                        proj[:, d + gs:d + 2 * gs].unflatten(1, (G, S)), dev(c["D"]), proj[:, d + 2 * gs:],
                        dev(c["dt_bias"]), True, sd, True, begin=i32(begin), end=i32(end), out=buf[:, D:2 * D])
    near(buf[:, D:2 * D], want, ref.stored(want, tol, tt), "y (NaN: left alone)")
    assert buf[:, 2 * D:].isnan().all() and torch.equal(buf[:, :D].cpu(), c["u"])
    near(sd, after, atol, "state")


@pytest.mark.parametrize("t", T3)
@pytest.mark.parametrize("N,D,S,G,gate,rest", [
    (1, 1, 1, 1, False, False), (1, 2048, 16, 1, True, True), (33, 100, 13, 2, True, True), (7, 65, 64, 1, False, True),
    (200, 64, 8, 1, True, True), (2, 30, 256, 3, True, False), (3, 48, 100, 1, True, True)])
def test_scan_step(t, N, D, S, G, gate, rest):
    tt = ref.TYPES[t]
    c = scan_case(tt, N, N, D, S, G, N + S, gate, rest)
    want, after, tol, atol = scan_want(c, [(i, i + 1) for i in range(N)], True, True)
    sd = dev(c["state"])
    y = mg3m.selective_scan_step(dev(c["u"]), dev(c["dt"]), dev(c["A"]), dev(c["B"]), dev(c["C"]), sd, dev(c["D"]),
                                 dev(c["z"]), dev(c["dt_bias"]), True)
    near(y, want, ref.stored(want, tol, tt), "y")
    near(sd, after, atol, "state")


@pytest.mark.parametrize("raw", [-80.0, -30.0, -17.0, -16.0, -5.0, -0.5, 0.0, 0.5, 5.0, 20.0, 80.0])
def test_softplus_keeps_its_relative_precision(raw):
    """One token, A = 0, B = u = C = 1: y is the step size itself."""
    x = torch.linspace(raw - 0.45, raw + 0.45, 640).view(1, 640)
    one = torch.ones(1, 640).cuda()
    y = mg3m.selective_scan_step(one, dev(x), torch.zeros(640, 1).cuda(), torch.ones(1, 1).cuda(), torch.ones(1, 1).cuda(),
                                 torch.zeros(1, 640, 1).cuda(), softplus=True)
    want = torch.nn.functional.softplus(x.double(), threshold=100.0)
    near(y, want, want * (3 * x.double().abs() + 24) * ref.H + 2.0 ** -126)


def test_scan_special_values_stay_in_their_channel():
    """An infinite or NaN input reaches its own channel's later outputs only;
    a step of zero leaves the state as it was."""
    T, D, S = 300, 70, 16
    c = scan_case(torch.float32, T, 1, D, S, 1, 3, gate=False)
    c["u"][100, 5], c["u"][200, 6] = float("nan"), float("inf")
    c["dt"][50:, 7] = float("-inf")
    want, after, tol, atol = scan_want(c, [(0, T)], True, True)
    sd = dev(c["state"])
    y = scan_run(c, sd).cpu().double()
    bad = ~want.isfinite()
    assert not y[bad].isfinite().any() and y[~bad].isfinite().all()
    near(y[~bad], want[~bad], ref.stored(want, tol, torch.float32)[~bad])
    near(sd[0, 7:], after[0, 7:], atol[0, 7:], "state")


# ------------------------------------------------------------- 4-bit product
def w4_case(t, M, C, K, group, seed, zero, integer=False):
    g = gen(seed)
    q = torch.randint(0, 256, (K, C // 2), generator=g, dtype=torch.int32).to(torch.uint8)
    z = torch.randint(0, 16, (K, C // group), generator=g, dtype=torch.int32).to(torch.uint8) if zero else None
    if integer:
        return ints(g, -4, 4, M, C, t=t), q, torch.pow(2.0, ints(g, -6, -5, K, C // group)).to(t), z
    return randn(g, M, C, t=t), q, (0.02 * torch.exp(randn(g, K, C // group, std=0.5))).to(t), z


W4 = [(1, 32, 1, 32, False), (1, 256, 288, 128, True), (2, 96, 33, 32, False), (16, 512, 64, 64, True),
      (5, 2048, 100, 128, False), (13, 640, 17, 160, True), (17, 128, 40, 32, True), (40, 256, 16, 256, False),
      (1, 4096, 1000, 4096, False), (3, 8192, 260, 64, True), (16, 8192, 48, 128, False)]


@pytest.mark.parametrize("t", T3)
@pytest.mark.parametrize("M,C,K,group,zero", W4)
def test_w4(t, M, C, K, group, zero):
    tt = ref.TYPES[t]
    x, q, s, z = w4_case(tt, M, C, K, group, M + C, zero)
    want, tol = ref.w4(x, q, s, z, group)
    y = mg3m.matvec_w4(dev(x), dev(q), dev(s), dev(z))
    near(y, want, ref.stored(want, tol, tt))


@pytest.mark.parametrize("t", T3)
@pytest.mark.parametrize("M,C,K,group,zero", W4 + [(8, 12288, 500, 128, True), (1, 28672, 20, 32, True)])
def test_w4_integers_are_exact(t, M, C, K, group, zero):
    """Small integers and power-of-two scales: every partial sum is exact."""
    tt = ref.TYPES[t]
    x, q, s, z = w4_case(tt, M, C, K, group, C + K, zero, integer=True)
    want, _ = ref.w4(x, q, s, z, group)
    y = mg3m.matvec_w4(dev(x), dev(q), dev(s), dev(z))
    assert torch.equal(y.cpu(), want.to(tt))


def test_w4_strided_rows_and_vector():
    x, q, s, z = w4_case(torch.bfloat16, 4, 256, 50, 64, 9, True)
    wide = torch.zeros(4, 301, dtype=torch.bfloat16).cuda()
    wide[:, 3:259] = dev(x)
    out = torch.full((4, 77), float("nan"), dtype=torch.bfloat16).cuda()
    y = mg3m.matvec_w4(dev(x), dev(q), dev(s), dev(z))
    mg3m.matvec_w4(wide[:, 3:259], dev(q), dev(s), dev(z), out=out[:, 5:55])
    assert torch.equal(out[:, 5:55], y) and out[:, :5].isnan().all() and out[:, 55:].isnan().all()
    assert torch.equal(mg3m.matvec_w4(dev(x[1]), dev(q), dev(s), dev(z)), y[1])


def test_w4_rows_do_not_mix():
    """A NaN or infinite token spoils its own row alone; so does a scale its own column."""
    x, q, s, z = w4_case(torch.float32, 6, 128, 40, 32, 21, True)
    clean = mg3m.matvec_w4(dev(x), dev(q), dev(s), dev(z))
    x[2, 7], x[4, 100] = float("nan"), float("inf")
    y = mg3m.matvec_w4(dev(x), dev(q), dev(s), dev(z))
    assert y[2].isnan().all() and not y[4].isfinite().all()
    keep = [0, 1, 3, 5]
    assert torch.equal(y[keep], clean[keep])
    s[11, 2] = float("nan")
    y = mg3m.matvec_w4(dev(x), dev(q), dev(s), dev(z))
    assert y[keep][:, 11].isnan().all() and torch.equal(y[keep][:, :11], clean[keep][:, :11])
