"""The sequence operators as they are used: a state space layer run over
prompts in parts and then token by token, on streams, in HIP graphs, with the
library's workspace and a caller's, and on tensors past 32-bit offsets.  Every
stage is held to its 64-bit reference on the inputs that it was given."""
import pytest
import torch

import seq_ref as ref
from paper_2307_04941_amd import mg3m
from test_seq_gpu import T3, dev, edges_of, gen, near, randn, scan_case, scan_run, scan_want, w4_case

pytestmark = pytest.mark.gpu


def cpu(v):
    return None if v is None else v.detach().cpu()


# ------------------------------------------------------------ a whole layer
class Layer:
    """x -> (x, z) -> convolution -> (dt, B, C) -> scan, gated by z -> y."""
    M, D, S, RANK, TAPS = 96, 160, 16, 12, 4

    def __init__(self, t, seed=0):
        g = gen(seed)
        D, S, r = self.D, self.S, self.RANK
        self.t = t
        self.q = {}                                    # 4-bit projections, and the same in fp32 for prompts
        for name, c, k in (("in", self.M, 2 * D), ("x", D, r + 2 * S), ("out", D, self.M)):
            _, q, s, z = w4_case(t, 1, c, k, 32, seed + len(name), True)
            s = (s.float() * c ** -0.5).to(t)
            codes = torch.stack([q & 15, q >> 4], -1).flatten(1).float().view(k, c // 32, 32)
            w = ((codes - z.float()[..., None]) * s.float()[..., None]).flatten(1)
            self.q[name] = (q.cuda(), s.cuda(), z.cuda(), w)
        self.dtw = randn(g, r, D, std=r ** -0.5)
        self.w, self.b = randn(g, self.TAPS, D, t=t, std=0.5), randn(g, D, t=t, std=0.1)
        self.A = -torch.rand(D, S, generator=g) * 8 - 0.1
        self.skip, self.bias = randn(g, D), randn(g, D) - 3

    def one_by_one(self, x, w):
        """The library's 1x1 convolution on [T][C] rows: an HWCN image of height 1."""
        T, C = x.shape
        x = x.contiguous()
        y = mg3m.conv2d_fwd(x.view(1, T, C, 1), w.t().contiguous().cuda().view(1, 1, C, -1)).view(T, -1)
        want = x.double().cpu() @ w.double().t()
        near(y, want, 1e-5 * (x.double().cpu().abs() @ w.double().abs().t()) + 1e-30, "1x1")
        return y

    def project(self, x, name, token):
        q, s, z, w = self.q[name]
        if not token:
            return self.one_by_one(x, w)
        y = mg3m.matvec_w4(x, q, s, z)
        want, tol = ref.w4(x.cpu(), q.cpu(), s.cpu(), z.cpu(), 32)
        near(y, want, ref.stored(want, tol, self.t), name)
        return y

    def run(self, x, conv_state, state, ranges=None, offsets=None, load=True):
        """Prompts (ranges, offsets) or one token of each sequence."""
        token, D, S, r, t = ranges is None, self.D, self.S, self.RANK, self.t
        n = state.shape[0]
        if token:
            ranges = [(i, i + 1) for i in range(n)]
        xz = self.project(x, "in", token)
        before, hbefore = cpu(conv_state), cpu(state)
        w, b = dev(self.w), dev(self.b)
        if token:
            u = mg3m.conv1d_causal_step(xz[:, :D], w, conv_state, b, True)
        else:
            u = mg3m.conv1d_causal(xz[:, :D], w, b, True, conv_state, load, offsets=offsets)
        want, after, tol = ref.conv(cpu(xz[:, :D]), self.w, self.b, before, ranges, load, True)
        near(u, want, ref.stored(want, tol, t), "convolution")
        assert torch.equal(cpu(conv_state).double(), after)
        dbc = self.project(u, "x", token)
        dt = self.one_by_one(dbc[:, :r].float(), self.dtw.t()).to(t)
        B, C, z = dbc[:, r:r + S], dbc[:, r + S:], xz[:, D:]
        args = (dt, dev(self.A), B, C)
        if token:
            y = mg3m.selective_scan_step(u, *args, state, dev(self.skip), z, dev(self.bias), True)
        else:
            y = mg3m.selective_scan(u, *args, dev(self.skip), z, dev(self.bias), True, state, load, offsets)
        want, after, tol, atol = ref.scan(cpu(u), cpu(dt), self.A, cpu(B)[:, None], cpu(C)[:, None], self.skip, cpu(z),
                                          self.bias, True, hbefore, ranges, load)
        near(y, want, ref.stored(want, tol, t), "scan")
        near(state, after, atol, "state")
        return self.project(y, "out", token)


def test_layer_prompts_in_parts_then_tokens():
    """Three ragged sequences, their prompts in two parts, then four tokens
    each; the whole is near the layer over the sequences at once, too."""
    layer, g, n, f32 = Layer(torch.float32), gen(5), 3, torch.float32
    parts, tokens = [[70, 3, 0], [5, 130, 41]], 4
    conv_state, state = torch.zeros(n, 3, layer.D).cuda(), torch.zeros(n, layer.D, layer.S).cuda()
    rows, outs = [[] for _ in range(n)], [[] for _ in range(n)]
    for k, lens in enumerate(parts):
        e = edges_of(lens)
        x = randn(g, e[-1], layer.M)
        y = layer.run(dev(x), conv_state, state, list(zip(e, e[1:])), torch.tensor(e, dtype=torch.int32).cuda(), k > 0)
        for i in range(n):
            rows[i].append(x[e[i]:e[i + 1]])
            outs[i].append(cpu(y[e[i]:e[i + 1]]))
    for _ in range(tokens):
        x = randn(g, n, layer.M)
        y = layer.run(dev(x), conv_state, state)
        for i in range(n):
            rows[i].append(x[i:i + 1])
            outs[i].append(cpu(y[i:i + 1]))
    x = torch.cat([torch.cat(r) for r in rows])
    e = edges_of([sum(len(v) for v in r) for r in rows])
    c2, s2 = torch.zeros_like(conv_state), torch.zeros_like(state)
    whole = cpu(layer.run(dev(x), c2, s2, list(zip(e, e[1:])), torch.tensor(e, dtype=f32).int().cuda(), False))
    got = torch.cat([torch.cat(o) for o in outs])
    # Both runs are near the same function; the stages' own bounds are checked above.
    assert (got - whole).norm() <= 1e-4 * whole.norm()
    assert (state - s2).norm() <= 1e-4 * s2.norm()


@pytest.mark.parametrize("t", ["bf16", "f16"])
@pytest.mark.parametrize("n", [1, 9])
def test_layer_tokens_in_16_bits(t, n):
    layer, g, tt = Layer(ref.TYPES[t]), gen(6), ref.TYPES[t]
    conv_state, state = randn(g, n, 3, layer.D, t=tt).cuda(), randn(g, n, layer.D, layer.S).cuda()
    for _ in range(3):
        layer.run(randn(g, n, layer.M, t=tt).cuda(), conv_state, state)


# --------------------------------------------------- streams, graphs, spaces
def big_case(t=torch.bfloat16, L=1500, D=256):
    c = {k: dev(v) for k, v in scan_case(t, L, 1, D, 16, 1, 8).items()}
    return c


def run_big(c, state, **kw):
    return mg3m.selective_scan(c["u"], c["dt"], c["A"], c["B"], c["C"], c["D"], c["z"], c["dt_bias"], True, state, True,
                               **kw)


def test_results_are_the_same_from_run_to_run():
    c = big_case()
    first = None
    for _ in range(5):
        s = c["state"].clone()
        y = run_big(c, s)
        if first is not None:
            assert torch.equal(y, first[0]) and torch.equal(s, first[1])
        first = (y, s)
    x, q, s, z = (dev(v) for v in w4_case(torch.bfloat16, 13, 4096, 200, 64, 1, True))
    y = mg3m.matvec_w4(x, q, s, z)
    assert all(torch.equal(mg3m.matvec_w4(x, q, s, z), y) for _ in range(5))


def test_a_callers_workspace():
    c = big_case()
    want_s = c["state"].clone()
    want = run_big(c, want_s)
    need = mg3m.selective_scan_workspace_bytes(1500, 256, 1, 16, 1)
    assert need > 0
    ws = torch.full((need + 64,), 255, dtype=torch.uint8).cuda()       # NaN where read before written
    s = c["state"].clone()
    assert torch.equal(run_big(c, s, workspace=ws[:need]), want) and torch.equal(s, want_s)
    assert (ws[need:] == 255).all()
    with pytest.raises(mg3m.Mg3mError, match="WORKSPACE"):
        run_big(c, s, workspace=ws[:need - 1])


def test_streams_side_by_side():
    """Two streams, no waiting between the calls; each has its own workspace."""
    cases = [big_case(L=1500), big_case(L=2100, D=192)]
    wants = []
    for c in cases:
        s = c["state"].clone()
        wants.append((run_big(c, s), s))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    states = [[c["state"].clone() for _ in range(6)] for c in cases]
    torch.cuda.synchronize()
    got = []
    for i in range(6):
        for k in range(2):
            with torch.cuda.stream(streams[k]):
                got.append((k, run_big(cases[k], states[k][i]), states[k][i]))
    torch.cuda.synchronize()
    for k, y, s in got:
        assert torch.equal(y, wants[k][0]) and torch.equal(s, wants[k][1])
    # a stream given to the call, while another one is current
    s = cases[0]["state"].clone()
    torch.cuda.synchronize()
    y = run_big(cases[0], s, stream=streams[1], out=torch.empty_like(cases[0]["u"]))
    streams[1].synchronize()
    assert torch.equal(y, wants[0][0]) and torch.equal(s, wants[0][1])


def test_captured_and_replayed():
    """One token and one prompt of a layer's operators in two graphs, replayed
    with other work between; states advance with each replay."""
    g = gen(3)
    t, N, C, S = torch.bfloat16, 5, 192, 16
    x, w, b = (randn(g, *s, t=t).cuda() for s in ((N, C), (4, C), (C,)))
    c = {k: dev(v) for k, v in scan_case(t, N, N, C, S, 1, 4).items()}
    xq, q, sc, z = (dev(v) for v in w4_case(t, N, 192, 64, 64, 2, True))
    big = big_case()
    conv_state, state, big_state = randn(g, N, 3, C, t=t).cuda(), c["state"].clone(), big["state"].clone()

    def token(conv_state, state):
        return (mg3m.conv1d_causal_step(x, w, conv_state, b, True),
                mg3m.selective_scan_step(c["u"], c["dt"], c["A"], c["B"], c["C"], state, c["D"], c["z"], c["dt_bias"], True),
                mg3m.matvec_w4(xq, q, sc, z))

    def prompt(s):
        return (run_big(big, s), mg3m.conv1d_causal(big["u"], w[:, :1].expand(4, 256).contiguous(), None, True))

    eager = (conv_state.clone(), state.clone(), big_state.clone())
    token(conv_state.clone(), state.clone())
    prompt(big_state.clone())
    torch.cuda.synchronize()
    graphs, outs = [], []
    for f, a in ((token, (conv_state, state)), (prompt, (big_state,))):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(f(*a))
        graphs.append(graph)
    for _ in range(4):
        graphs[0].replay()
        graphs[1].replay()
        want = (*token(eager[0], eager[1]), *prompt(eager[2]))
        torch.cuda.synchronize()
        for a, e in zip((*outs[0], *outs[1], conv_state, state, big_state), (*want, *eager)):
            assert torch.equal(a, e)


# ----------------------------------------------------------- large tensors
def test_rows_past_32_bit_offsets():
    """64 columns at the end of rows 64 KB apart: element offsets past 2^31."""
    T, ld, C, t = 70000, 32768, 64, torch.bfloat16
    wide = torch.zeros(T, ld, dtype=t, device="cuda")
    x = randn(gen(1), T, C, t=t).cuda()
    wide[:, -C:] = x
    w = randn(gen(2), 4, C, t=t).cuda()
    y = mg3m.conv1d_causal(x, w, None, True)
    assert torch.equal(mg3m.conv1d_causal(wide[:, -C:], w, None, True, out=wide[:, :C]), y)
    assert torch.equal(wide[:, -C:], x)
    A = -torch.rand(C, 8, generator=gen(3)).cuda()
    B = randn(gen(4), T, 8, t=t).cuda()
    want = mg3m.selective_scan(x, x, A, B, B, z=x, softplus=True)
    got = mg3m.selective_scan(wide[:, -C:], wide[:, -C:], A, B, B, z=wide[:, -C:], softplus=True, out=wide[:, C:2 * C])
    assert torch.equal(got, want)


def test_states_past_32_bit_offsets():
    N, D, S = 8300, 16384, 16
    state = torch.zeros(N, D, S, device="cuda")
    assert state.numel() > 2 ** 31
    u = randn(gen(1), 4, D, t=torch.bfloat16).cuda()
    B = randn(gen(2), 4, S, t=torch.bfloat16).cuda()
    A = -torch.rand(D, S, generator=gen(3)).cuda()
    rows = lambda v: v[:1].expand(N, *v.shape[1:]).clone()  # noqa: E731
    ub, Bb = rows(u), rows(B)
    ub[-4:], Bb[-4:] = u, B
    y = mg3m.selective_scan_step(ub, ub, A, Bb, Bb, state, softplus=True)
    small = torch.zeros(4, D, S, device="cuda")
    assert torch.equal(mg3m.selective_scan_step(u, u, A, B, B, small, softplus=True), y[-4:])
    assert torch.equal(state[-4:], small) and torch.equal(state[0], state[5000])


@pytest.mark.parametrize("M", [1, 5])
def test_weights_past_32_bit_offsets(M):
    K, C = 140000, 32768
    q = torch.randint(0, 256, (K, C // 2), dtype=torch.uint8, device="cuda")
    assert q.numel() > 2 ** 31
    x = randn(gen(1), M, C, t=torch.bfloat16).cuda()
    s = (torch.rand(K, C // 128, device="cuda") * 0.01).bfloat16()
    y = mg3m.matvec_w4(x, q, s)
    # the same rows by themselves, from a row that is a tile's first either way
    assert torch.equal(mg3m.matvec_w4(x, q[-40000:].clone(), s[-40000:].clone()), y[:, -40000:])
    codes = torch.stack([q[-64:] & 15, q[-64:] >> 4], -1).flatten(1).double().cpu()
    want = x.double().cpu() @ ((codes - 8) * s[-64:].double().cpu().repeat_interleave(128, 1)).t()
    near(y[:, -64:], want, ref.stored(want, C * ref.H * 31 * (x.double().cpu().abs().sum(1, True) * 0.01), torch.bfloat16))


# ------------------------------------------------------------- bad row ranges
def test_ranges_outside_the_tensor_are_clamped():
    """begin and end outside 0..T are taken as the nearest of them, an end
    before its begin as an empty sequence (tests/seq_pieces.cpp has the rest)."""
    T, C = 300, 70
    c = scan_case(torch.float32, T, 3, C, 16, 1, 9)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32).cuda()  # noqa: E731
    begin, end = [-5, 100, 250], [90, 60, 2000]
    taken = [(0, 90), (100, 100), (250, 300)]
    want, after, tol, atol = scan_want(c, taken, True, True)
    sd, out = dev(c["state"]), torch.full((T, C), float("nan")).cuda()
    scan_run(c, sd, begin=i32(begin), end=i32(end), out=out)
    near(out, want, ref.stored(want, tol, torch.float32))
    near(sd, after, atol)
    x, w, s = randn(gen(1), T, C), randn(gen(2), 4, C), randn(gen(3), 3, 3, C)
    want, after, tol = ref.conv(x, w, None, s, taken, True, False)
    sd, out = dev(s), torch.full((T, C), float("nan")).cuda()
    mg3m.conv1d_causal(dev(x), dev(w), None, False, sd, True, begin=i32(begin), end=i32(end), out=out)
    near(out, want, ref.stored(want, tol, torch.float32))
    assert torch.equal(sd.cpu().double(), after)


@pytest.mark.parametrize("t", T3)
def test_no_rows_at_all(t):
    tt = ref.TYPES[t]
    x, st = torch.zeros(0, 24, dtype=tt).cuda(), torch.ones(2, 3, 24, dtype=tt).cuda()
    off = torch.zeros(3, dtype=torch.int32).cuda()
    assert mg3m.conv1d_causal(x, torch.ones(4, 24, dtype=tt).cuda(), state=st, load_state=True, offsets=off).shape == (0, 24)
    assert (st == 1).all()
    mg3m.conv1d_causal(x, torch.ones(4, 24, dtype=tt).cuda(), state=st, offsets=off)
    assert (st == 0).all()


def test_growing_states_that_start_at_the_end():
    """Decays above one, inputs in the last tokens only: a piece's factor
    passes fp32, the states stay small integers.  exp(4) per token, u = 0 but
    for the last token, whose state is delta B u exactly."""
    L, D, S = 4096, 64, 16
    u = torch.zeros(1, L, D).cuda()
    u[:, -1] = torch.arange(D).float().cuda() + 1
    one = torch.ones(1, L, D).cuda()
    B = torch.ones(1, L, S).cuda()
    state = torch.zeros(1, D, S).cuda()
    y = mg3m.selective_scan(u, one, torch.full((D, S), 4.0).cuda(), B, B, state=state)
    assert torch.equal(state[0], u[0, -1][:, None].expand(D, S))
    assert torch.equal(y[:, -1], u[:, -1] * S) and not y[:, :-1].any()


# ------------------------------------------------------------ the binding
@pytest.mark.parametrize("t", T3)
def test_quick_binding_and_general_one_agree(t):
    """A given stream takes the general path through the binding: the same
    results, bit for bit, for dense, strided and three-dimensional rows."""
    tt, N, L, D, S = ref.TYPES[t], 3, 40, 48, 16
    g, st, quick = gen(12), torch.cuda.current_stream(), mg3m.load_binding()
    wide = randn(g, N, L, 2 * D + 5, t=tt).cuda()
    x, z = wide[..., 3:3 + D], wide[..., 4 + D:4 + 2 * D]
    w, b = randn(g, 4, D, t=tt).cuda(), randn(g, D, t=tt).cuda()
    A, B = -torch.rand(D, S, generator=g).cuda(), randn(g, N, L, 2, S, t=tt).cuda()
    off = torch.tensor([0, 7, 7, N * L], dtype=torch.int32).cuda()
    q = torch.randint(0, 256, (20, D // 2 + 8), generator=g, dtype=torch.int32).to(torch.uint8).cuda()
    s = randn(g, 20, 2, t=tt).cuda()
    xq = randn(g, 5, 70, t=tt).cuda()[:, 2:66]
    for v in (x, x.contiguous(), x.contiguous().flatten(0, 1), x.flatten(0, 1)):
        flat = v.dim() == 2
        zz, BB, o = (z.flatten(0, 1), B.flatten(0, 1), off) if flat else (z, B, None)
        got = []
        for kw in ({}, {"stream": st}):
            cs, hs = torch.ones(N, 3, D, dtype=tt).cuda(), torch.ones(N, D, S).cuda()
            y = mg3m.conv1d_causal(v, w, b, True, cs, True, offsets=o, **kw)
            y2 = mg3m.selective_scan(v, y, A, BB, BB, A[:, 0].contiguous(), zz, None, True, hs, True, o, **kw)
            rows = v if flat else v[:, 0]
            cs2, hs2 = (u[:1].expand(len(rows), *u.shape[1:]).contiguous() for u in (cs, hs))
            y3 = mg3m.conv1d_causal_step(rows, w, cs2, b, False, **kw)
            y4 = mg3m.selective_scan_step(rows, y3, A, BB if flat else BB[:, 0], BB if flat else BB[:, 0], hs2, **kw)
            got.append((y, y2, cs, hs, y3, y4, cs2, hs2, mg3m.matvec_w4(xq, q, s, **kw)))
        for a, c in zip(*got):
            assert torch.equal(a, c)
    taken = quick.conv1d(False, x, w, b, True, None, False, None, None, None, None)
    assert taken is not None and torch.equal(taken, mg3m.conv1d_causal(x, w, b, True, stream=st))
    assert quick.w4(xq, q, s, None, None) is not None
    out = torch.empty_like(x.contiguous())
    assert mg3m.conv1d_causal(x, w, b, True, out=out) is out and torch.equal(out, taken)


def test_binding_refusals_on_the_gpu():
    x, w, st = torch.zeros(4, 8).cuda(), torch.zeros(4, 8).cuda(), torch.zeros(4, 3, 8).cuda()
    with pytest.raises(TypeError):
        mg3m.conv1d_causal_step(x, w.half(), st)
    with pytest.raises(ValueError, match="shape"):
        mg3m.conv1d_causal_step(x, w, st[:3])
    with pytest.raises(ValueError, match="contiguous"):
        mg3m.conv1d_causal(x.t(), torch.zeros(4, 4).cuda())
    with pytest.raises(ValueError):
        mg3m.conv1d_causal(x, w, offsets=torch.zeros(3, dtype=torch.int32).cuda(), begin=torch.zeros(2).int().cuda())
    with pytest.raises(mg3m.Mg3mError, match="ALIAS"):
        mg3m.conv1d_causal(x, w, out=x)
    with pytest.raises(mg3m.Mg3mError, match="SHAPE"):
        mg3m.conv1d_causal(x, torch.zeros(9, 8).cuda())
    with pytest.raises(mg3m.Mg3mError, match="SHAPE"):
        mg3m.conv1d_causal(x[:1].expand(4, 8), w)


def test_graphs_replayed_side_by_side():
    """Two captured prompts, each with its own workspace, replayed on two
    streams at once, with eager work between."""
    cases = [big_case(L=1500), big_case(L=2100, D=192)]
    wants, graphs, outs, states = [], [], [], []
    for c in cases:
        s = torch.zeros_like(c["state"])
        y = mg3m.selective_scan(c["u"], c["dt"], c["A"], c["B"], c["C"], c["D"], c["z"], c["dt_bias"], True, s)
        wants.append((y, s))
        states.append(torch.zeros_like(s))
    torch.cuda.synchronize()
    for c, s in zip(cases, states):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(mg3m.selective_scan(c["u"], c["dt"], c["A"], c["B"], c["C"], c["D"], c["z"], c["dt_bias"], True, s))
        graphs.append(graph)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(4):
        for y, s in zip(outs, states):
            y.zero_()
            s.zero_()
        torch.cuda.synchronize()
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
        again = run_big(cases[0], torch.zeros_like(wants[0][1]))
        torch.cuda.synchronize()
        for y, s, (want, after) in zip(outs, states, wants):
            assert torch.equal(y, want) and torch.equal(s, after)
        assert torch.equal(again, wants[0][0])


# --------------------------------------------------- small and growing values
@pytest.mark.parametrize("M", [1, 2, 5, 16])
def test_w4_subnormal_tokens(M):
    """fp16 tokens below the type's normal range count in full."""
    x = (ints_small(M, 128) * 2.0 ** -22).half()
    q = torch.randint(0, 256, (40, 64), generator=gen(2), dtype=torch.int32).to(torch.uint8)
    s = torch.full((40, 2), 1024.0).half()
    want, _ = ref.w4(x, q, s, None, 64)
    assert torch.equal(mg3m.matvec_w4(dev(x), dev(q), dev(s)).cpu(), want.half())


def ints_small(M, C):
    return torch.randint(-3, 4, (M, C), generator=gen(M)).float()


@pytest.mark.parametrize("t", T3)
@pytest.mark.parametrize("M,C,K,group,zero", [(3, 256, 64, 64, True), (4, 2080, 70, 32, False), (13, 4096, 70, 128, True),
                                              (7, 8192, 33, 32, False), (34, 4096, 50, 4096, True), (3, 1024, 5000, 64, True),
                                              (6, 2048, 2051, 64, False)])
def test_w4_few_rows_and_few_tokens(t, M, C, K, group, zero):
    """Both sides of the rule that picks the vector ALU or the matrix cores, groups of tokens that are not full."""
    tt = ref.TYPES[t]
    x, q, s, z = w4_case(tt, M, C, K, group, M + K, zero)
    want, tol = ref.w4(x, q, s, z, group)
    near(mg3m.matvec_w4(dev(x), dev(q), dev(s), dev(z)), want, ref.stored(want, tol, tt))
    x, q, s, z = w4_case(tt, M, C, K, group, M + K, zero, integer=True)
    assert torch.equal(mg3m.matvec_w4(dev(x), dev(q), dev(s), dev(z)).cpu(), ref.w4(x, q, s, z, group)[0].to(tt))


@pytest.mark.parametrize("t", ["bf16", "f16"])
@pytest.mark.parametrize("group", [32, 64, 96, 512])
@pytest.mark.parametrize("M,K", [(5, 8200), (16, 12500), (13, 17001), (9, 25000), (40, 3001)])
def test_w4_every_tile(t, group, M, K):
    """Work-groups of two, three, four and six tiles of rows, one to a compute unit, and of four, several."""
    tt, C = ref.TYPES[t], 1536
    x, q, s, z = w4_case(tt, M, C, K, group, K, True, integer=True)
    assert torch.equal(mg3m.matvec_w4(dev(x), dev(q), dev(s), dev(z)).cpu(), ref.w4(x, q, s, z, group)[0].to(tt))
    x, q, s, z = w4_case(tt, M, C, K, group, K, False)
    want, tol = ref.w4(x, q, s, z, group)
    near(mg3m.matvec_w4(dev(x), dev(q), dev(s), dev(z)), want, ref.stored(want, tol, tt))


@pytest.mark.parametrize("t", T3)
@pytest.mark.parametrize("L,D", [(70, 64), (700, 130)])
def test_padding_may_hold_anything(t, L, D):
    """NaN and infinities in the rows of a padded batch that belong to no
    sequence: results and states as without them, those rows left alone."""
    tt, N, S = ref.TYPES[t], 3, 16
    c = {k: dev(v) for k, v in scan_case(tt, N * L, N, D, S, 1, L).items()}
    w = randn(gen(1), 4, D, t=tt).cuda()
    begin, length = torch.arange(N) * L, torch.tensor([L - 9, 0, 17])
    pad = torch.ones(N * L, dtype=torch.bool)
    for b, n in zip(begin.tolist(), length.tolist()):
        pad[b:b + n] = False
    be = [v.int().cuda() for v in (begin, begin + length)]
    got = []
    for bad in (0.0, float("nan"), float("inf")):
        v = {k: c[k].clone() for k in ("u", "dt", "B", "C", "z")}
        for x in v.values():
            x[pad.cuda()] = bad
        hs, cs, out, out2 = c["state"].clone(), torch.ones(N, 3, D, dtype=tt).cuda(), *(torch.full_like(v["u"], 5.0) for _ in "12")
        mg3m.selective_scan(v["u"], v["dt"], c["A"], v["B"], v["C"], c["D"], v["z"], c["dt_bias"], True, hs, True,
                            begin=be[0], end=be[1], out=out)
        mg3m.conv1d_causal(v["u"], w, None, True, cs, True, begin=be[0], end=be[1], out=out2)
        assert (out[pad.cuda()] == 5).all() and (out2[pad.cuda()] == 5).all()
        got.append((out, out2, hs, cs))
    for g in got[1:]:
        assert all(torch.equal(a, b) for a, b in zip(got[0], g))
