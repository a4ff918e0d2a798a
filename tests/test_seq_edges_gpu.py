"""The sequence operators (include/mg3m_seq.h) on the GPU where a rule of
theirs changes sides: states that grow across the pieces of a cut
prompt, weights at their zero point, results on a given
stream, launches of many threads."""
import pytest
import torch

import scan_ref
import seq_ref as ref
from paper_2307_04941_amd import mg3m
from test_seq_gpu import dev, near

pytestmark = pytest.mark.gpu


# ------------------------------------------------- states that grow or fade
# A rate, and the state's first value: a piece's factor passes fp32 at its
# upper end or its lower one, no state does.
@pytest.mark.parametrize("L,A,h0", [(33, 4.0, 1e-30), (40, 4.0, -1e-34), (63, 2.8, 2.0 ** -140), (33, 5.4, 2.0 ** -140),
                                    (70, 2.4, 1e-37), (40, -3.2, 1e38)])
@pytest.mark.parametrize("signed", [False, True])
def test_states_grow_across_pieces_as_the_formula_says(L, A, h0, signed):
    """One sequence of few channels is cut at 32 tokens; without inputs its
    state is h0 exp(A delta t), finite at its end.  signed: rates below zero
    with negative step sizes, the same."""
    D, S = 64, 16
    c = dict(u=torch.zeros(L, D), dt=torch.full((L, D), -1.0 if signed else 1.0),
             A=torch.full((D, S), -A if signed else A), B=torch.ones(L, 1, S), C=torch.ones(L, 1, S), D=None, z=None,
             dt_bias=None, state=torch.full((1, D, S), h0))
    want, after, tol, atol = scan_ref.scan(**c, softplus=False, ranges=[(0, L)], load=True, W=32)
    assert want.abs().max() < 2.0 ** 127           # the states are of one sign, so no part of y is larger
    sd = dev(c["state"])
    y = mg3m.selective_scan(dev(c["u"]), dev(c["dt"]), dev(c["A"]), dev(c["B"]), dev(c["C"]), state=sd, load_state=True)
    near(sd, after, atol, "state")
    near(y, want, ref.stored(want, tol, torch.float32), "y")
    zero = torch.zeros_like(sd)                    # a state of nothing stays nothing
    y = mg3m.selective_scan(dev(c["u"]), dev(c["dt"]), dev(c["A"]), dev(c["B"]), dev(c["C"]), state=zero, load_state=True)
    assert not y.any() and not zero.any()


# ------------------------------------------------- fp32 tokens, 4-bit weights
@pytest.mark.parametrize("M,C,K", [(1, 4096, 300), (2, 4096, 300), (4, 2048, 40), (16, 4096, 60), (7, 1024, 5000)])
@pytest.mark.parametrize("group", [32, 128])
def test_w4_weights_at_their_zero_point_add_nothing(M, C, K, group):
    """fp32 tokens meet q - zero itself: rows that hold their zero points are
    zero to the last bit, and with one weight beside them y is its product,
    which rounds three times."""
    g = torch.Generator().manual_seed(M + C)
    x = torch.randn(M, C, generator=g) * 8
    zero = torch.randint(0, 16, (K, C // group), generator=g).to(torch.uint8)
    codes = zero.repeat_interleave(group, 1)
    scale = 0.01 * torch.exp(torch.randn(K, C // group, generator=g))
    at = torch.arange(K) % C
    for bump in (0, 1):
        codes[torch.arange(K), at] ^= bump              # by one, to either side
        q = codes[:, 0::2] | (codes[:, 1::2] << 4)
        y = mg3m.matvec_w4(dev(x), dev(q), dev(scale), dev(zero)).cpu()
        if not bump:
            assert not y.any()
            continue
        rows = torch.arange(K)
        off = codes[rows, at].double() - zero[rows, at // group].double()
        want = x.double()[:, at] * (off * scale[rows, at // group].double())
        near(y, want, want.abs() * 3 * ref.H)


# ------------------------------------------------------ results on a stream
def on_a_stream(call, shape, t, stream):
    """The result of a call on a stream that is not the current one, which is
    not to come from a block of the current one's."""
    free = torch.empty(shape, dtype=t, device="cuda")
    at = free.data_ptr()
    del free
    torch.cuda.synchronize()
    y = call(stream)
    torch.cuda.synchronize()
    again = torch.empty(shape, dtype=t, device="cuda")
    assert again.data_ptr() == at != y.data_ptr()
    return y


@pytest.mark.parametrize("raw", [False, True])
@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_results_come_from_the_given_stream(t, raw):
    tt, N, C, S = ref.TYPES[t], 40, 192, 16
    g = torch.Generator().manual_seed(1)
    rn = lambda *s, t=tt: torch.randn(*s, generator=g).to(t).cuda()  # noqa: E731
    x, w, B, A = rn(N, C), rn(4, C), rn(N, S), -rn(C, S, t=torch.float32).abs()
    q, scale = torch.randint(0, 256, (C, C // 2), generator=g).to(torch.uint8).cuda(), rn(C, C // 64)
    conv_state, state = rn(N, 3, C), rn(N, C, S, t=torch.float32)
    copies = [(conv_state.clone(), state.clone()) for _ in range(2)]
    side = torch.cuda.Stream()
    given = side.cuda_stream if raw else side
    for f in (lambda st, s: mg3m.conv1d_causal(x, w, silu=True, stream=st),
              lambda st, s: mg3m.conv1d_causal_step(x, w, s[0], stream=st),
              lambda st, s: mg3m.selective_scan(x, x, A, B, B, z=x, softplus=True, stream=st),
              lambda st, s: mg3m.selective_scan_step(x, x, A, B, B, s[1], softplus=True, stream=st),
              lambda st, s: mg3m.matvec_w4(x, q, scale, stream=st)):
        want = f(None, copies[0])
        assert torch.equal(on_a_stream(lambda st: f(st, copies[1]), (N, C), tt, given), want)
    # raw handles of the current stream, and of the default one while another is current
    assert torch.equal(mg3m.matvec_w4(x, q, scale, stream=torch.cuda.current_stream().cuda_stream), want)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        y = mg3m.matvec_w4(x, q, scale, stream=0)
    torch.cuda.synchronize()
    assert torch.equal(y, want)


# ------------------------------------------- launches of 2^31 threads and more
@pytest.fixture
def large():
    yield
    torch.cuda.empty_cache()


def test_conv_step_of_2_to_the_31_threads(large):
    N, C = 65536, 32769                              # odd: a thread per channel
    x = torch.empty(N, C, device="cuda")
    x.copy_((torch.arange(N, device="cuda") % 61)[:, None] + torch.arange(C, device="cuda") % 7)
    w, b = (torch.arange(C, device="cuda") % 5).float()[None], (torch.arange(C, device="cuda") % 3).float()
    y = mg3m.conv1d_causal_step(x, w, None, b)
    for i in range(0, N, 4096):
        assert torch.equal(y[i:i + 4096], x[i:i + 4096] * w + b)


def test_conv_of_2_to_the_31_threads(large):
    """A million sequences, one row among them: the others' states stay."""
    N, C, n, t = 1 << 20, 2049, 1000003, torch.bfloat16
    state = torch.empty(N, 1, C, dtype=t, device="cuda")
    state.copy_((torch.arange(N, device="cuda") % 61)[:, None, None] + torch.arange(C, device="cuda") % 7)
    before = state.clone()
    x, w = torch.full((1, C), 3, dtype=t, device="cuda"), torch.full((2, C), 2, dtype=t, device="cuda")
    offsets = (torch.arange(N + 1, device="cuda") > n).int()
    y = mg3m.conv1d_causal(x, w, state=state, load_state=True, offsets=offsets)
    assert torch.equal(y[0], 2 * before[n, 0] + 6)
    before[n] = 3
    assert torch.equal(state, before)


def test_w4_of_2_to_the_31_threads(large):
    K, C, t = (1 << 27) + 64, 1056, torch.bfloat16
    if torch.cuda.mem_get_info()[0] < 120 << 30:
        pytest.skip("needs 80 GB")
    x = torch.randint(-3, 4, (1, C), generator=torch.Generator().manual_seed(1)).to(t).cuda()
    q = torch.full((K, C // 2), 0x98, dtype=torch.uint8, device="cuda")      # 0, 1
    q[-96:] = 0x7b                                                           # 3, -1
    scale = torch.ones(K, C // 32, dtype=t, device="cuda")
    y = mg3m.matvec_w4(x, q, scale)[0].float()
    even, odd = x[0, 0::2].float().sum(), x[0, 1::2].float().sum()
    assert (y[:-96] == odd.to(t).float()).all() and (y[-96:] == (3 * even - odd).to(t).float()).all()
