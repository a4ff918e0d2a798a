"""Tensors that the convolution, the pooling and the network executor make for
a call on a given stream belong to that stream."""
import pytest
import torch

from paper_2307_04941_amd import mg3m
from test_seq_edges_gpu import on_a_stream

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("raw", [False, True])
def test_results_and_workspaces_come_from_the_given_stream(raw, monkeypatch):
    g = torch.Generator().manual_seed(2)
    x, w = torch.randn(12, 12, 16, 8, generator=g).cuda(), torch.randn(3, 3, 16, 32, generator=g).cuda()
    net = mg3m.Net([dict(op="conv", K=32, R=3, pad=1, relu=1, w=w), dict(op="maxpool", R=2, stride=2)], (8, 16, 12, 12))
    side = torch.cuda.Stream()
    given = side.cuda_stream if raw else side
    # an override whose workspace the call makes itself
    split = next(p for p in ("split=2", "split=4") if mg3m.conv2d_fwd_f32_hw_workspace_bytes(
        8, 16, 12, 12, 32, 3, 3, 1, 1, 1, 1, "HWCN", p) > 0)
    for f, shape in ((lambda st: mg3m.conv2d_fwd(x, w, 1, 1, stream=st), (12, 12, 32, 8)),
                     (lambda st: mg3m.conv2d_fwd(x, w, 1, 1, acc64=True, stream=st), (12, 12, 32, 8)),
                     (lambda st: mg3m.maxpool2d(x, 2, stream=st), (6, 6, 16, 8)),
                     (lambda st: net.forward(x, stream=st), (6, 6, 32, 8))):
        want = f(None)
        assert torch.equal(on_a_stream(f, shape, torch.float32, given), want)
    want = mg3m.conv2d_fwd(x, w, 1, 1, plan=split)
    torch.cuda.synchronize()
    taken, empty = [], torch.empty

    def recorded(*a, **k):
        taken.append(torch.cuda.current_stream().cuda_stream)
        return empty(*a, **k)
    monkeypatch.setattr(torch, "empty", recorded)
    y = mg3m.conv2d_fwd(x, w, 1, 1, plan=split, stream=given)
    monkeypatch.undo()
    torch.cuda.synchronize()
    assert taken == [side.cuda_stream] * 2 and torch.equal(y, want)
