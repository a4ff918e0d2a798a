"""Sizes of the sequence operators at the ends of their integers, without a
GPU: what the header accepts reaches the launch, which then finds no device."""
import pytest
import torch

from paper_2307_04941_amd import mg3m
from test_seq_host import CONV, HIP, TOO_LARGE, W4, at, call


@pytest.mark.skipif(torch.cuda.is_available(), reason="addresses are made up")
@pytest.mark.parametrize("fn,packer,base,change,rc", [
    # 2^31 threads and more, below 2^32
    ("conv1d_causal_step", "_CONV1D", CONV, dict(N=65536, C=32769, ldx=32769, ldy=32769, dtype=0), HIP),
    ("conv1d_causal_fwd", "_CONV1D", CONV, dict(T=1, N=1 << 20, C=2049, ldx=2049, ldy=2049, begin=at(20), end=at(21)), HIP),
    ("matvec_w4_fwd", "_W4", W4, dict(M=1, K=1 << 27, C=1056, group=32, ldx=1056, ldy=1 << 27), HIP),
    # 2^32
    ("conv1d_causal_step", "_CONV1D", CONV, dict(N=65536, C=65537, ldx=65537, ldy=65537, dtype=0), TOO_LARGE),
    ("conv1d_causal_fwd", "_CONV1D", CONV, dict(T=1, N=1 << 20, C=4097, ldx=4097, ldy=4097, begin=at(20), end=at(21)), TOO_LARGE),
    ("matvec_w4_fwd", "_W4", W4, dict(M=1, K=1 << 28, C=1056, group=32, ldx=1056, ldy=1 << 28), TOO_LARGE)])
def test_launches_of_up_to_2_to_the_32_threads(fn, packer, base, change, rc):
    far = {k: at(100 * (i + 1)) for i, k in enumerate(base) if base[k] >= at(0) and k not in change}
    assert call(fn, getattr(mg3m, packer), base, **far, **change) == rc


@pytest.mark.parametrize("at_", range(5))
@pytest.mark.parametrize("size", [(1 << 32) + 64, 1 << 31, -(1 << 32) + 64])
def test_workspace_of_sizes_past_an_int(at_, size):
    """Not the workspace of the size's low 32 bits."""
    sizes = [64, 64, 64, 64, 64]
    assert mg3m.selective_scan_workspace_bytes(*sizes) > 0
    sizes[at_] = size
    with pytest.raises(ValueError, match="integer"):
        mg3m.selective_scan_workspace_bytes(*sizes)
