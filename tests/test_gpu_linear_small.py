"""The gated linear recurrence where its inputs cancel or are small: a bias is
added to p before anything is made of the sum, and what is small is good
relative to itself, forward and back."""

import pytest
import torch

from paper_1905_00689_amd import binding as B

from .gpu_helpers import say

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def passes(p, dh, dc, c0, bias, lengths=None):
    """Everything that a run and its backward pass write."""
    T, Bn, H = dh.shape
    h, c, save = torch.empty_like(dh), torch.empty_like(c0), torch.empty(-(-T // 8), Bn, H, device="cuda")
    dp, dc0, db = torch.empty_like(p), torch.empty_like(c0), torch.empty(4 * H, device="cuda")
    B.approx_lstm_linear_run(p, h, bias=bias, lengths=lengths, c0=c0, c_out=c, c_save=save)
    B.approx_lstm_linear_backward(p, dh, save, dp, bias=bias, lengths=lengths, dc_out=dc, dc0=dc0, dbias=db)
    return dict(h=h, c=c, save=save, dp=dp, dc0=dc0, dbias=db)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("T,Bn,H", [(1, 3, 64), (12, 2, 33), (100, 2, 64), (700, 2, 65)])
def test_a_bias_that_cancels_leaves_nothing_behind(T, Bn, H, dtype):
    """p = v - b with a bias of b, where both differences are exact: the bits of
    p = v without one."""
    say("bias", T, Bn, H, dtype)
    g = torch.Generator().manual_seed(T + H)
    # steps of 1/2 near 64 are what bf16 holds; fp32 holds steps of 2^-14 near 1000
    b, step = (64.0, 0.5) if dtype is BF16 else (1000.0, 2.0 ** -14)
    v = torch.randint(-int(4 / step), int(4 / step) + 1, (T, Bn, 4 * H), generator=g).float() * step
    bias = torch.where(torch.arange(4 * H) % 2 == 0, b, -b)
    dh, dc, c0 = (torch.randn(s, generator=g).cuda() for s in ((T, Bn, H), (Bn, H), (Bn, H)))
    p = (v - bias).to(dtype)
    assert torch.equal(p.double() + bias.double(), v.double())
    got = passes(p.cuda(), dh.to(dtype), dc, c0, bias.cuda())
    want = passes(v.to(dtype).cuda(), dh.to(dtype), dc, c0, None)
    for name in want:
        assert torch.equal(got[name], want[name]), name
