"""The gated linear recurrence where its inputs cancel or are small: a bias is
added to p before anything is made of the sum, and what is small is good
relative to itself, forward and back."""

import numpy as np
import pytest
import torch

from oracle import gated
from paper_1905_00689_amd import binding as B

from .gpu_helpers import say

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
HALF = {F32: 2.0 ** -24, BF16: 2.0 ** -8}


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


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("ragged", [False, True], ids=["", "ragged"])
@pytest.mark.parametrize("T,Bn,H", [(1, 3, 64), (12, 2, 33), (100, 2, 64), (700, 2, 65)])
def test_small_candidates_and_states_are_good_relative_to_themselves(T, Bn, H, ragged, dtype):
    """Candidates g and states c of 1e-7 to 1, a magnitude to a unit: h, c and
    the gradients against float64 within bounds relative to what they are made of."""
    say("small", T, Bn, H, ragged, dtype)
    r = np.random.default_rng([190500689, 77, T, H])
    size = 10.0 ** (-7 + 7 * np.arange(H) / H)
    p = r.normal(size=(T, Bn, 4, H))
    p[:, :, 0] *= 2
    p[:, :, 1] += 1
    p[:, :, 2] *= size
    bias = r.normal(size=(4, H))
    bias[2] *= size
    t = lambda a, d=F32: torch.from_numpy(a).to(d).cuda()  # noqa: E731
    p, bias = t(p.reshape(T, Bn, 4 * H), dtype), t(bias.reshape(4 * H))
    c0, dh, dc = t(r.normal(size=(Bn, H)) * size), t(r.normal(size=(T, Bn, H)), dtype), t(r.normal(size=(Bn, H)))
    lengths = torch.tensor([T, 2 * T // 3, 0][:Bn], dtype=torch.int32, device="cuda") if ragged else None
    got = passes(p, dh, dc, c0, bias, lengths)
    host = lambda a: None if a is None else a.double().cpu().numpy()  # noqa: E731
    n = None if lengths is None else lengths.cpu().numpy()
    h, c, _, _ = gated.linear_lstm(host(p), host(bias), n, host(c0))
    g, _ = gated.linear_lstm_grad(host(p), host(dh), host(dc), host(bias), n, host(c0))
    bound = gated.linear_lstm_small(host(p), host(dh), host(dc), host(bias), n, host(c0))
    for name, want, b, half in (("h", h, bound["h"], HALF[dtype]), ("c", c[-1], bound["c"][-1], HALF[F32]),
                                ("save", c[:-1][::8], bound["c"][:-1][::8], HALF[F32]),
                                ("dp", g["dp"], bound["dp"], HALF[dtype]), ("dc0", g["dc0"], bound["dc0"], HALF[F32])):
        worst = np.max(np.abs(host(got[name]) - want) / (b * (1 + half) + half * np.abs(want) + 1e-30))
        say(name, "worst share of the tolerance %.2f" % worst)
        assert np.isfinite(host(got[name])).all() and worst <= 1.0, (name, worst)
