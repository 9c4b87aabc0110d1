"""The 4-bit gate product against the float64 oracle, elementwise within its
bound on fp32 errors (and, for bf16 outputs, half a step of bf16)."""

import numpy as np
import pytest
import torch

from oracle import gated
from paper_1905_00689_amd import binding as B

from .gpu_helpers import say

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
HALF = {F32: 2.0 ** -24, BF16: 2.0 ** -8}


def levels(R, D, G, seed=0):
    r = np.random.default_rng([190500689, seed, R, D, G])
    n = -(-D // G)
    q, z = r.integers(0, 16, (R, D)).astype(np.uint8), r.integers(0, 16, (R, n)).astype(np.uint8)
    return q, (r.random((R, n)) + 0.1).astype(np.float32), z


def load(q, s, z, G):
    dev = lambda a: None if a is None else torch.from_numpy(a).cuda()  # noqa: E731
    return B.approx_lstm_q4_load(dev(gated.q4_pack(q)), dev(s), dev(z), q.shape[1], G)


def place(a, dtype, shift=0):
    t = torch.zeros(a.size + shift, dtype=dtype, device="cuda")
    t[shift:] = torch.from_numpy(a.reshape(-1)).to(dtype).cuda()
    return t[shift:].view(a.shape)


def check(y, q, s, z, G, x, bias):
    want, bound = gated.q4_product(q, s, z, G, x.double().cpu().numpy(), None if bias is None else bias.cpu().numpy())
    got, half = y.double().cpu().numpy(), HALF[y.dtype]
    worst = np.max(np.abs(got - want) / (bound * (1 + half) + half * np.abs(want) + 1e-30))
    assert np.isfinite(got).all() and worst <= 1.0, worst
    say("worst share of the tolerance %.3f" % worst)


SHAPES = [(1, 1, 1, 32), (1, 128, 64, 128), (1, 100, 77, 32), (2, 16, 128, 64), (3, 33, 129, 128), (5, 256, 2048, 128),
          (16, 48, 260, 32), (17, 64, 96, 64), (31, 129, 500, 128), (48, 300, 257, 64), (64, 20, 1000, 32),
          (65, 512, 64, 32), (100, 256, 1030, 32), (129, 130, 127, 64), (300, 272, 520, 128), (700, 96, 40, 32),
          (1100, 4000, 200, 32), (2050, 2100, 300, 128), (4200, 1000, 129, 64), (70, 33000, 64, 32),
          (1, 8200, 200, 64), (2, 8200, 200, 64), (1, 16400, 130, 32), (5, 16400, 130, 32), (40, 8200, 300, 128),
          (20, 8200, 300, 128)]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("N,R,D,G", SHAPES)
def test_product(N, R, D, G, dtype):
    say("q4", N, R, D, G, dtype)
    q, s, z = levels(R, D, G)
    r = np.random.default_rng(N)
    x = place(r.normal(size=(N, D)), dtype)
    bias = torch.from_numpy(r.normal(size=R).astype(np.float32)).cuda()
    m, y = load(q, s, z, G), torch.full((N, R), float("nan"), dtype=dtype, device="cuda")
    B.approx_lstm_q4_run(m, x, y, bias=bias)
    check(y, q, s, z, G, x, bias)
    # without a bias, on rows that start at any element: the same bits where nothing else differs
    y2 = place(np.zeros((N, R)), dtype, 1)
    B.approx_lstm_q4_run(m, place(x.double().cpu().numpy(), dtype, 1), y2)
    check(y2, q, s, z, G, x, None)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_every_row_is_itself(dtype):
    """A row of y depends on its row of x alone, to the bit, wherever it stands;
    a row with an infinity has nothing finite, and no other is touched."""
    q, s, z = levels(70, 300, 64)
    m = load(q, s, z, 64)
    x = place(np.random.default_rng(3).normal(size=(16, 300)), dtype)
    y = torch.empty(16, 70, dtype=dtype, device="cuda")
    B.approx_lstm_q4_run(m, x, y)
    order = torch.tensor([3, 15, 0, 7, 1, 2, 4, 5, 6, 8, 14, 13, 12, 11, 10, 9], device="cuda")
    moved = torch.empty_like(y)
    B.approx_lstm_q4_run(m, x[order].contiguous(), moved)
    assert torch.equal(moved, y[order])
    for v in (float("inf"), float("-inf"), float("nan")):
        bad = x.clone()
        bad[5, 299] = v
        z2 = torch.empty_like(y)
        B.approx_lstm_q4_run(m, bad, z2)
        assert not torch.isfinite(z2[5]).any()
        keep = [n for n in range(16) if n != 5]
        assert torch.equal(z2[keep], y[keep])


@pytest.mark.parametrize("R,D,G", [(4, 64, 32), (37, 77, 32), (16, 300, 128), (130, 129, 64)])
def test_prepare_rounds_as_the_oracle_and_get_gives_it_back(R, D, G):
    w = np.random.default_rng(R).normal(size=(R, D)).astype(np.float32)
    w[0] = 0.0
    q, s, z = gated.q4_round(w, G)
    got = B.approx_lstm_q4_get(B.approx_lstm_q4_prepare(w, G))
    assert np.array_equal(got["q"], gated.q4_pack(q)) and np.array_equal(got["scale"], s)
    assert np.array_equal(got["zero"], z)
    q, s, z = levels(R, D, G)
    got = B.approx_lstm_q4_get(load(q, s, z, G))
    assert np.array_equal(got["q"], gated.q4_pack(q)) and np.array_equal(got["scale"], s)
    assert np.array_equal(got["zero"], z)


def test_no_zero_levels_means_eight():
    q, s, z = levels(20, 100, 32)
    m = load(q, s, None, 32)
    x = place(np.random.default_rng(4).normal(size=(3, 100)), F32)
    y = torch.empty(3, 20, device="cuda")
    B.approx_lstm_q4_run(m, x, y)
    check(y, q, s, np.full_like(z, 8), 32, x, None)
    assert (B.approx_lstm_q4_get(m)["zero"] == 8).all()


def test_exact_where_every_sum_is():
    """Whole numbers within fp32's range come out exactly, in both types."""
    r = np.random.default_rng(6)
    q, s, z = levels(40, 384, 128)
    s[:] = 0.5
    xi = r.integers(-8, 9, (9, 384)).astype(np.float64)
    want, _ = gated.q4_product(q, s, z, 128, xi)
    m, y = load(q, s, z, 128), torch.empty(9, 40, device="cuda")
    B.approx_lstm_q4_run(m, place(xi, F32), y)
    assert np.array_equal(y.double().cpu().numpy(), want)
    yb = torch.empty(9, 40, dtype=BF16, device="cuda")
    B.approx_lstm_q4_run(m, place(xi, BF16), yb)
    assert torch.equal(yb, y.to(BF16))


@pytest.mark.parametrize("N", [1, 20, 300])
def test_captured_and_replayed(N):
    q, s, z = levels(96, 260, 64)
    m = load(q, s, z, 64)
    x = place(np.random.default_rng(7).normal(size=(N, 260)), BF16)
    y, want = (torch.empty(N, 96, dtype=BF16, device="cuda") for _ in range(2))
    B.approx_lstm_q4_run(m, x, want)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.approx_lstm_q4_run(m, x, y)
    for _ in range(3):
        y.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)


def test_refusals_on_the_device():
    q, s, z = levels(8, 64, 32)
    m = load(q, s, z, 32)
    z[3, 1] = 16
    with pytest.raises(B.ApproxLstmError):
        load(q, s, z, 32)
    x, y = torch.zeros(2, 64, device="cuda"), torch.full((2, 8), float("nan"), device="cuda")
    for a in ((x[:, :63], y), (x, y[:1]), (x.t().contiguous().t(), y), (x, y.bfloat16()), (x.cpu(), y), (x.double(), y)):
        with pytest.raises((TypeError, ValueError)):
            B.approx_lstm_q4_run(m, *a)
    with pytest.raises(ValueError):
        B.approx_lstm_q4_run(m, x, y, bias=torch.zeros(7, device="cuda"))
    assert torch.isnan(y).all()
    B.approx_lstm_q4_run(m, x[:0], y[:0])


def test_more_rows_than_a_launch_takes():
    """1.1 million rows of x, and an output of more than 2^31 elements: the last
    rows are those of a small call."""
    for N, D, R, dtype in ((1100000, 40, 20, F32), (40000, 33, 60000, BF16)):
        q, s, z = levels(R, D, 32)
        m = load(q, s, z, 32)
        x = torch.randn(N, D, device="cuda").to(dtype)
        y = torch.empty(N, R, dtype=dtype, device="cuda")
        B.approx_lstm_q4_run(m, x, y)
        for rows in (slice(0, 3), slice(N // 2, N // 2 + 3), slice(N - 3, N)):
            check(y[rows].contiguous(), q, s, z, 32, x[rows], None)
        del x, y


def test_layer_of_product_and_recurrence():
    """The two as they are used: gate pre-activations of every frame by the 4-bit
    product, then the recurrence (its bias there), forward, and back to the
    gradients of the pre-activations."""
    T, Bn, D, H, G = 30, 3, 100, 24, 32
    r = np.random.default_rng(8)
    w, b = r.normal(size=(4 * H, D)).astype(np.float32) / 10, r.normal(size=4 * H).astype(np.float32)
    m = B.approx_lstm_q4_prepare(w, G)
    x = place(np.maximum(r.normal(size=(T * Bn, D)), 0), F32)
    p, h = torch.empty(T, Bn, 4 * H, device="cuda"), torch.empty(T, Bn, H, device="cuda")
    bias = torch.from_numpy(b).cuda()
    B.approx_lstm_q4_run(m, x, p.view(T * Bn, 4 * H))
    save = torch.empty(-(-T // 8), Bn, H, device="cuda")
    B.approx_lstm_linear_run(p, h, bias=bias, c_save=save)
    q, s, z = gated.q4_round(w, G)
    want, bound = gated.q4_product(q, s, z, G, x.double().cpu().numpy())
    ho, _, he, _ = gated.linear_lstm(want.reshape(T, Bn, 4 * H), b.astype(np.float64))
    # an error e of every pre-activation moves c by at most e (|c|/4 + 1 + 1/4) a step; |c| <= T
    e = bound.max() * T * (T / 4 + 1.25)
    assert (np.abs(h.double().cpu().numpy() - ho) <= he + e).all()
    dh = place(r.normal(size=(T, Bn, H)), F32)
    dp, db = torch.empty_like(p), torch.empty(4 * H, device="cuda")
    B.approx_lstm_linear_backward(p, dh, save, dp, bias=bias, dbias=db)
    g, ge = gated.linear_lstm_grad(p.double().cpu().numpy(), dh.double().cpu().numpy(), None, b.astype(np.float64))
    assert (np.abs(dp.double().cpu().numpy() - g["dp"]) <= ge["dp"] + 2.0 ** -24 * np.abs(g["dp"])).all()
    assert (np.abs(db.double().cpu().numpy() - g["dbias"]) <= ge["dbias"] + 2.0 ** -24 * np.abs(g["dbias"])).all()
