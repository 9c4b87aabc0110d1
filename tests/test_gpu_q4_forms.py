"""Every kernel instance of the 4-bit products at group lengths of 32, 64 and
128 columns, over one block of columns and over several."""

import numpy as np
import pytest
import torch

from paper_1905_00689_amd import binding as B

from .gpu_helpers import say
from .q4_cases import ALL, BF16, F32, FORMS, IDS, levels, one_column, one_column_share, rms_share
from .test_gpu_q4 import check, load, place

pytestmark = pytest.mark.gpu


def product(m, x, dtype, bias=None):
    y = torch.full((x.shape[0], m.rows), float("nan"), dtype=dtype, device="cuda")
    B.approx_lstm_q4_run(m, x, y, bias=bias)
    return y


@pytest.mark.parametrize("G", [32, 64, 128])
@pytest.mark.parametrize("form,dtype", ALL, ids=IDS)
def test_every_kernel(form, dtype, G):
    N, R, widths = FORMS[form]
    if torch.cuda.get_device_properties(0).multi_processor_count != 256:
        pytest.skip("the cases are chosen for 256 compute units")
    for D in widths:
        say(form, dtype, G, D)
        assert B.approx_lstm_q4_plan(R, D, G, N, dtype) == form
        q, s, z = levels(R, D, G)
        m, r = load(q, s, z, G), np.random.default_rng([1, N, D])
        x, bias = place(r.normal(size=(N, D)), dtype), torch.from_numpy(r.normal(size=R).astype(np.float32)).cuda()
        y = product(m, x, dtype, bias)
        check(y, q, s, z, G, x, bias)
        assert torch.equal(product(m, x, dtype, bias), y)
        if dtype is F32:
            worst = rms_share(product(m, x, dtype).double().cpu().numpy(), q, s, z, G, x.double().cpu().numpy())
            say("root mean square %.2f of what roundings may make" % worst)
            assert worst <= 1.0
        # one column a row: 24 bits of x, and in bf16 the nearest bf16 number
        if dtype is BF16:
            s = np.exp2(np.floor(np.log2(s))).astype(np.float32)
            m = load(q, s, z, G)
        x, at, v = one_column(N, R, D, G)
        x = place(x, dtype)
        got = product(m, x, dtype)
        if dtype is F32:
            worst = one_column_share(got.double().cpu().numpy(), q, s, z, G, at, v)
            say("one column: %.2f of the tolerance" % worst)
            assert worst <= 1.0
        else:
            # (q - z) x has 4 + 8 bits, s is a power of two: fp32 holds the sum
            d = torch.from_numpy((q[:, at].astype(np.int64) - z[:, at // G]).T * s[:, at // G].T.astype(np.float64)).cuda()
            want = d * x.double()[torch.arange(N, device="cuda"), torch.from_numpy(at).cuda()][:, None]
            assert torch.equal(got, want.to(BF16))


@pytest.mark.parametrize("form,dtype", ALL, ids=IDS)
def test_the_largest_values_of_x(form, dtype):
    """Finite rows of x up to the type's largest number have finite rows of y
    wherever that is what the product is, infinities of its sign where it is
    beyond, and change no bit of another row; infinities and NaN stay."""
    N, R, widths = FORMS[form]
    D, G, big = widths[-1], 64, float(torch.finfo(dtype).max)
    say(form, dtype, D)
    q, s, z = levels(R, D, G)
    s = (s * 2.0 ** -12).astype(np.float32)
    s[::3] *= 4096   # the largest number times these and more than one level is beyond fp32
    m, r = load(q, s, z, G), np.random.default_rng([2, N, D])
    x = place(r.normal(size=(N, D)), dtype)
    clean = product(m, x, dtype)
    rows = sorted({0, N // 2, N - 1})
    at = r.integers(0, D, len(rows))
    for n, d in zip(rows, at):
        x[n] = 0
        x[n, d] = big if n else -big
    y = product(m, x, dtype)
    keep = [n for n in range(N) if n not in rows]
    assert torch.equal(y[keep], clean[keep])
    v = x.double()[rows, torch.from_numpy(at).cuda()].cpu().numpy()
    d = (q[:, at].astype(np.float64) - z[:, at // G]).T
    sd = s[:, at // G].T.astype(np.float64)
    want = torch.from_numpy(d * sd * v[:, None]).float().double().numpy()
    got = y[rows].double().cpu().numpy()
    near = np.abs(want) < 0.99 * big
    # roundings as in one_column_share (bf16: exact but for the scale), then the output's
    tol = 2.0 ** -24 * sd * np.abs(v)[:, None] * (2.1 * 15 + 15 + 2 * np.abs(d)) + {F32: 2.0 ** -24, BF16: 2.0 ** -8}[dtype] * np.abs(want)
    assert near.any() and (np.abs(got[near] - want[near]) <= 1.01 * tol[near]).all()
    far = np.isinf(want)
    assert far.any() and (got[far] == want[far]).all()
    # two that cancel, in one group: what is left is theirs times the difference of their levels
    if D > 1:
        x[rows[0]] = 0
        x[rows[0], 0], x[rows[0], 1] = big, -big
        got = product(m, x, dtype)[rows[0]].double().cpu().numpy()
        want = (q[:, 0].astype(np.float64) - q[:, 1]) * s[:, 0] * big
        near = np.abs(want) < 0.99 * big
        tol = 2.0 ** -24 * s[:, 0].astype(np.float64) * big * (6 * 15 + 4 * 15) + {F32: 2.0 ** -24, BF16: 2.0 ** -8}[dtype] * np.abs(want)
        assert near.any() and (np.abs(got[near] - want[near]) <= 1.01 * tol[near]).all()
    for bad in (float("inf"), float("nan")):
        x[rows[0], D - 1] = bad
        assert not torch.isfinite(product(m, x, dtype)[rows[0]]).any()
