"""Short sequences of the gated linear recurrence on either side of the rule
between its forward kernels: few columns and many, 8 to 25 timesteps."""

import pytest
import torch

from .gpu_helpers import say
from .test_gpu_linear import BF16, F32, Case, check

pytestmark = pytest.mark.gpu

# 64 pairs of units are a column: few, more than two and more than four a compute unit (of 256)
WIDTHS = [(3, 130), (513, 128), (1026, 127)]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("Bn,H", WIDTHS)
@pytest.mark.parametrize("T", [8, 9, 16, 17, 24, 25])
def test_short_sequences(T, Bn, H, dtype):
    say("short", T, Bn, H, dtype)
    k = Case(T, Bn, H, dtype)
    o = k.out()
    k.run(o)
    k.back(o)
    check(k, o)


@pytest.mark.parametrize("Bn,H", WIDTHS)
@pytest.mark.parametrize("T", [9, 16, 24])
def test_short_sequences_of_unequal_lengths(T, Bn, H):
    say("short and ragged", T, Bn, H)
    n = [(5 * b) % (T + 3) - 1 for b in range(Bn)]
    k = Case(T, Bn, H, BF16, lengths=n, pad=float("nan"))
    o = k.out()
    k.run(o)
    k.back(o)
    clean = Case(T, Bn, H, BF16, lengths=n, pad=0.0)
    clean.p, clean.dh = torch.nan_to_num(k.p), torch.nan_to_num(k.dh)
    check(clean, o)
