"""Sizes that no call of the gated linear recurrence takes are refused before
anything is computed from them, by the workspace query as by the calls (no GPU)."""

import ctypes

import numpy as np
import pytest
import torch

from paper_1905_00689_amd import binding as B

P = ctypes.c_void_p(4096)      # an address that no refused call looks at


def query(T, Bn, H, backward):
    n = ctypes.c_uint64(77)
    return B.lib.approx_lstm_linear_workspace(T, Bn, H, backward, ctypes.byref(n)), n.value


# 4 B H elements of 2 bytes make 2 GiB from B H = 2^28; 2^30 x 2^30 x 16 bytes are 0 modulo 2^64
@pytest.mark.parametrize("Bn,H", [(1 << 28, 1), (1, 1 << 28), (1 << 30, 1 << 30), (1 << 15, 1 << 15),
                                  ((1 << 31) - 1, (1 << 31) - 1)])
def test_timesteps_of_2_gib(Bn, H):
    for dtype in (0, 1):
        assert B.lib.approx_lstm_linear_run(P, None, 1, Bn, H, dtype, None, None, P, None, None, None, 0, None) == 6
        assert B.lib.approx_lstm_linear_backward(P, None, 1, Bn, H, dtype, None, P, P, None, P, None, None, None, 0,
                                                 None) == 6
    for backward in (0, 1, 2):
        assert query(1, Bn, H, backward) == (6, 77)


@pytest.mark.parametrize("T,Bn,H", [(1 << 28, 1024, 2), ((1 << 28) + 1, 1, 2), (1 << 30, 1 << 20, 100),
                                    ((1 << 31) - 1, 1, 1)])
def test_backward_passes_of_too_many_pieces(T, Bn, H):
    """T / 64 x B H / 128 above 2^22 (the first: B T / 64 = 2^32 rows of partial sums)."""
    for backward in (1, 2):
        assert query(T, Bn, H, backward) == (6, 77)
    assert B.lib.approx_lstm_linear_backward(P, None, T, Bn, H, 1, None, P, P, None, P, None, P, None, 0, None) == 6


def test_sizes_of_more_than_32_bits_are_not_cut():
    """2^32 + 5 timesteps are not five."""
    for T, Bn, H in (((1 << 32) + 5, 1, 64), (5, (1 << 32) + 1, 64), (5, 1, (1 << 32) + 64), (1 << 31, 1, 1)):
        with pytest.raises(ValueError):
            B.approx_lstm_linear_workspace(T, Bn, H, 0, "cuda:0")
    assert B._int32((1 << 31) - 1, "n") == (1 << 31) - 1


@pytest.mark.gpu
def test_tensors_of_more_than_2_32_rows_are_refused():
    n = 1 << 32
    p, h = torch.empty(n + 5, 1, 4, dtype=torch.bfloat16, device="cuda"), torch.empty(n + 5, 1, 1, dtype=torch.bfloat16,
                                                                                      device="cuda")
    with pytest.raises(ValueError):
        B.approx_lstm_linear_run(p, h)
    with pytest.raises(ValueError):   # as many sequences
        B.approx_lstm_linear_run(p.view(1, n + 5, 4), h.view(1, n + 5, 1))
    del p
    m = B.approx_lstm_q4_prepare(np.ones((1, 1), np.float32), 32)
    with pytest.raises(ValueError):
        B.approx_lstm_q4_run(m, h.view(n + 5, 1), torch.empty_like(h).view(n + 5, 1))


def test_streams_of_another_device_are_refused(monkeypatch):
    """A kernel runs on its stream's GPU, where the tensors are not."""

    class Stream:
        device_index, cuda_stream = 1, 4096

    called = []
    monkeypatch.setattr(B, "_linear_workspace", lambda *a: 64)
    with pytest.raises(ValueError, match="GPU 1"):
        B._launch(0, Stream(), called.append)
    with pytest.raises(ValueError, match="GPU 1"):
        B._linear_call(lambda *a: called.append(a), 5, 1, 64, 0, 0, None, Stream(), ())
    assert not called
