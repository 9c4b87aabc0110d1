"""A workspace taken from torch comes from the memory of the stream that the
kernels run on, whichever is current: memory of another stream could be
handed out again while they run."""

import pytest
import torch

from paper_1905_00689_amd import binding as B

pytestmark = pytest.mark.gpu


def test_workspace_is_of_the_stream_that_uses_it(monkeypatch):
    index, taken, used = torch.cuda.current_device(), [], []
    T, Bn, H = 5000, 1, 64
    n = B.approx_lstm_linear_workspace(T, Bn, H)
    assert n
    side, other, default = torch.cuda.Stream(), torch.cuda.Stream(), torch.cuda.default_stream()
    empty = torch.empty

    def recorded(*a, **kw):
        taken.append(B._raw_stream(index))
        return empty(*a, **kw)

    monkeypatch.setattr(B.torch, "empty", recorded)
    for current in (side, default):
        for given in (None, 0, default, other, other.cuda_stream, current):
            with torch.cuda.stream(current):   # (a call that launches nothing: its stream alone is looked at)
                B._linear_call(lambda at, size, s: used.append(s) or B.OK, T, Bn, H, 0, index, None, given, ())
            want = current.cuda_stream if given is None else getattr(given, "cuda_stream", given)
            assert taken[-1] == used[-1] == want
            assert torch.cuda.current_stream() == default
