"""The stream the binding hands to the library: torch's current one, by its short cut or, in a torch that has none, through
the Stream object."""
import types

import pytest
import torch

from paper_2607_05147_b200 import binding as B


def test_a_torch_without_the_short_cut(monkeypatch):
    monkeypatch.setattr(B, "_raw_stream", None)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: types.SimpleNamespace(cuda_stream=1234))
    assert B._stream() == 1234


@pytest.mark.gpu
def test_it_is_the_current_stream():
    side = torch.cuda.Stream()
    for _ in range(2):
        assert B._stream() == torch.cuda.current_stream().cuda_stream
        with torch.cuda.stream(side):
            assert B._stream() == side.cuda_stream
