"""Workspaces that the operators' binding makes itself belong to the stream that the call runs on.  No GPU."""
import contextlib

import pytest
import torch

from paper_1805_08768_amd import binding as sbc


class Recorder:
    """Stands in for torch's streams and allocator: notes under which stream each allocation is made."""

    def __init__(self, monkeypatch):
        self.under, self.made = None, []
        empty = torch.empty
        monkeypatch.setattr(torch.cuda, "stream", self.stream)
        monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, device=None: ("handle", handle))
        monkeypatch.setattr(torch, "empty", lambda *a, **kw: (self.made.append(self.under), empty(*a, **kw))[1])
        monkeypatch.setattr(torch.Tensor, "record_stream", lambda *a: None)

    @contextlib.contextmanager
    def stream(self, s):
        before, self.under = self.under, s
        yield
        self.under = before


class OfSomeLibrary:
    cuda_stream = 77


@pytest.mark.parametrize("stream,under", [(None, None), (1234, ("handle", 1234)), (0, ("handle", 0)), (OfSomeLibrary(), ("handle", 77))])
def test_a_workspace_is_allocated_under_the_calls_stream(monkeypatch, stream, under):
    """Otherwise the block may be one whose last users are still queued on the current stream, which nothing orders
    before the call on its own."""
    made = Recorder(monkeypatch)
    keep, ptr, size = sbc._scratch(100, None, torch.device("cpu"), stream)
    assert made.made == [under] and size == 100 and keep.data_ptr() == ptr


def test_no_workspace_where_none_is_needed():
    assert sbc._scratch(0, None, torch.device("cpu"), 1234) == (None, None, 0)
