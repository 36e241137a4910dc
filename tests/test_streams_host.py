"""Memory that the binding allocates for a call on a given stream comes from that stream."""
import contextlib

import pytest
import torch

from paper_2608_13263_amd import binding as B


@pytest.fixture
def streams(monkeypatch):
    """torch.cuda's streams by names: what is current, where each allocation is made and which
    streams it is kept for."""
    log = {"at": [], "kept": []}
    current = ["current"]

    class Stream:
        def __init__(self, name):
            self.cuda_stream = name

    @contextlib.contextmanager
    def within(stream):
        current.append(stream.cuda_stream)
        yield
        current.pop()

    empty = torch.empty

    def made(shape, dtype, device):
        log["at"].append(current[-1])
        return empty(shape, dtype=dtype, device="cpu")

    monkeypatch.setattr(torch.cuda, "Stream", Stream)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda raw, device: Stream(raw))
    monkeypatch.setattr(torch.cuda, "default_stream", lambda device: Stream("default"))
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: Stream(current[-1]))
    monkeypatch.setattr(torch.cuda, "stream", within)
    monkeypatch.setattr(torch, "empty", made)
    monkeypatch.setattr(torch.Tensor, "record_stream",
                        lambda x, s: log["kept"].append(s.cuda_stream))
    log["Stream"] = Stream
    return log


def test_memory_of_the_stream_that_writes_it(streams):
    x = B._empty((3, 2), torch.float32, "cuda", None)
    assert x.shape == (3, 2) and x.dtype == torch.float32
    B._empty(4, torch.int32, "cuda", streams["Stream"](7))
    B._empty(4, torch.int32, "cuda", 11)    # by its handle
    B._empty(4, torch.int32, "cuda", 0)     # the handle of the default stream
    assert streams["at"] == ["current", 7, 11, "default"]
    assert streams["kept"] == ["current"] * 3


def test_workspaces_are_the_streams_own(streams):
    """No other stream touches a workspace: the next call on its stream may have it at once."""
    B._on(streams["Stream"](7), False)(3, 2, dtype=torch.float32, device="cuda")
    assert streams["at"] == [7] and streams["kept"] == []
    B._on(streams["Stream"](7))(5, dtype=torch.float32, device="cuda")
    assert streams["at"] == [7, 7] and streams["kept"] == ["current"]
