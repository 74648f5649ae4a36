"""Where the binding takes memory for what a call writes on a stream that it is given (on the host, with stand-ins for
torch's streams and memory)."""
import contextlib

import pytest

torch = pytest.importorskip("torch")

from paper_2607_24377_amd import mxattn  # noqa: E402


class Stream:
    def __init__(self, handle, device=None):
        self.cuda_stream = handle


class Memory:
    def __init__(self, owner):
        self.owner, self.users = owner, []

    def record_stream(self, stream):
        self.users.append(stream.cuda_stream)


@pytest.fixture
def streams(monkeypatch):
    now = [Stream(5)]

    @contextlib.contextmanager
    def on(stream):
        now.append(stream)
        yield
        now.pop()

    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: now[-1])
    monkeypatch.setattr(torch.cuda, "ExternalStream", Stream)
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch, "empty", lambda shape, dtype, device: Memory(now[-1].cuda_stream))
    return now


@pytest.mark.parametrize("stream,owner,users", [(None, 5, []), (5, 5, []), (Stream(5), 5, []), (9, 9, [5]), (Stream(9), 9, [5])])
def test_memory_is_of_the_stream_that_writes_it(streams, stream, owner, users):
    m = mxattn._empty((3,), torch.int32, "cuda:0", stream)
    assert (m.owner, m.users) == (owner, users)
    assert len(streams) == 1
