"""The binding of the token operators, without a device: where a call's memory comes
from."""
import contextlib

import pytest
import torch


@pytest.fixture()
def native():
    from paper_1508_00703_amd import native

    return native


class Memory:
    """Stands for a tensor: the stream it was made on and those it was recorded on."""

    def __init__(self, home):
        self.home, self.recorded = home, []

    def record_stream(self, stream):
        self.recorded.append(stream)

    def data_ptr(self):
        return 4096

    def numel(self):
        return 100


class Stream:
    def __init__(self, handle):
        self.cuda_stream = handle


class Like:
    device = torch.device("cuda", 0)

    def get_device(self):
        return 0


@pytest.fixture()
def streams(monkeypatch):
    """Two streams, the first one current, and torch's allocations noting theirs."""
    now = [Stream(10)]
    other = Stream(20)

    @contextlib.contextmanager
    def on(stream):
        now.append(stream)
        yield
        now.pop()

    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: now[-1])
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: now[-1].cuda_stream,
                        raising=False)
    monkeypatch.setattr(torch, "empty", lambda *a, **k: Memory(now[-1]))
    return now[0], other


def test_memory_comes_from_the_stream_of_the_call(native, streams):
    """Memory that the current stream has freed may still be read by it: a call on
    another stream must not write there."""
    current, other = streams
    for stream, home in ((None, current), (current, current), (other, other), (Stream(20), None)):
        home = home or stream
        out = native._empty(Like(), (3, 4), torch.float32, stream)
        assert out.home is home
        # a result may be used and dropped on the current stream
        assert home is current or out.recorded == [current]
        _, _, ws = native._space(None, 100, Like(), stream)
        assert ws.home is home


CALLS = {
    "pdb_embed_lookup": ("table", "tokens"),
    "pdb_embed_grad": ("dy", "tokens", "grad"),
    "pdb_token_logprobs": ("logits",),
    "pdb_token_logprobs_grad": ("logits", "tokens", "stats"),
    "pdb_distill": ("logits", "ids", "teacher"),
}


@pytest.mark.parametrize("call", CALLS)
def test_every_argument_by_name(native, call):
    """The arguments are taken (and then refused, for they are on no device); one that is
    missing is named."""
    given = {name: torch.zeros(3, 10) for name in CALLS[call]}
    with pytest.raises(ValueError, match="device"):
        getattr(native, call)(**given)
    for name in given:
        with pytest.raises(TypeError, match="'%s'" % name):
            getattr(native, call)(**{k: x for k, x in given.items() if k != name})
