"""The kept status word of feed-forward calls that have nothing else to put in a workspace: calls of
every stream write there, so its memory must have no user left on the stream that it was taken
from.  On the CPU, with fake CUDA tensors and a stand-in for the library."""
import pytest
import torch

from test_streams_cpu import Stream, fake_tensor, kdn, log  # noqa: F401

BF = torch.bfloat16


@pytest.fixture
def events(log, monkeypatch):  # noqa: F811
    """(what, stream) in their order: words made, streams waited for, calls of the library."""
    seen = []

    class Small:
        def __getattr__(self, name):
            if name.endswith("_bytes"):
                return lambda *a: 256
            return lambda *a: seen.append(("call", torch.cuda.current_stream().cuda_stream)) or 0

    empty = torch.empty

    def alloc(*a, **kw):
        if kw.get("dtype") == torch.uint8:
            seen.append(("word", torch.cuda.current_stream().cuda_stream))
        return empty(*a, **kw)
    monkeypatch.setattr(torch, "empty", alloc)
    monkeypatch.setattr(kdn, "lib", Small)
    monkeypatch.setattr(kdn, "_status_words", {})
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: True)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(Stream, "synchronize", lambda s: seen.append(("done", s.cuda_stream)), raising=False)
    e = lambda *s: empty(*s, dtype=BF, device="cuda:0")
    x, wg, wd = e(5, 64), e(96, 64), e(64, 96)
    return seen, lambda s=None: kdn.kdn_ffn_fwd(x, wg, wg, wd, want_saved=False, stream=s)


@pytest.mark.parametrize("first", [1, 7])
def test_its_memory_has_no_user_left(events, first):
    """Freed memory is handed out while the kernels of its own stream still use it; another stream may write
    there only when they are done.  The wait comes once, on the stream that the word was taken from."""
    seen, call = events
    call(Stream(7) if first == 7 else None)
    assert seen == [("word", first), ("done", first), ("call", first)]
    seen.clear()
    for s in (None, Stream(7), Stream(0), None):
        call(s)
    assert seen == [("call", 1), ("call", 7), ("call", 0), ("call", 1)]


def test_in_a_capture_it_is_the_graphs(events, monkeypatch):
    """A captured call's word comes with the call, on its stream; nothing is waited for or kept."""
    seen, call = events
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    for _ in range(2):
        call(Stream(7))
    assert seen == [("word", 7), ("call", 7)] * 2 and not kdn._status_words
