"""A call on a stream other than the current one: what it allocates comes from that
stream's memory (freed memory is handed out again in the order of the stream that it belongs
to, so a workspace of another stream could be overwritten while the kernels still use it),
and its outputs are recorded on the caller's stream.  On the CPU, with fake CUDA tensors and
a stand-in for the library."""
import contextlib

import pytest
import torch

fake_tensor = pytest.importorskip("torch._subclasses.fake_tensor")

import paper_2609_07816_gb300 as kdn  # noqa: E402
from test_binding_cpu import FakeLib, acts, state  # noqa: E402

BF, F32 = torch.bfloat16, torch.float32


class Stream:
    def __init__(self, handle=7):
        self.cuda_stream, self.device = handle, torch.device("cuda:0")


@pytest.fixture
def log(monkeypatch):
    """Allocations as the stream that was current, and (tensor, stream) recordings."""
    at, made, recorded = [Stream(1)], [], []

    @contextlib.contextmanager
    def on(s):
        at.append(s)
        yield
        at.pop()

    def counted(fn):
        def alloc(*a, **kw):
            t = fn(*a, **kw)
            made.append((t, at[-1].cuda_stream))
            return t
        return alloc

    monkeypatch.setattr(kdn, "lib", FakeLib)
    monkeypatch.setattr(kdn, "_ptr", lambda t: None)
    monkeypatch.setattr(kdn, "_stream", lambda s: None)
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: at[-1])
    monkeypatch.setattr(torch.cuda, "ExternalStream", Stream)
    monkeypatch.setattr(torch.cuda, "default_stream", lambda *a: Stream(0))
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: recorded.append((t, s.cuda_stream)))
    with fake_tensor.FakeTensorMode(allow_non_fake_inputs=True):
        for n in ("empty", "empty_like"):
            monkeypatch.setattr(torch, n, counted(getattr(torch, n)))
        yield made, recorded


def calls():
    e = lambda *s, dtype=BF: torch.empty(*s, dtype=dtype, device="cuda")
    q, k, o, lse = e(2, 9, 6, 64), e(2, 9, 3, 64), e(2, 9, 6, 64), e(2, 6, 9, dtype=F32)
    at = dict(window=4, sinks=2)
    q1, k1, kc, pos = e(2, 6, 64), e(2, 3, 64), e(2, 3, 6, 64), e(2, dtype=torch.int32)
    x, w, rstd = e(5, 64), e(64), e(5, dtype=F32)
    yield "swa_fwd", 3, lambda s: kdn.kdn_swa_fwd(q, k, k, stream=s, **at)
    yield "swa_bwd", 4, lambda s: kdn.kdn_swa_bwd(q, k, k, o, lse, o, stream=s, **at)
    yield "swa_decode", 1, lambda s: kdn.kdn_swa_decode_step(q1, k1, k1, kc, kc, pos, stream=s, **at)
    yield "norm", 3, lambda s: kdn.kdn_add_rmsnorm_fwd(x, w, x, stream=s)
    yield "norm_f8", 4, lambda s: kdn.kdn_add_rmsnorm_fwd(x, w, x, out_dtype=torch.float8_e4m3fn, stream=s)
    yield "norm_bwd", 3, lambda s: kdn.kdn_add_rmsnorm_bwd(x, w, rstd, x, stream=s)
    for v in ("diag", "iso"):
        f = lambda n: getattr(kdn, f"kdn_{v}_{n}")
        a, (S, p) = acts(v, 2, 9, 3, 128, 128), state(v, 2, 3, 128, 128)
        one = [e(2, 3, *t.shape[3:]) for t in a]
        dO, saved = e(2, 9, 3, 128), e(4096, dtype=torch.uint8)
        yield v, 4, lambda s: f("fwd")(*a, stream=s)
        yield v, 10, lambda s: f("bwd")(*a, S, p, dO, stream=s)
        yield v, 5, lambda s: f("fwd_save")(*a, stream=s)
        yield v, 10, lambda s: f("bwd_saved")(*a, saved, dO, stream=s)
        yield v, 1, lambda s: f("beta_eff")(a[1], a[2], a[3], a[5], saved, stream=s)
        yield v, 1, lambda s: f("decode_step")(*one, S, p, stream=s)


def tensors(out):
    out = list(out.values()) if isinstance(out, dict) else list(out) if isinstance(out, tuple) else [out]
    return [t for t in out if t is not None]


def test_what_a_call_makes_belongs_to_its_stream(log):
    made, recorded = log
    for name, n, call in calls():
        for stream, handle in ((Stream(7), 7), (Stream(0), 0)):
            made.clear(), recorded.clear()
            out = tensors(call(stream))
            assert len(made) == n and {s for _, s in made} == {handle}, name
            assert len(recorded) == len(out) and all(t is o and s == 1 for (t, s), o in zip(recorded, out)), name
        made.clear(), recorded.clear()
        call(None)  # on the current stream: as ever
        assert len(made) == n and {s for _, s in made} == {1} and not recorded, name


def test_the_callers_own_buffers_are_left_alone(log):
    made, recorded = log
    e = lambda *s, dtype=BF: torch.empty(*s, dtype=dtype, device="cuda")
    q, lse, ws = e(2, 9, 6, 64), e(2, 6, 9, dtype=F32), e(4096, dtype=torch.uint8)
    G = {n: e(2, 9, 6, 64) for n in ("dq", "dk", "dv")}
    made.clear()
    o, l = kdn.kdn_swa_fwd(q, q, q, window=4, o=q, lse=lse, workspace=ws, stream=Stream())
    assert o is q and l is lse
    assert kdn.kdn_swa_bwd(q, q, q, q, lse, q, window=4, grads=G, workspace=ws, stream=Stream()) is G
    assert not made and not recorded
    x, w = e(5, 64), e(64)
    y, h, rstd, _ = kdn.kdn_add_rmsnorm_fwd(x, w, stream=Stream())  # h is x
    assert h is x and [id(t) for t, _ in recorded] == [id(y), id(rstd)]
