"""Tensors of one call share a device, the one that its kernels are launched on: a pointer
into another GPU's memory is refused before the library is reached.  On the CPU, with fake
CUDA tensors and a stand-in for the library."""
import pytest
import torch

fake_tensor = pytest.importorskip("torch._subclasses.fake_tensor")

import paper_2609_07816_gb300 as kdn  # noqa: E402
from test_binding_cpu import FakeLib  # noqa: E402

BF, F32, U8, I32 = torch.bfloat16, torch.float32, torch.uint8, torch.int32


@pytest.fixture
def lib(monkeypatch):
    L = FakeLib()
    monkeypatch.setattr(kdn, "lib", lambda: L)
    monkeypatch.setattr(kdn, "_ptr", lambda t: None)
    monkeypatch.setattr(kdn, "_stream", lambda s: None)
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: True)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    with fake_tensor.FakeTensorMode(allow_non_fake_inputs=True):
        yield L


def E(*s, dtype=BF, dev="cuda:0"):
    return torch.empty(*s, dtype=dtype, device=dev)


def calls():
    """(name, function, positional tensors, keyword tensors, other keywords)."""
    q, k, cache, row = E(2, 9, 6, 64), E(2, 9, 3, 64), E(2, 3, 6, 64), E(2, 6, 9, dtype=F32)
    lens, ws, at = E(2, dtype=I32), E(4096, dtype=U8), dict(window=4, sinks=2)
    yield kdn.kdn_swa_fwd, [q, k, k], dict(lens=lens, o=q, lse=row, workspace=ws), at
    yield kdn.kdn_swa_bwd, [q, k, k, q, row, q], dict(lens=lens, grads=dict(dq=q, dk=k, dv=k), workspace=ws), at
    yield kdn.kdn_swa_cache_fill, [k, k, cache, cache], dict(lens=lens), at
    yield kdn.kdn_swa_decode_step, [E(2, 6, 64), E(2, 3, 64), E(2, 3, 64), cache, cache, lens], dict(o=E(2, 6, 64)), at
    x, w, rstd = E(5, 64), E(64), E(5, dtype=F32)
    yield kdn.kdn_add_rmsnorm_fwd, [x, w, x], dict(y=E(5, 64, dtype=torch.float8_e4m3fn), h=x, rstd=rstd,
                                                   scales=rstd), dict(out_dtype=torch.float8_e4m3fn)
    yield kdn.kdn_add_rmsnorm_bwd, [x, w, rstd, x, x], dict(dx=x, dw=E(64, dtype=F32), workspace=ws), {}
    for v, per in (("diag", (128,)), ("iso", ())):
        f = lambda n: getattr(kdn, f"kdn_{v}_{n}")
        a = [E(2, 9, 3, 128), E(2, 9, 3, 128), E(2, 9, 3, 128), E(2, 9, 3, *per), E(2, 9, 3, *per), E(2, 9, 3)]
        one = [E(2, 3, *t.shape[3:]) for t in a]
        S, p, o = E(2, 3, 128, 128, dtype=F32), E(2, 3, *per, dtype=F32), E(2, 9, 3, 128)
        out = dict(o=o, ST=S, pT=p, workspace=ws)
        G = {**dict(zip(("dq", "dk", "dv", "dg", "domega", "dr"), a)), "dS0": S, "dp0": p, "dmu": E(2, 3, dtype=F32)}
        bf = dict(out_dtype=BF)
        yield f("fwd"), [*a, S, p], out, bf
        yield f("bwd"), [*a, S, p, o, S, p], dict(grads=G, workspace=ws), bf
        yield f("fwd_save"), [*a, S, p], dict(out, saved=ws), bf
        yield f("bwd_saved"), [*a, ws, o, S, p], dict(grads=G, workspace=ws), bf
        yield f("beta_eff"), [a[1], a[2], a[3], a[5], ws], dict(out=E(2, 9, 3, dtype=F32)), {}
        yield f("decode_step"), [*one, S, p], dict(o=one[2]), bf
        if v == "diag":
            yield f("fwd_noalloc"), [*a, S, p], dict(o=o, ST=S, pT=p), {}


def moved(t):
    return E(*t.shape, dtype=t.dtype, dev="cuda:1")


def test_every_tensor_is_on_the_calls_device(lib):
    for fn, pos, kw, rest in calls():
        lib.calls.clear()
        fn(*pos, **kw, **rest)
        assert lib.calls == [fn.__name__]
        places = [(i, None) for i in range(len(pos))]
        for n, t in kw.items():
            places += [(n, g) for g in t] if isinstance(t, dict) else [(n, None)]
        # k, v and g of beta_eff only give the descriptor's sizes
        if "beta_eff" in fn.__name__:
            places.remove((1, None)), places.remove((2, None))
        for at, inner in places:
            p, q = list(pos), {n: dict(t) if isinstance(t, dict) else t for n, t in kw.items()}
            into = p if isinstance(at, int) else q
            if inner is None:
                into[at] = moved(into[at])
            else:
                into[at][inner] = moved(into[at][inner])
            lib.calls.clear()
            with pytest.raises(ValueError, match="cuda:1|cuda:0"):
                fn(*p, **q, **rest)
            assert not lib.calls, (fn.__name__, at, inner)


def test_the_calls_device_is_the_current_one(lib, monkeypatch):
    for fn, pos, kw, rest in calls():
        p = [moved(t) for t in pos]
        q = {n: {g: moved(x) for g, x in t.items()} if isinstance(t, dict) else moved(t) for n, t in kw.items()}
        lib.calls.clear()
        with pytest.raises(ValueError, match="current device"):
            fn(*p, **q, **rest)
        assert not lib.calls
        with monkeypatch.context() as m:
            m.setattr(torch._C, "_cuda_getDevice", lambda: 1, raising=False)
            fn(*p, **q, **rest)
        assert lib.calls == [fn.__name__]
