"""Rotary positions without a GPU: the table of frequencies, what the C entry points refuse
before any CUDA call, and what the Python binding refuses before the C entry point."""
import ctypes
import math

import pytest
import torch

import rope_ref as ref

BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32
FAKE = ctypes.c_void_p(1 << 20)       # aligned, never dereferenced
MIS = ctypes.c_void_p((1 << 20) + 8)  # not 16-byte aligned


@pytest.fixture(scope="module")
def kdn():
    from paper_2609_07816_gb300 import build
    build.build()
    import paper_2609_07816_gb300 as m
    return m


@pytest.mark.parametrize("rot", [2, 6, 20, 64, 128, 256])
@pytest.mark.parametrize("base", [10000.0, 500000.0, 1.5])
@pytest.mark.parametrize("factor,trained", [(1.0, 0), (1.0, 4096), (8.0, 0), (16.0, 4096), (40.0, 8192), (1.5, 1)])
def test_table_is_the_formula(kdn, rot, base, factor, trained):
    f = kdn.kdn_rope_freqs(rot, base=base, factor=factor, trained=trained)
    want, m = ref.table(rot, base, factor, trained)
    assert len(f.turns) == rot // 2 and f.rot == rot
    assert abs(f.mscale - m) <= 2.0 ** -23
    for a, b in zip(f.turns, want):
        # a power, a few products and a quotient in 64 bits on either side; w times a frequency
        # that it nearly keeps loses what its two parts cancel, at most 32 / 31
        assert abs(a / 2.0 ** 64 * 2 * math.pi - b) <= 64 * 2.0 ** -52 * b + 2.0 ** -62


def test_table_refusals(kdn):
    inv, uns = kdn.KDN_ERR_INVALID_ARG, kdn.KDN_ERR_UNSUPPORTED
    ok = dict(rot=64)
    for over, want in ((dict(rot=0), inv), (dict(rot=-2), inv), (dict(rot=7), inv), (dict(rot=258), uns),
                       (dict(base=1.0), inv), (dict(base=math.inf), inv), (dict(base=math.nan), inv),
                       (dict(factor=0.5), inv), (dict(factor=math.nan), inv), (dict(factor=math.inf), inv),
                       (dict(trained=-1), inv), (dict(trained=math.inf), inv), (dict(beta_fast=1.0), inv),
                       (dict(beta_slow=-1.0), inv), (dict(beta_fast=math.inf), inv), (dict(beta_slow=math.nan), inv)):
        with pytest.raises(kdn.KdnError) as e:
            kdn.kdn_rope_freqs(**{**ok, **over})
        assert e.value.status == want, over
    assert kdn.lib().kdn_rope_freqs(None, (ctypes.c_ulonglong * 1)(), None) == inv
    f = kdn.kdn_rope_freqs_t(2, 1e4, 1.0, 0.0, 32.0, 1.0)
    assert kdn.lib().kdn_rope_freqs(ctypes.byref(f), None, None) == inv
    t = (ctypes.c_ulonglong * 1)()
    assert kdn.lib().kdn_rope_freqs(ctypes.byref(f), t, None) == kdn.KDN_OK and t[0]  # mscale not wanted
    with pytest.raises(ValueError):
        kdn.RopeFreqs(8, t, 1.0)


def desc(kdn, **over):
    base = dict(B=2, T=8, H=4, Hk=2, d=64, rot=64, interleaved=0, pos_per_token=0, dtype=1, mscale=1.0, ldq=0, ldk=0,
                ldqo=0, ldko=0)
    base.update(over)
    return kdn.kdn_rope_desc_t(*base.values())


def status(kdn, back, d, args=None, turns=None):
    fn = kdn.lib().kdn_rope_bwd if back else kdn.lib().kdn_rope_fwd
    q, k, pos, lens, qo, ko = args or [ctypes.c_void_p(1 << (20 + i)) for i in range(6)]
    return fn(ctypes.byref(d) if d else None, turns or (ctypes.c_ulonglong * 128)(), q, k, pos, lens, qo, ko, None)


@pytest.mark.parametrize("back", [False, True])
def test_refusals(kdn, back):
    inv, uns = kdn.KDN_ERR_INVALID_ARG, kdn.KDN_ERR_UNSUPPORTED
    for over, want in ((dict(B=-1), inv), (dict(T=-1), inv), (dict(H=-1), inv), (dict(Hk=-1), inv), (dict(d=0), inv),
                       (dict(rot=0), inv), (dict(rot=33), inv), (dict(rot=66), inv), (dict(dtype=2), inv),
                       (dict(interleaved=2), inv), (dict(pos_per_token=-1), inv), (dict(mscale=math.nan), inv),
                       (dict(mscale=math.inf), inv), (dict(ldq=255), inv), (dict(ldk=127), inv), (dict(ldqo=-256), inv),
                       (dict(ldko=1), inv), (dict(ldq=2**31 + 8), uns), (dict(d=60, rot=60), uns),
                       (dict(d=264, rot=64), uns), (dict(T=2**21 + 1), uns), (dict(H=65536), uns),
                       (dict(Hk=65536), uns), (dict(B=1025, T=2**21), uns)):
        assert status(kdn, back, desc(kdn, **over)) == want, over
    assert status(kdn, back, None) == inv
    good = [ctypes.c_void_p(1 << (20 + i)) for i in range(6)]
    for i in range(6):
        for bad in (None, MIS) if i not in (2, 3) else (MIS,):
            a = list(good)
            a[i] = bad
            assert status(kdn, back, desc(kdn), a) == inv, i
    a = list(good)
    a[2] = None
    assert status(kdn, back, desc(kdn, pos_per_token=1), a) == inv  # no positions
    # in place, but with other row distances
    for i, j, over in ((0, 4, dict(ldq=512)), (1, 5, dict(ldko=512))):
        a = list(good)
        a[j] = a[i]
        assert status(kdn, back, desc(kdn, **over), a) == inv
    fn = kdn.lib().kdn_rope_bwd if back else kdn.lib().kdn_rope_fwd
    assert fn(ctypes.byref(desc(kdn)), None, *good, None) == inv
    for over in (dict(B=0), dict(T=0), dict(H=0, Hk=0)):
        assert fn(ctypes.byref(desc(kdn, **over)), None, *[None] * 7) == kdn.KDN_OK


# ------------------------------------------------------------------ the binding


class FakeLib:
    def __init__(self, log):
        self.log = log

    def __getattr__(self, name):
        def call(d, *args):
            self.log.append((name, d._obj))
            return 0
        return call


@pytest.fixture
def fake(monkeypatch, kdn):
    fake_tensor = pytest.importorskip("torch._subclasses.fake_tensor")
    f = kdn.kdn_rope_freqs(64)
    log = []
    monkeypatch.setattr(kdn, "lib", lambda: FakeLib(log))
    monkeypatch.setattr(kdn, "_ptr", lambda t: None)
    monkeypatch.setattr(kdn, "_stream", lambda s: None)
    with fake_tensor.FakeTensorMode(allow_non_fake_inputs=True):
        yield kdn, f, log


def E(*s, dtype=BF, dev="cuda"):
    return torch.empty(*s, dtype=dtype, device=dev)


def test_binding_reaches_the_library(fake):
    m, f, log = fake
    q, k, lens, pos = E(2, 9, 6, 64), E(2, 9, 3, 64), E(2, dtype=I32), E(2, dtype=I32)
    qo, ko = m.kdn_rope_fwd(q, k, f, pos=pos, lens=lens)
    assert qo.shape == q.shape and ko.shape == k.shape
    dq, dk = m.kdn_rope_bwd(qo, None, f, pos=E(2, 9, dtype=I32), interleaved=True)
    assert dq.shape == q.shape and dk is None
    assert [n for n, _ in log] == ["kdn_rope_fwd", "kdn_rope_bwd"]
    d = log[0][1]
    assert (d.B, d.T, d.H, d.Hk, d.d, d.rot, d.interleaved, d.pos_per_token, d.dtype) == (2, 9, 6, 3, 64, 64, 0, 0, 1)
    d = log[1][1]
    assert (d.Hk, d.interleaved, d.pos_per_token) == (0, 1, 1)
    # a single token of every sequence, and heads of a fused projection
    qkv = E(2, 9, 12, 64)
    q, k, _ = qkv.split((6, 3, 3), 2)
    assert m.kdn_rope_fwd(q, k, f, qo=q, ko=k) == (q, k)
    d = log[-1][1]
    assert (d.ldq, d.ldk, d.ldqo, d.ldko) == (768,) * 4
    q, k, _ = E(5, 12, 64).split((6, 3, 3), 1)
    dq, dk = m.kdn_rope_bwd(q, k, f, pos=E(5, dtype=I32))
    d = log[-1][1]
    assert (d.B, d.T, d.ldq, d.ldqo, d.ldko) == (5, 1, 0, 768, 768) and dq.is_contiguous()  # 0: dense
    # a batch or a length of one says nothing about the distance of the other's rows
    m.kdn_rope_fwd(E(4, 3, 12, 64)[:, 1:2, :6], None, f)
    assert log[-1][1].ldq == 3 * 768
    m.kdn_rope_fwd(E(4, 3, 12, 64)[1:2, :, 2:8], None, f)
    assert log[-1][1].ldq == 768


def test_binding_refuses_bad_tensors(fake):
    m, f, log = fake
    q, k = E(2, 9, 6, 64), E(2, 9, 3, 64)
    fwd = m.kdn_rope_fwd
    bad = [
        lambda: fwd(E(2, 9, 6, 64, dev="cpu"), k, f),
        lambda: fwd(None, k, f),
        lambda: fwd(q.half(), k.half(), f),
        lambda: fwd(q, k.float(), f),
        lambda: fwd(q, E(2, 8, 3, 64), f),
        lambda: fwd(q, E(2, 9, 3, 32), f),
        lambda: fwd(q, E(9, 3, 64), f),
        lambda: fwd(q[0, 0], None, f),
        lambda: fwd(q[None], None, f),
        lambda: fwd(q, k, None),
        lambda: fwd(q, k, f.turns),
        lambda: fwd(q, k, f, pos=E(3, dtype=I32)),
        lambda: fwd(q, k, f, pos=E(2, dtype=torch.int64)),
        lambda: fwd(q, k, f, pos=E(9, 2, dtype=I32)),
        lambda: fwd(q, k, f, pos=E(2, 9, 1, dtype=I32)),
        lambda: fwd(q, k, f, pos=5),
        lambda: fwd(q, k, f, lens=E(2, 9, dtype=I32)),
        lambda: fwd(q, k, f, lens=E(2, dtype=torch.int64)),
        lambda: fwd(q.transpose(1, 2), None, f),            # heads apart
        lambda: fwd(E(2, 9, 6, 128)[..., ::2], None, f),    # channels apart
        lambda: fwd(E(2, 9, 6, 128)[..., :64], None, f),    # heads not dense
        lambda: fwd(E(2, 12, 6, 64)[:, :9], None, f),       # sequences apart
        lambda: fwd(E(1, 1, 6, 64).expand(2, 9, 6, 64), None, f),
        lambda: fwd(q, k, f, qo=E(2, 9, 6, 64, dtype=F32)),
        lambda: fwd(q, k, f, ko=E(2, 9, 4, 64)),
        lambda: fwd(q, k, f, qo=E(18, 6, 64)),
        lambda: fwd(q, None, f, ko=k),
        lambda: m.kdn_rope_bwd(q, k, f, dq=E(2, 9, 6, 64, dev="cpu")),
        lambda: m.kdn_rope_bwd(None, k, f),
    ]
    for i, call in enumerate(bad):
        with pytest.raises((ValueError, TypeError)):
            call()
        assert not log, i


def test_binding_devices_and_streams(fake, monkeypatch):
    m, f, log = fake
    q, k, pos = E(2, 9, 6, 64), E(2, 9, 3, 64), E(2, dtype=I32)
    far = lambda t: E(*t.shape, dtype=t.dtype, dev="cuda:1")
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: True)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    for kw in (dict(q=far(q)), dict(k=far(k)), dict(pos=far(pos)), dict(lens=far(pos)), dict(qo=far(q)),
               dict(ko=far(k))):
        with pytest.raises(ValueError, match="cuda:"):
            m.kdn_rope_fwd(**{**dict(q=q, k=k, freqs=f, pos=pos), **kw})
        assert not log


def test_a_table_of_other_entries_is_refused(kdn):
    """The library reads rot/2 entries of 64 bits: behind the end of an array of 32-bit ones, and the bits
    of floating-point numbers as turns."""
    for kind in (ctypes.c_uint32, ctypes.c_double, ctypes.c_longlong):
        with pytest.raises(TypeError):
            kdn.RopeFreqs(8, (kind * 4)(), 1.0)
    with pytest.raises(TypeError):
        kdn.RopeFreqs(8, [1, 2, 3, 4], 1.0)
    assert kdn.RopeFreqs(8, (ctypes.c_ulonglong * 4)(), 1.0).rot == 8
