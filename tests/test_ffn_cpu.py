"""The gated feed-forward block without a GPU: what the C entry points refuse before any CUDA
call, what the Python binding refuses before the C entry point, and the 64-bit reference's
gradients against differences."""
import ctypes

import pytest
import torch

import ffn_ref as ref

BF, F32 = torch.bfloat16, torch.float32
FAKE = ctypes.c_void_p(1 << 20)       # aligned, never dereferenced
MIS = ctypes.c_void_p((1 << 20) + 8)  # not 16-byte aligned


@pytest.fixture(scope="module")
def kdn():
    from paper_2609_07816_gb300 import build
    build.build()
    import paper_2609_07816_gb300 as m
    return m


def desc(kdn, **over):
    base = dict(rows=4, D=64, F=96, dtype=1, act=0, dw_dtype=1)
    base.update(over)
    return kdn.kdn_ffn_desc_t(*base.values())


def calls(kdn, d, at=None, bad=None, ws=FAKE, n=1 << 40):
    L, p = kdn.lib(), ctypes.byref(d) if d else None
    args = lambda m: [bad if i == at else FAKE for i in range(m)]
    return {"fwd": lambda: L.kdn_ffn_fwd(p, *args(8), ws, n, None), "bwd": lambda: L.kdn_ffn_bwd(p, *args(12), ws, n, None)}


def test_refuses_bad_descriptors(kdn):
    inv, uns = kdn.KDN_ERR_INVALID_ARG, kdn.KDN_ERR_UNSUPPORTED
    for over, want in ((dict(rows=-1), inv), (dict(D=0), inv), (dict(D=-8), inv), (dict(F=0), inv), (dict(F=-64), inv),
                       (dict(dtype=2), inv), (dict(dtype=-1), inv), (dict(act=2), inv), (dict(act=-1), inv),
                       (dict(dw_dtype=2), inv), (dict(dtype=0), inv), (dict(D=60), uns), (dict(F=97), uns),
                       (dict(D=2**20 + 8), uns), (dict(F=2**20 + 8), uns), (dict(rows=2**31), uns)):
        d = desc(kdn, **over)
        for name, call in calls(kdn, d).items():
            assert call() == want, (over, name)
        assert kdn.lib().kdn_ffn_fwd_workspace_bytes(ctypes.byref(d)) == 0
        assert kdn.lib().kdn_ffn_bwd_workspace_bytes(ctypes.byref(d)) == 0
    for name, call in calls(kdn, None).items():
        assert call() == inv


def test_refuses_bad_pointers_and_workspaces(kdn):
    inv = kdn.KDN_ERR_INVALID_ARG
    d = desc(kdn)
    for name, n in (("fwd", 8), ("bwd", 12)):
        for i in range(n):
            for bad in (None, MIS):  # (one of g and u alone is missing in the forward)
                assert calls(kdn, d, i, bad)[name]() == inv, (name, i)
    for name, fn in (("fwd", kdn.lib().kdn_ffn_fwd_workspace_bytes), ("bwd", kdn.lib().kdn_ffn_bwd_workspace_bytes)):
        need = fn(ctypes.byref(d))
        assert need >= 256
        for ws, n in ((None, 1 << 40), (MIS, 1 << 40), (FAKE, need - 1)):
            assert calls(kdn, d, ws=ws, n=n)[name]() == kdn.KDN_ERR_WORKSPACE


@pytest.mark.parametrize("rows", [1, 16, 17, 61, 256, 1777, 32768])
@pytest.mark.parametrize("D,F", [(64, 64), (2048, 5632), (2304, 6144), (4096, 8192)])
@pytest.mark.parametrize("dtype", [0, 1])
def test_workspace_is_bounded(kdn, rows, D, F, dtype):
    """Partial sums of products that leave most SMs idle: at most 608 tiles of 256 x 128; the backward keeps
    dg and du beside them.  float32 keeps its operands in three bfloat16s an element, but up to 16 rows
    only dg and du."""
    d = ctypes.byref(desc(kdn, rows=rows, D=D, F=F, dtype=dtype, dw_dtype=dtype))
    part = 608 * 256 * 128 * 4
    xs, hs, ws = rows * D, rows * F, 3 * D * F
    few = rows <= 16
    keeps = (0, 4 * hs) if dtype else (0, 8 * hs) if few else (6 * (xs + hs + ws), 6 * (2 * xs + 3 * hs + ws))
    for fn, n in zip((kdn.lib().kdn_ffn_fwd_workspace_bytes, kdn.lib().kdn_ffn_bwd_workspace_bytes), keeps):
        assert 256 <= fn(d) - n <= 256 * 10 + part


def test_no_rows(kdn):
    d = desc(kdn, rows=0)
    assert kdn.lib().kdn_ffn_fwd(ctypes.byref(d), *[None] * 9, 0, None) == kdn.KDN_OK
    # the weights' gradients are sums over nothing, to be written
    assert kdn.lib().kdn_ffn_bwd(ctypes.byref(d), *[None] * 13, 0, None) == kdn.KDN_ERR_INVALID_ARG


# ------------------------------------------------------------------ the binding


class FakeLib:
    def __init__(self, log):
        self.log = log

    def __getattr__(self, name):
        if name.endswith("_bytes"):
            return lambda *a: 4096

        def call(d, *args):
            self.log.append((name, d._obj))
            return 0
        return call


@pytest.fixture
def fake(monkeypatch):
    fake_tensor = pytest.importorskip("torch._subclasses.fake_tensor")
    import paper_2609_07816_gb300 as m
    log = []
    monkeypatch.setattr(m, "lib", lambda: FakeLib(log))
    monkeypatch.setattr(m, "_ptr", lambda t: None)
    monkeypatch.setattr(m, "_stream", lambda s: None)
    with fake_tensor.FakeTensorMode(allow_non_fake_inputs=True):
        yield m, log


def E(*s, dtype=BF, dev="cuda"):
    return torch.empty(*s, dtype=dtype, device=dev)


def test_binding_reaches_the_library(fake):
    m, log = fake
    x, wg, wu, wd = E(3, 5, 64), E(96, 64), E(96, 64), E(64, 96)
    y, g, u, h = m.kdn_ffn_fwd(x, wg, wu, wd, act=m.KDN_ACT_GELU)
    assert y.shape == x.shape and g.shape == u.shape == h.shape == (3, 5, 96)
    G = m.kdn_ffn_bwd(x, wg, wu, wd, g, u, h, y, dw_dtype=F32)
    assert G["dx"].shape == x.shape and G["dwg"].shape == (96, 64) and G["dwd"].shape == (64, 96)
    assert G["dwg"].dtype == F32 and G["dx"].dtype == BF
    y, g, u, h2 = m.kdn_ffn_fwd(x, wg, wu, wd, want_saved=False, h=h)
    assert g is None and u is None and h2 is h
    m.kdn_ffn_bwd(x, wg, wu, wd, h, h, h, y, grads=G, dw_dtype=F32, workspace=E(8192, dtype=torch.uint8))
    assert [n for n, _ in log] == ["kdn_ffn_fwd", "kdn_ffn_bwd"] * 2
    d = log[0][1]
    assert (d.rows, d.D, d.F, d.dtype, d.act, d.dw_dtype) == (15, 64, 96, 1, 1, 1)
    assert log[1][1].dw_dtype == 0


def test_binding_refuses_bad_tensors(fake):
    m, log = fake
    x, wg, wu, wd, g = E(5, 64), E(96, 64), E(96, 64), E(64, 96), E(5, 96)
    dw = {"dwg": E(96, 64), "dwu": E(96, 64), "dwd": E(64, 96)}
    fwd = m.kdn_ffn_fwd
    bwd = lambda *a, **k: m.kdn_ffn_bwd(x, wg, wu, wd, *a, **k)
    bad = [
        lambda: fwd(E(5, 64, dev="cpu"), wg, wu, wd), lambda: fwd(x.half(), wg, wu, wd), lambda: fwd(E(), wg, wu, wd),
        lambda: fwd(x, wg.float(), wu, wd), lambda: fwd(x, E(96, 72), E(96, 72), wd), lambda: fwd(x, wg, E(88, 64), wd),
        lambda: fwd(x, wg, wu, E(96, 64)), lambda: fwd(x, wg, wu, E(96, 64).T), lambda: fwd(E(64, 5).T, wg, wu, wd),
        lambda: fwd(x, wg, wu, wd, g=g), lambda: fwd(x, wg, wu, wd, u=g), lambda: fwd(x, wg, wu, wd, g=g, u=E(5, 88)),
        lambda: fwd(x, wg, wu, wd, h=E(5, 96, dtype=F32)), lambda: fwd(x, wg, wu, wd, y=E(4, 64)),
        lambda: fwd(x, wg, wu, wd, workspace=E(4096)), lambda: bwd(None, g, g, x), lambda: bwd(g, g, g, E(5, 96)),
        lambda: bwd(g, g, g.float(), x), lambda: bwd(g, g, g, x, dw_dtype=torch.float16),
        lambda: bwd(g, g, g, x, grads={"dx": x, "dwg": wg, "dwu": wu}),
        lambda: bwd(g, g, g, x, grads={"dx": x, **dw}, dw_dtype=F32), lambda: bwd(g, g, g, x, grads={**dw, "dx": g}),
    ]
    for i, call in enumerate(bad):
        with pytest.raises((ValueError, TypeError)):
            call()
        assert not log, i


def test_binding_devices(fake, monkeypatch):
    m, log = fake
    x, wg, wu, wd, g = E(5, 64), E(96, 64), E(96, 64), E(64, 96), E(5, 96)
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: True)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    ws = E(8192, dtype=torch.uint8)
    for fn, kw in ((m.kdn_ffn_fwd, dict(x=x, wg=wg, wu=wu, wd=wd, g=g, u=g, h=g, y=x, workspace=ws)),
                   (m.kdn_ffn_bwd, dict(x=x, wg=wg, wu=wu, wd=wd, g=g, u=g, h=g, dy=x, workspace=ws))):
        for n, t in kw.items():
            with pytest.raises(ValueError, match="cuda:"):
                fn(**{**kw, n: E(*t.shape, dtype=t.dtype, dev="cuda:1")})
            assert not log, n


@pytest.mark.parametrize("name", ["silu", "gelu"])
def test_reference_gradients_are_the_differences(name):
    gen = torch.Generator().manual_seed(1)
    r = lambda *s: torch.randn(*s, generator=gen, dtype=torch.float64)
    w = [r(9, 16), r(24, 16) / 4, r(24, 16) / 4, r(16, 24) / 5]
    dy, dirs = r(9, 16), [r(*t.shape) for t in w]
    y, g, u, h = ref.forward(*w, name)
    G = ref.backward(*w, g, u, h, dy, name)
    for i, n in enumerate(("dx", "dwg", "dwu", "dwd")):
        loss = lambda e: float((ref.forward(*[t + e * dirs[i] if j == i else t for j, t in enumerate(w)], name)[0] * dy).sum())
        # truncation e^2 and rounding 1e-14 / e at e = 1e-5
        assert abs((loss(1e-5) - loss(-1e-5)) / 2e-5 - float((G[n] * dirs[i]).sum())) <= 1e-7


@pytest.mark.parametrize("D,F", [(768, 2048), (1280, 1280)])
def test_workspace_of_long_sums(kdn, D, F):
    """Weights' gradients in bfloat16 whose sums are not cut: of more than 65536 rows they go through float32."""
    for rows, dw, part in ((65536, 1, 0), (65537, 1, 12 * D * F), (300000, 1, 12 * D * F), (300000, 0, 0)):
        n = kdn.lib().kdn_ffn_bwd_workspace_bytes(ctypes.byref(desc(kdn, rows=rows, D=D, F=F, dw_dtype=dw)))
        assert n == 256 + 2 * -(-rows * F * 2 // 256) * 256 + part, (rows, dw)
