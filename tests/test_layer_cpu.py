"""The hybrid layer's operators without a GPU: what the C entry points refuse before
any CUDA call, what the Python binding refuses before the C entry point, and the 64-bit
reference's gradients against differences."""
import ctypes
import math

import pytest
import torch

import swa_ref as ref

BF, F32 = torch.bfloat16, torch.float32
FAKE = ctypes.c_void_p(1 << 20)       # aligned, never dereferenced
MIS = ctypes.c_void_p((1 << 20) + 8)  # not 16-byte aligned


@pytest.fixture(scope="module")
def kdn():
    from paper_2609_07816_gb300 import build
    build.build()
    import paper_2609_07816_gb300 as m
    return m


def swa_calls(kdn, desc, at=None, bad=None, ws=FAKE, ws_bytes=1 << 40):
    """Status of every attention entry point; pointer number `at` replaced by `bad`."""
    L, d = kdn.lib(), ctypes.byref(desc)

    def args(n):
        return [bad if i == at else FAKE for i in range(n)]
    return {"fwd": lambda: L.kdn_swa_fwd(d, *args(6), ws, ws_bytes, None),
            "bwd": lambda: L.kdn_swa_bwd(d, *args(10), ws, ws_bytes, None),
            "fill": lambda: L.kdn_swa_cache_fill(d, *args(5), None),
            "decode": lambda: L.kdn_swa_decode_step(d, *args(7), None)}


def test_attention_refuses_bad_descriptors(kdn):
    base = dict(B=1, T=8, H=4, Hk=2, d=64, dtype=kdn.KDN_BF16, window=4, sinks=0, scale=None)
    inv, uns = kdn.KDN_ERR_INVALID_ARG, kdn.KDN_ERR_UNSUPPORTED
    cases = [(dict(B=-1), inv), (dict(H=-4), inv), (dict(Hk=3), inv), (dict(Hk=0), inv), (dict(Hk=-2), inv),
             (dict(window=0), inv), (dict(window=-3), inv), (dict(sinks=-1), inv), (dict(dtype=2), inv),
             (dict(dtype=-1), inv), (dict(scale=0.0), inv), (dict(scale=-1.0), inv), (dict(scale=math.inf), inv),
             (dict(d=0), inv), (dict(d=96), uns), (dict(d=256), uns), (dict(B=65536), uns),
             (dict(H=65536, Hk=65536), uns), (dict(window=2**30, sinks=1), uns)]
    for over, want in cases:
        desc = kdn.make_swa_desc(**{**base, **over})
        for name, call in swa_calls(kdn, desc).items():
            assert call() == want, (over, name)
        assert kdn.lib().kdn_swa_fwd_workspace_bytes(ctypes.byref(desc)) == 0
        assert kdn.lib().kdn_swa_bwd_workspace_bytes(ctypes.byref(desc)) == 0
    for over, want in ((dict(T=-1), inv), (dict(T=2**21 + 1), uns), (dict(B=1024, T=2**21, H=4), uns)):
        desc = kdn.make_swa_desc(**{**base, **over})
        for name in ("fwd", "bwd", "fill"):
            assert swa_calls(kdn, desc)[name]() == want, (over, name)
    L = kdn.lib()
    assert L.kdn_swa_fwd(None, *[FAKE] * 7, 1 << 40, None) == inv
    assert L.kdn_swa_decode_step(None, *[FAKE] * 8) == inv


def test_attention_refuses_kv_heads_without_query_heads(kdn):
    """Their dk and dv (sums over no heads) and the cache would stay as they were."""
    desc = kdn.make_swa_desc(1, 8, 0, 2, 64, BF, window=4)
    for name, call in swa_calls(kdn, desc).items():
        assert call() == kdn.KDN_ERR_INVALID_ARG, name
    assert kdn.lib().kdn_swa_fwd_workspace_bytes(ctypes.byref(desc)) == 0
    assert kdn.lib().kdn_swa_bwd_workspace_bytes(ctypes.byref(desc)) == 0


def test_attention_refuses_bad_pointers_and_workspaces(kdn):
    desc = kdn.make_swa_desc(1, 8, 4, 2, 64, BF, window=4)
    required = {"fwd": (0, 1, 2, 4), "bwd": (0, 1, 2, 4, 5, 6, 7, 8, 9), "fill": (0, 1, 3, 4),
                "decode": range(7)}
    optional = {"fwd": (3, 5), "bwd": (3,), "fill": (2,), "decode": ()}
    for name, idx in required.items():
        for i in idx:
            for bad in (None, MIS):
                assert swa_calls(kdn, desc, i, bad)[name]() == kdn.KDN_ERR_INVALID_ARG, (name, i)
        for i in optional[name]:
            assert swa_calls(kdn, desc, i, MIS)[name]() == kdn.KDN_ERR_INVALID_ARG, (name, i)
    need = {"fwd": kdn.lib().kdn_swa_fwd_workspace_bytes(ctypes.byref(desc)),
            "bwd": kdn.lib().kdn_swa_bwd_workspace_bytes(ctypes.byref(desc))}
    for name, n in need.items():
        assert n >= 256
        for ws, m in ((None, 1 << 40), (MIS, 1 << 40), (FAKE, n - 1)):
            assert swa_calls(kdn, desc, ws=ws, ws_bytes=m)[name]() == kdn.KDN_ERR_WORKSPACE, name


@pytest.mark.parametrize("T,W,ns", [(65536, 128, 4), (65536, 128, 4096), (65536, 512, 4096), (8192, 128, 1024),
                                    (1 << 21, 1, 1 << 21), (1 << 21, 16, 4), (4096, 2048, 4), (3000, 64, 3000),
                                    (1777, 512, 16), (512, 2048, 0)])
def test_workspace_of_the_gradients_is_bounded(kdn, T, W, ns):
    """Two floats a query head and token, and at most 8 partial sums of 128 keys' dk and dv
    (64 keys' in float32) for each of 152 SMs: it does not grow with the sinks."""
    for B, H, Hk in ((1, 1, 1), (1, 16, 16), (8, 16, 2), (8, 16, 16), (1, 64, 1), (3, 40, 5)):
        for d, dtype, tile in ((128, BF, 128), (64, BF, 128), (32, F32, 64), (128, F32, 64)):
            desc = kdn.make_swa_desc(B, T, H, Hk, d, dtype, window=W, sinks=ns)
            n = kdn.lib().kdn_swa_bwd_workspace_bytes(ctypes.byref(desc))
            if B * H * T >= 1 << 31:
                assert n == 0
                continue
            rows = 256 + 2 * (4 * B * H * T + 255)
            assert 0 < n <= rows + 8 * 152 * 2 * tile * d * 4, (B, H, Hk, d, dtype)


def test_empty_problems_need_nothing(kdn):
    for B, T, H, Hk in ((0, 8, 4, 2), (1, 0, 4, 2), (1, 8, 0, 0)):
        desc = kdn.make_swa_desc(B, T, H, Hk, 64, BF, window=4)
        L, d = kdn.lib(), ctypes.byref(desc)
        assert L.kdn_swa_fwd(d, *[None] * 7, 0, None) == kdn.KDN_OK
        assert L.kdn_swa_bwd(d, *[None] * 11, 0, None) == kdn.KDN_OK
        assert L.kdn_swa_cache_fill(d, *[None] * 6) == kdn.KDN_OK
    assert kdn.lib().kdn_add_rmsnorm_fwd(ctypes.byref(kdn.kdn_norm_desc_t(0, 8, 1, 1, 0, 0.0)), *[None] * 8) == 0


def test_norm_refusals(kdn):
    L = kdn.lib()
    inv, uns = kdn.KDN_ERR_INVALID_ARG, kdn.KDN_ERR_UNSUPPORTED

    def fwd(rows=4, D=64, dtype=1, out=1, block=0, eps=1e-6, at=None, bad=None):
        d = kdn.kdn_norm_desc_t(rows, D, dtype, out, block, eps)
        return L.kdn_add_rmsnorm_fwd(ctypes.byref(d), *[bad if i == at else FAKE for i in range(7)], None)

    for over, want in ((dict(rows=-1), inv), (dict(D=0), inv), (dict(D=-8), inv), (dict(dtype=2), inv),
                       (dict(dtype=0, out=1), inv), (dict(out=3), inv), (dict(block=128), inv),
                       (dict(out=2, block=64), inv), (dict(eps=-1e-6), inv), (dict(eps=math.nan), inv),
                       (dict(eps=math.inf), inv), (dict(D=12), uns), (dict(D=16392), uns), (dict(rows=2**31), uns)):
        assert fwd(**over) == want, over
    for i in (0, 2, 3):
        assert fwd(at=i, bad=None) == inv
    for i in range(7):
        assert fwd(at=i, bad=MIS) == inv
    assert fwd(out=2, at=6, bad=None) == inv  # 8 bits need their scales

    def bwd(out=1, at=None, bad=None, ws=FAKE, n=1 << 40):
        d = kdn.kdn_norm_desc_t(4, 64, 1, out, 0, 0.0)
        return L.kdn_add_rmsnorm_bwd(ctypes.byref(d), *[bad if i == at else FAKE for i in range(7)], ws, n, None)

    assert bwd(out=2) == inv
    for i in (0, 1, 2, 3, 5, 6):
        assert bwd(at=i, bad=None) == inv and bwd(at=i, bad=MIS) == inv
    assert bwd(at=4, bad=MIS) == inv
    need = L.kdn_add_rmsnorm_bwd_workspace_bytes(ctypes.byref(kdn.kdn_norm_desc_t(4, 64, 1, 1, 0, 0.0)))
    for ws, n in ((None, 1 << 40), (MIS, 1 << 40), (FAKE, need - 1)):
        assert bwd(ws=ws, n=n) == kdn.KDN_ERR_WORKSPACE


# ------------------------------------------------------------------ the binding


class FakeLib:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        if name.endswith("_bytes"):
            return lambda *a: 4096

        def call(*args):
            self.calls.append(name)
            return 0
        return call


@pytest.fixture
def fake(monkeypatch):
    fake_tensor = pytest.importorskip("torch._subclasses.fake_tensor")
    import paper_2609_07816_gb300 as m
    L = FakeLib()
    monkeypatch.setattr(m, "lib", lambda: L)
    monkeypatch.setattr(m, "_ptr", lambda t: None)
    monkeypatch.setattr(m, "_stream", lambda s: None)
    with fake_tensor.FakeTensorMode(allow_non_fake_inputs=True):
        yield m, L


def E(*s, dtype=BF, dev="cuda"):
    return torch.empty(*s, dtype=dtype, device=dev)


def test_binding_reaches_the_library_and_refuses_bad_tensors(fake):
    m, L = fake
    I32 = torch.int32
    q, k, v, dO = E(2, 9, 6, 64), E(2, 9, 3, 64), E(2, 9, 3, 64), E(2, 9, 6, 64)
    lens = E(2, dtype=I32)
    o, lse = m.kdn_swa_fwd(q, k, v, window=4, sinks=2, lens=lens)
    assert o.shape == q.shape and lse.shape == (2, 6, 9)
    G = m.kdn_swa_bwd(q, k, v, o, lse, dO, window=4, sinks=2, lens=lens)
    assert G["dk"].shape == k.shape
    kc, vc = E(2, 3, 6, 64), E(2, 3, 6, 64)
    m.kdn_swa_cache_fill(k, v, kc, vc, window=4, sinks=2)
    q1, k1, v1, pos = E(2, 6, 64), E(2, 3, 64), E(2, 3, 64), E(2, dtype=I32)
    m.kdn_swa_decode_step(q1, k1, v1, kc, vc, pos, window=4, sinks=2)
    x, w, r = E(5, 7, 64), E(64), E(5, 7, 64)
    y, h, rstd, s = m.kdn_add_rmsnorm_fwd(x, w, r, out_dtype=torch.float8_e4m3fn, block=128)
    assert s.shape == (5, 7, 1) and rstd.shape == (5, 7)
    m.kdn_add_rmsnorm_bwd(h, w, rstd, x, r)
    assert L.calls == ["kdn_swa_fwd", "kdn_swa_bwd", "kdn_swa_cache_fill", "kdn_swa_decode_step",
                       "kdn_add_rmsnorm_fwd", "kdn_add_rmsnorm_bwd"]
    L.calls.clear()
    t = lambda a: a.transpose(1, 2)
    bad = [
        lambda: m.kdn_swa_fwd(E(2, 9, 6, 64, dev="cpu"), k, v, window=4),
        lambda: m.kdn_swa_fwd(q.half(), k, v, window=4),
        lambda: m.kdn_swa_fwd(q, k.float(), v, window=4),
        lambda: m.kdn_swa_fwd(t(E(2, 6, 9, 64)), k, v, window=4),
        lambda: m.kdn_swa_fwd(q, E(2, 8, 3, 64), E(2, 8, 3, 64), window=4),
        lambda: m.kdn_swa_fwd(q, k, E(2, 9, 2, 64), window=4),
        lambda: m.kdn_swa_fwd(q, k, E(2, 9, 3, 32), window=4),
        lambda: m.kdn_swa_fwd(q[0], k[0], v[0], window=4),
        lambda: m.kdn_swa_fwd(q, k, v, window=4, lens=E(2, dtype=torch.int64)),
        lambda: m.kdn_swa_fwd(q, k, v, window=4, lens=E(3, dtype=I32)),
        lambda: m.kdn_swa_fwd(q, k, v, window=4, o=E(2, 9, 6, 64, dtype=F32)),
        lambda: m.kdn_swa_fwd(q, k, v, window=4, lse=E(2, 9, 5, dtype=F32)),
        lambda: m.kdn_swa_bwd(q, k, v, o, None, dO, window=4),
        lambda: m.kdn_swa_bwd(q, k, v, o, lse, dO.float(), window=4),
        lambda: m.kdn_swa_bwd(q, k, v, o, lse, dO, window=4, grads={"dq": q, "dk": k}),
        lambda: m.kdn_swa_cache_fill(k, v, kc, vc, window=5, sinks=2),
        lambda: m.kdn_swa_cache_fill(k, v, kc, E(2, 3, 6, 64, dtype=F32), window=4, sinks=2),
        lambda: m.kdn_swa_decode_step(q1, k1, v1, kc, vc, pos, window=4, sinks=1),
        lambda: m.kdn_swa_decode_step(q1, k1, v1, kc, vc, E(2, dtype=torch.int64), window=4, sinks=2),
        lambda: m.kdn_swa_decode_step(q, k, v, kc, vc, pos, window=4, sinks=2),
        lambda: m.kdn_add_rmsnorm_fwd(x, w.float(), r),
        lambda: m.kdn_add_rmsnorm_fwd(x, E(63), r),
        lambda: m.kdn_add_rmsnorm_fwd(x, w, E(5, 6, 64)),
        lambda: m.kdn_add_rmsnorm_fwd(x, w, r, out_dtype=F32),
        lambda: m.kdn_add_rmsnorm_fwd(t(x), w, None),
        lambda: m.kdn_add_rmsnorm_bwd(h, w, None, x),
        lambda: m.kdn_add_rmsnorm_bwd(h, w, rstd, x, dw=E(64)),
    ]
    for i, call in enumerate(bad):
        with pytest.raises((ValueError, TypeError)):
            call()
        assert not L.calls, i


def test_reference_gradients_are_the_differences():
    g = torch.Generator().manual_seed(1)
    q, k, v, dO = (torch.randn(2, 23, h, 8, generator=g, dtype=torch.float64) for h in (4, 2, 2, 4))
    lens = torch.tensor([23, 9])
    R = ref.attention(q, k, v, 5, 2, lens, None, dO)
    for n, x in (("dq", 0), ("dk", 1), ("dv", 2)):
        t = torch.randn(*(q, k, v)[x].shape, generator=g, dtype=torch.float64)

        def loss(e):
            a = [y + e * t if i == x else y for i, y in enumerate((q, k, v))]
            return float((ref.attention(*a, 5, 2, lens)["o"] * dO).sum())
        # truncation e^2 and rounding 1e-15 / e at e = 1e-5
        assert abs((loss(1e-5) - loss(-1e-5)) / 2e-5 - float((R[n] * t).sum())) <= 1e-7
