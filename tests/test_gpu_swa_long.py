"""Attention over long sequences with a narrow window, and over many sinks: key tiles whose
queries are split over CTAs in lists of every length, against the 64-bit definition; and the
strips' definition against the plain one."""
import ctypes

import pytest
import torch

import swa_ref as ref
import swa_strips as strips

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def kdn():
    import paper_2609_07816_gb300 as m
    m.lib()
    return m


def rand(seed, *shapes, dtype=BF):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randn(*s, generator=g, device="cuda").to(dtype) for s in shapes]


def run(kdn, q, k, v, dO, W, ns, lens=None):
    desc = kdn.make_swa_desc(*q.shape[:3], k.shape[2], q.shape[3], q.dtype, window=W, sinks=ns)
    ws = torch.full((kdn.lib().kdn_swa_bwd_workspace_bytes(ctypes.byref(desc)),), 255, dtype=torch.uint8, device="cuda")
    kw = dict(window=W, sinks=ns, lens=lens, workspace=ws)
    o, lse = kdn.kdn_swa_fwd(q, k, v, **kw)
    assert kdn.kdn_get_device_status(ws) == kdn.KDN_OK
    G = kdn.kdn_swa_bwd(q, k, v, o, lse, dO, **kw)
    assert kdn.kdn_get_device_status(ws) == kdn.KDN_OK
    return {"o": o, "lse": lse, **G}


def check(got, b, hk, G, n, R):
    """Kv head hk of sequence b and its query heads, n tokens of them."""
    H = slice(hk * G, hk * G + G)
    for x in ("o", "dq"):
        ref.check(x, got[x][b, :n, H], R[x], R["e" + x])
    ref.check("lse", got["lse"][b, H, :n], R["lse"], R["else"])
    for x in ("dk", "dv"):
        ref.check(x, got[x][b, :n, hk], R[x], R["e" + x])


def test_strips_are_the_definition():
    """Values to 64-bit rounding; bounds never wider than the plain definition's (a strip's
    largest score and number of keys are at most the sequence's)."""
    for dtype in (BF, F32):
        q, k, v, dO = rand(1, (1, 700, 4, 64), (1, 700, 2, 64), (1, 700, 2, 64), (1, 700, 4, 64), dtype=dtype)
        for W, ns in ((50, 3), (300, 0), (7, 400), (1000, 5)):
            want = ref.attention(q, k, v, W, ns, dO=dO)
            for hk in range(2):
                H = slice(2 * hk, 2 * hk + 2)
                got = strips.group(q[0, :, H], k[0, :, hk], v[0, :, hk], dO[0, :, H], W, ns)
                for n, w in [(n, want[n][0, :, H]) for n in ("o", "dq")] + [(n, want[n][0, :, hk]) for n in ("dk", "dv")]:
                    assert (got[n] - w).abs().max() <= 1e-12 * w.abs().max(), n
                    e = want["e" + n][0, :, H if n in ("o", "dq") else hk]
                    assert (got["e" + n] > 0).all() and (got["e" + n] <= e * (1 + 1e-12)).all(), n


# (B, T, H, Hk, W, ns): lists of a sink tile cut into parts of 3, 5, 7 and 17 query tiles, and
# not at all although they are far longer than the others'; ends that are no whole tiles
SPLITS = [(1, 8200, 4, 4, 128, 4), (1, 5000, 8, 8, 100, 200), (2, 9001, 8, 8, 60, 16), (1, 30011, 16, 16, 128, 4),
          (6, 2100, 16, 16, 40, 500), (2, 4000, 16, 4, 30, 300)]


@pytest.mark.parametrize("B,T,H,Hk,W,ns", SPLITS)
@pytest.mark.parametrize("d,dtype", [(128, BF), (64, BF), (32, F32)])
def test_splits_of_the_sinks_tiles(kdn, B, T, H, Hk, W, ns, d, dtype):
    G = H // Hk
    q, k, v, dO = rand(T + W, (B, T, H, d), (B, T, Hk, d), (B, T, Hk, d), (B, T, H, d), dtype=dtype)
    lens = None if B == 1 else torch.tensor([T, T - 333] + [T // (b + 1) for b in range(B - 2)], dtype=torch.int32,
                                            device="cuda")
    got = run(kdn, q, k, v, dO, W, ns, lens)
    again = run(kdn, q, k, v, dO, W, ns, lens)
    assert all(torch.equal(got[n], again[n]) for n in got)
    for b, hk in {(0, 0), (0, Hk - 1), (B - 1, Hk // 2), (B // 2, 1 % Hk)}:
        n = T if lens is None else int(lens[b])
        H_ = slice(hk * G, hk * G + G)
        check(got, b, hk, G, n, strips.group(q[b, :n, H_], k[b, :n, hk], v[b, :n, hk], dO[b, :n, H_], W, ns))
