"""Tensors of more than 2^31 elements: the attention's forward, gradients and cache, and the
norm, at the first and the last rows, whose offsets lie past 32 bits.  What lies between holds
zeros, and its results are zeros."""
import math

import pytest
import torch

import swa_ref as ref
import swa_strips as strips
from test_gpu_swa import fill_ref
from test_gpu_swa_long import check

pytestmark = pytest.mark.gpu

BF, F32, F8 = torch.bfloat16, torch.float32, torch.float8_e4m3fn


@pytest.fixture(scope="module")
def kdn():
    import paper_2609_07816_gb300 as m
    m.lib()
    yield m
    torch.cuda.empty_cache()


def ends(seed, n, rest, dtype, count):
    """`count` tensors [n, *rest] with random first and last entries and zeros between."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    out = []
    for _ in range(count):
        x = torch.zeros(n, *rest, dtype=dtype, device="cuda")
        for b in (0, n - 1):
            x[b] = torch.randn(*rest, generator=g, device="cuda").to(dtype)
        out.append(x)
    return out


@pytest.mark.parametrize("dtype", [BF, F32])
def test_attention(kdn, dtype):
    B, T, H, d, W, ns = 65, 4096, 64, 128, 100, 5
    assert B * T * H * d > 2 ** 31
    q, k, v, dO = ends(1, B, (T, H, d), dtype, 4)
    at = dict(window=W, sinks=ns)
    o, lse = kdn.kdn_swa_fwd(q, k, v, **at)
    got = {"o": o, "lse": lse, **kdn.kdn_swa_bwd(q, k, v, o, lse, dO, **at)}
    for b, h in ((0, 0), (0, H - 1), (B - 1, 0), (B - 1, H - 1)):
        one = slice(h, h + 1)
        check(got, b, h, 1, T, strips.group(q[b, :, one], k[b, :, h], v[b, :, h], dO[b, :, one], W, ns))
    for n in ("o", "dq", "dk", "dv"):
        assert not any(bool(got[n][b].any()) for b in range(1, B - 1))
    del got, o, lse, q, dO
    kc, vc = (torch.full((B, H, W + ns, d), math.nan, dtype=dtype, device="cuda") for _ in range(2))
    kdn.kdn_swa_cache_fill(k, v, kc, vc, **at)
    for b in (0, B - 1):
        x, y = torch.empty_like(kc[:1]), torch.empty_like(vc[:1])
        fill_ref(k[b:b + 1], v[b:b + 1], x, y, W, ns, [T])
        assert torch.equal(kc[b:b + 1], x) and torch.equal(vc[b:b + 1], y)
    assert not any(bool(kc[b].any()) for b in range(1, B - 1))


def test_norm(kdn):
    rows, D, eps = 1_100_003, 2048, 1e-6
    assert rows * D > 2 ** 31
    x, res, dy, dh = ends(2, rows, (D,), BF, 4)
    w = torch.randn(D, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda").to(BF)
    y, h, rstd, _ = kdn.kdn_add_rmsnorm_fwd(x, w, res, eps=eps)
    dx, dw = kdn.kdn_add_rmsnorm_bwd(h, w, rstd, dy, dh)
    pick = torch.tensor([0, rows - 1], device="cuda")
    X = lambda t: t[pick].double()
    # a stored bfloat16 within 2^-8, float32 sums over a row within 2^-16 of their magnitudes
    H = X(x) + X(res)
    R = (H.square().mean(1, keepdim=True) + eps).rsqrt()
    Y = H * R * w.double()
    assert ((X(y) - Y).abs() <= (2.0 ** -8 + 2.0 ** -16) * Y.abs()).all()
    xh, g = X(h) * X(rstd)[:, None], X(dy) * w.double()
    want = R * (g - xh * (g * xh).mean(1, keepdim=True)) + X(dh)
    assert ((X(dx) - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -16 * (R * (g.abs() + xh.abs() * (
        g * xh).abs().mean(1, keepdim=True)) + X(dh).abs())).all()
    terms = X(dy) * xh
    assert ((dw.double() - terms.sum(0)).abs() <= 2.0 ** -16 * terms.abs().sum(0)).all()
    assert not y[1:-1].any() and not dx[1:-1].any()
    del dx, dy, dh, y
    y, _, _, scales = kdn.kdn_add_rmsnorm_fwd(x, w, res, eps=eps, out_dtype=F8, block=128)
    amax = Y.abs().view(2, D // 128, 128).amax(-1)
    assert ((X(scales) - amax / 448).abs() <= 2.0 ** -16 * amax).all() and (scales[1:-1] == 1).all()
    z = Y / X(scales).repeat_interleave(128, 1)
    step = torch.exp2(torch.floor(torch.log2(z.abs().clamp_min(2.0 ** -6))) - 3)
    assert ((X(y.float()) - z).abs() <= step / 2 + 2.0 ** -16 * z.abs()).all()
