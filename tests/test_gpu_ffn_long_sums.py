"""Long sums of the feed-forward block in bfloat16: of positive terms, where what an accumulator loses
adds up.

The tensor cores truncate, at most 2^-23 of an accumulator for every 16 terms.  A float32 output's sum leaves the
accumulator every 512 terms (32 additions: 2^-18 of them) and goes on in float32, rounded to nearest: n / 512 additions,
8 sqrt(n / 512) 2^-24 as random errors.  A bfloat16 output's sum takes at most 65536 terms into one accumulator (4096
additions: 2^-11 of it); a longer one leaves it every 4096 (2^-15).  Then it is rounded once, half a step of 2^-8."""
import math

import pytest
import torch

import ffn_ref as ref
from test_gpu_ffn import check, kdn  # noqa: F401

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


def positive(rows, D, F):
    """x, wg, wu, wd, g, u, h, dy: tokens and hidden values in [0, 1), weights that give no other gradients."""
    gen = torch.Generator(device="cuda").manual_seed(rows)
    r = lambda *s: torch.rand(*s, generator=gen, device="cuda").to(BF)
    z = lambda *s: torch.zeros(*s, dtype=BF, device="cuda")
    h = r(rows, F)
    return z(rows, D), z(F, D), z(F, D), z(D, F), h, h, h, r(rows, D)


def sums(dy, h, cols):
    """dy^T h of the first columns of dy, in 64 bits."""
    want = torch.zeros(cols, h.shape[1], dtype=torch.float64, device="cuda")
    for i in range(0, h.shape[0], 8192):
        want += dy[i:i + 8192, :cols].double().T @ h[i:i + 8192].double()
    return want


@pytest.mark.parametrize("rows,D,F", [(129, 64, 72), (511, 264, 520), (513, 72, 136), (577, 2048, 1032), (777, 64, 256),
                                      (1025, 520, 264), (4104, 1032, 520), (32768, 2048, 4096), (65537, 1024, 2048)])
def test_float32_gradients_of_weights(kdn, rows, D, F):  # noqa: F811
    *a, dy = positive(rows, D, F)
    got = kdn.kdn_ffn_bwd(*a, dy, dw_dtype=F32)["dwd"]
    want = sums(dy, a[-1], min(D, 64))
    tol = 2.0 ** -18 + 8 * math.sqrt(rows / 512 + 1) * 2.0 ** -24
    assert float(((got[:want.shape[0]].double() - want).abs() / want).max()) <= tol


# (sums in several parts and, of the last two, in one)
@pytest.mark.parametrize("rows,D,F", [(131080, 1024, 4096), (300000, 1024, 4096), (131080, 1280, 1280), (70000, 768, 2048)])
def test_bfloat16_gradients_of_many_rows(kdn, rows, D, F):  # noqa: F811
    """A sum that is off by no more than `lost` rounds to what lies between its ends' roundings, since rounding
    keeps the order; one that is off by more passes a boundary somewhere among 81920 elements or more."""
    *a, dy = positive(rows, D, F)
    got = kdn.kdn_ffn_bwd(*a, dy)["dwd"][:64]
    want = sums(dy, a[-1], 64)
    lost = 2.0 ** -15 + 8 * math.sqrt(rows / 4096) * 2.0 ** -24
    assert bool((got >= (want * (1 - lost)).to(BF)).all()) and bool((got <= (want * (1 + lost)).to(BF)).all())


@pytest.mark.parametrize("rows,D,F", [(40, 8, 65544), (200, 16, 131080), (130, 24, 40000)])
def test_long_hidden_axis(kdn, rows, D, F):  # noqa: F811
    """y and dx, sums over the hidden axis (dx over twice its length), of positive terms."""
    gen = torch.Generator(device="cuda").manual_seed(F)
    r = lambda *s: torch.rand(*s, generator=gen, device="cuda").to(BF)
    x, wg, wu, wd = r(rows, D), r(F, D) / D, r(F, D) / D, r(D, F) / 256
    y, g, u, h = kdn.kdn_ffn_fwd(x, wg, wu, wd)
    Y = h.double() @ wd.double().T
    # (h, dg and du are operands as stored; parts of a sum are joined in float32)
    lost = 2.0 ** -11
    e = (y.double() - Y) / Y
    assert float(e.abs().max()) <= 2.0 ** -8 + lost
    dy = r(rows, D)
    got = kdn.kdn_ffn_bwd(x, wg, wu, wd, g, u, h, dy)["dx"]
    want = ref.backward(x, wg, wu, wd, g, u, h, dy, "silu")["dx"]
    # dg and du: a short sum's loss and a rounding each, all terms positive
    assert float(((got.double() - want) / want).abs().max()) <= 2 * 2.0 ** -8 + lost + 2.0 ** -16


@pytest.mark.parametrize("rows,D,F", [(512, 264, 520), (1537, 64, 128), (2100, 328, 200)])
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_float32_gradients_between_chunks(kdn, rows, D, F, act):  # noqa: F811
    check(kdn, rows, D, F, BF, act, dw_dtype=F32)
