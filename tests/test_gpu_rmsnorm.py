"""Residual RMS norm on the GPU against its 64-bit definition.

Bounds: a stored bfloat16 is within 2^-9 of its value (2^-8 taken), float32 sums over
D columns within 8 sqrt(D) 2^-24 of the sum of magnitudes, as random rounding errors.
An 8-bit value is the nearest e4m3 number to y / scale, a step of at most 2^-3 of it
(2^-9 below the normal range), so it is within half a step, plus the float32 error
that may move a tie."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

BF, F32, F8 = torch.bfloat16, torch.float32, torch.float8_e4m3fn
EPS = 1e-6


@pytest.fixture(scope="module")
def kdn():
    import paper_2609_07816_gb300 as m
    m.lib()
    return m


def rand(seed, *shapes, dtype=BF, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [(torch.randn(*s, generator=g, device="cuda") * scale).to(dtype) for s in shapes]


def within(name, got, want, bound):
    over = (got.double() - want).abs() - bound
    assert torch.isfinite(got.double()).all(), name
    assert float(over.max()) <= 0, f"{name}: over its bound by {float(over.max()):.3e}"


def define(x, w, res):
    h = x.double() + (0 if res is None else res.double())
    rstd = (h.square().mean(-1, keepdim=True) + EPS).rsqrt()
    return h, rstd, h * rstd * w.double()


ROWS_D = [(1, 8), (1, 2304), (3, 256), (5, 264), (9, 512), (7, 520), (8, 1024), (17, 1032), (2, 2048), (33, 2056),
          (4, 4096), (3, 4104), (2, 8192), (5, 8200), (2, 16384), (700, 128), (1000, 2304)]


@pytest.mark.parametrize("rows,D", ROWS_D)
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("residual", [True, False])
def test_forward_and_gradients(kdn, rows, D, dtype, residual):
    x, r, dy, dh = rand(rows + D, *[(rows, D)] * 4, dtype=dtype)
    w, = rand(D, (D,), dtype=dtype)
    res = r if residual else None
    y, h, rstd, scales = kdn.kdn_add_rmsnorm_fwd(x, w, res, eps=EPS)
    H, R, Y = define(x, w, res)
    u = 2.0 ** -8 if dtype == BF else 2.0 ** -22
    s32 = 8 * math.sqrt(D) * 2.0 ** -24
    assert scales is None
    within("h", h, H, u * H.abs())
    within("rstd", rstd[:, None], R, (s32 + 2.0 ** -22) * R)
    within("y", y, Y, (u + s32) * Y.abs())
    # the gradients are those at the stored h, with the forward's rstd
    dx, dw = kdn.kdn_add_rmsnorm_bwd(h, w, rstd, dy, dh if residual else None)
    xh, g = h.double() * rstd.double()[:, None], dy.double() * w.double()
    mean = (g * xh).mean(-1, keepdim=True)
    want = rstd.double()[:, None] * (g - xh * mean) + (dh.double() if residual else 0)
    e = u * want.abs() + (s32 + 2.0 ** -20) * (rstd.double()[:, None] * (
        g.abs() + xh.abs() * (g * xh).abs().mean(-1, keepdim=True)) + (dh.double().abs() if residual else 0))
    within("dx", dx, want, e)
    terms = dy.double() * xh
    within("dw", dw, terms.sum(0), (8 * math.sqrt(rows) * 2.0 ** -24 + 2.0 ** -20) * terms.abs().sum(0))


@pytest.mark.parametrize("rows,D", ROWS_D)
@pytest.mark.parametrize("block", [0, 128])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_eight_bit_output(kdn, rows, D, block, dtype):
    x, res = rand(rows + D, *[(rows, D)] * 2, dtype=dtype)
    w, = rand(D, (D,), dtype=dtype)
    y, h, rstd, scales = kdn.kdn_add_rmsnorm_fwd(x, w, res, eps=EPS, out_dtype=F8, block=block)
    H, R, Y = define(x, w, res)
    b = block or D
    nb = -(-D // b)
    assert y.dtype == F8 and tuple(scales.shape) == (rows, nb)
    amax = torch.nn.functional.pad(Y.abs(), (0, nb * b - D)).view(rows, nb, b).amax(-1)
    s32 = 8 * math.sqrt(D) * 2.0 ** -24 + 2.0 ** -20
    within("scales", scales, amax / 448, s32 * amax / 448)
    wide = scales.double().repeat_interleave(b, 1)[:, :D]
    z = Y / wide
    step = torch.exp2(torch.floor(torch.log2(z.abs().clamp_min(2.0 ** -6))) - 3)
    within("q", y.double(), z, step / 2 + s32 * z.abs())
    assert float(y.double().abs().max()) <= 448


def test_eight_bit_special_rows(kdn):
    """All-zero rows and blocks have scale 1; a row with a NaN or an infinity is NaN where
    its norm is, and leaves the other rows alone."""
    D = 384
    x, = rand(1, (6, D))
    w, = rand(2, (D,))
    x[1] = 0
    x[2, 128:256] = 0
    x[3, 7] = math.nan
    x[4, 200] = math.inf
    for block in (0, 128):
        y, _, _, s = kdn.kdn_add_rmsnorm_fwd(x, w, out_dtype=F8, block=block)
        y = y.float()
        assert not y[1].any() and (s[1] == 1).all()
        assert y[3].isnan().all() and y[4, 200].isnan()
        assert torch.isfinite(y[[0, 1, 2, 5]]).all() and torch.isfinite(s).all()
        if block:
            assert s[2, 1] == 1 and not y[2, 128:256].any()
        alone = kdn.kdn_add_rmsnorm_fwd(x[5:].clone(), w, out_dtype=F8, block=block)
        assert torch.equal(alone[0].float()[0], y[5]) and torch.equal(alone[3][0], s[5])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("block", [0, 128])
@pytest.mark.parametrize("size", [1e-30, 1e-35, 1e-36, 1e-37, 2e-38, 1e-39, 1e-40, 3e-43, 3e-45])
def test_eight_bit_tiny_blocks(kdn, dtype, block, size):
    """Blocks whose largest magnitude is far below one, zeros among their elements: the scale
    is positive and y is q * scale as everywhere else.  Below float32's normal range each
    product of y = h (rstd w) is off by up to 2^-150, and the scale by 2^-149."""
    D, rows = 384, 5
    x, = rand(11, (rows, D), dtype=dtype)
    x[:, 3::7] = 0
    w = (rand(12, (D,), dtype=F32)[0] * size).to(dtype)
    if block:
        w[128:256], = rand(13, (128,), dtype=dtype)  # the block between them is of order one
    y, _, _, scales = kdn.kdn_add_rmsnorm_fwd(x, w, eps=EPS, out_dtype=F8, block=block)
    H, R, Y = define(x, w, None)
    b = block or D
    s32, tiny = 8 * math.sqrt(D) * 2.0 ** -24 + 2.0 ** -20, 2.0 ** -150 * (H.abs() + 1)
    amax = Y.abs().view(rows, D // b, b).amax(-1)
    assert torch.equal(scales == 1, amax == 0)
    within("scales", torch.where(amax > 0, scales, 0), amax / 448,
           s32 * amax / 448 + 2.0 ** -149 + float(tiny.max()) / 448)
    assert (scales > 0).all()
    wide = scales.double().repeat_interleave(b, 1)
    z = Y / wide
    step = torch.exp2(torch.floor(torch.log2(z.abs().clamp_min(2.0 ** -6))) - 3)
    within("q", y.double(), z, step / 2 + s32 * z.abs() + tiny / wide)
    assert float(y.double().abs().max()) <= 448 and not y.float()[Y == 0].any()


def test_in_place_shapes_streams_and_bits(kdn):
    x, res, dy, dh = rand(3, *[(2, 37, 2304)] * 4)
    w, = rand(4, (2304,))
    y, h, rstd, _ = kdn.kdn_add_rmsnorm_fwd(x, w, res)
    assert y.shape == x.shape and rstd.shape == (2, 37)
    r2 = res.clone()
    y2, h2, _, _ = kdn.kdn_add_rmsnorm_fwd(x, w, r2, h=r2)
    assert torch.equal(y, y2) and torch.equal(h, r2) and h2 is r2
    dx, dw = kdn.kdn_add_rmsnorm_bwd(h, w, rstd, dy, dh)
    for n in range(2):  # dx in the place of dy, then of dh
        io = [dy.clone(), dh.clone()]
        dx2, dw2 = kdn.kdn_add_rmsnorm_bwd(h, w, rstd, *io, dx=io[n])
        assert dx2 is io[n] and torch.equal(dx, dx2) and torch.equal(dw, dw2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y3 = kdn.kdn_add_rmsnorm_fwd(x, w, res, stream=side)[0]
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(y, y3)


def test_no_rows(kdn):
    x = torch.empty(0, 64, dtype=BF, device="cuda")
    w = torch.ones(64, dtype=BF, device="cuda")
    y, h, rstd, _ = kdn.kdn_add_rmsnorm_fwd(x, w, x.clone())
    dx, dw = kdn.kdn_add_rmsnorm_bwd(h, w, rstd, y)
    assert dx.numel() == 0 and not dw.any()


def test_gradient_against_differences(kdn):
    """Central differences of the float32 forward along random directions, e = 2^-8: the
    rounding of N = 1200 terms near one costs 2^-24 sqrt(N) / (2 e) = 3e-4, the third
    derivative (about 200 along a direction of the rows' own length) e^2 / 6 of it, 5e-4."""
    n, D = 6, 200
    x, dy, d1 = rand(7, *[(n, D)] * 3, dtype=F32)
    w, d2 = rand(8, (D,), (D,), dtype=F32)
    _, h, rstd, _ = kdn.kdn_add_rmsnorm_fwd(x, w)
    dx, dw = kdn.kdn_add_rmsnorm_bwd(h, w, rstd, dy)
    e = 2.0 ** -8

    def loss(a, b):
        return float((kdn.kdn_add_rmsnorm_fwd(a, b)[0].double() * dy.double()).sum())

    gx = (loss(x + e * d1, w) - loss(x - e * d1, w)) / (2 * e)
    gw = (loss(x, w + e * d2) - loss(x, w - e * d2)) / (2 * e)
    assert abs(gx - float((dx.double() * d1.double()).sum())) <= 1e-2
    assert abs(gw - float((dw.double() * d2.double()).sum())) <= 1e-2
