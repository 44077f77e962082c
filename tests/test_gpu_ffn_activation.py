"""The feed-forward block's activation in float32, value by value over the whole range where it is
neither 0 nor its argument, in the kernels of few and of many tokens.

With s = 1 / (1 + e^-z) the exponential is within 2^-22 of its value (its argument is carried in two parts, so that a
large one costs nothing) and six further roundings of 2^-24 or less lie on the way to act(g) u: 2^-20 of the value
together.  The derivative is the sum of s and act(g) (1 - s) dz/dg, each within twice that.  Where e^-|z| is no normal
float32 it is taken as 0: s or 1 - s, either below 2^-126, is lost, and with it up to 2^-126 of 1, |g| and
|g| dz/dg."""
import pytest
import torch

pytestmark = pytest.mark.gpu

F32, N = torch.float32, 64
ACT = {"silu": 0, "gelu": 1}


def values(rows, act):
    """rows x N arguments of the activation: evenly over all that matters, and at random around 0."""
    far = 90.0 if act == "silu" else 10.5
    g = torch.linspace(-far, far, rows * N, dtype=torch.float64).reshape(N, rows).T
    gen = torch.Generator().manual_seed(rows)
    g[:, ::4] = torch.randn(rows, N // 4, generator=gen, dtype=torch.float64) * 3
    return g.float().contiguous().cuda()


def terms(act, g):
    """act(g), its derivative, the sizes of the derivative's two terms, and dz/dg, in 64 bits and without
    cancellation in either tail."""
    k = 2 * (2 / torch.pi) ** 0.5
    z, dz = (g, 1.0) if act == "silu" else (k * (g + 0.044715 * g ** 3), k * (1 + 3 * 0.044715 * g * g))
    s = torch.sigmoid(z)
    a, rest = g * s, g * s * torch.sigmoid(-z) * dz
    return a, s + rest, s, rest.abs(), dz


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("rows", [1, 3, 8, 16, 40, 300])
def test_value_by_value(act, rows):
    import paper_2609_07816_gb300 as kdn
    g = values(rows, act)
    eye, zero, one = torch.eye(N, device="cuda"), torch.zeros(N, N, device="cuda"), torch.ones(N, N, device="cuda")
    tiny = 2.0 ** -126
    size = 1 + g.double().abs()
    # forward: g = x, and u = 1 from a channel of ones behind it
    x = torch.cat([g, torch.ones(rows, 8, device="cuda")], 1)
    wg, wu = torch.cat([eye, zero[:, :8]], 1), torch.cat([zero, one[:, :8] / 8], 1)
    _, G, U, h = kdn.kdn_ffn_fwd(x, wg, wu, torch.zeros(N + 8, N, device="cuda"), act=ACT[act])
    assert torch.equal(G, g) and bool((U == 1).all())
    a, da, s, rest, dz = terms(act, g.double())
    over = (h.double() - a).abs() - (2.0 ** -20 * a.abs() + tiny * size)
    assert float(over.max()) <= 0, f"act: {float(over.max()):.2e} at {float(g.flatten()[over.argmax()]):.4f}"
    # backward: dh = 1, so that dx is dg or du with the other's weights 0
    dy, wd = torch.zeros(rows, N, device="cuda"), torch.zeros_like(zero)
    dy[:, 0], wd[0] = 1, 1
    ones = torch.ones_like(g)
    dg = kdn.kdn_ffn_bwd(dy, eye, zero, wd, g, ones, ones, dy, act=ACT[act])["dx"]
    over = (dg.double() - da).abs() - (2.0 ** -19 * (s + rest) + tiny * size * (1 + dz))
    assert float(over.max()) <= 0, f"dg: {float(over.max()):.2e} at {float(g.flatten()[over.argmax()]):.4f}"
    du = kdn.kdn_ffn_bwd(dy, zero, eye, wd, g, ones, ones, dy, act=ACT[act])["dx"]
    over = (du.double() - a).abs() - (2.0 ** -20 * a.abs() + tiny * size)
    assert float(over.max()) <= 0, f"du: {float(over.max()):.2e} at {float(g.flatten()[over.argmax()]):.4f}"
