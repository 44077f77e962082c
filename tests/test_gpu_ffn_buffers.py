"""The feed-forward block's tensors side by side in one allocation, as a program that packs its weights and
gradients keeps them: nothing is shared, and nothing is refused."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [1, 40, 300])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_tensors_that_touch(rows, dtype):
    import paper_2609_07816_gb300 as kdn
    D, F = 64, 136
    shapes = [("x", (rows, D)), ("wg", (F, D)), ("wu", (F, D)), ("wd", (D, F)), ("dy", (rows, D)), ("g", (rows, F)),
              ("u", (rows, F)), ("h", (rows, F)), ("y", (rows, D)), ("dx", (rows, D)), ("dwg", (F, D)), ("dwu", (F, D)),
              ("dwd", (D, F))]
    block = torch.zeros(sum(a * b for _, (a, b) in shapes), dtype=dtype, device="cuda")
    t, at = {}, 0
    for n, (a, b) in shapes:
        t[n] = block[at:at + a * b].view(a, b)
        at += a * b
    gen = torch.Generator(device="cuda").manual_seed(1)
    ins = ("x", "wg", "wu", "wd", "dy")
    for n in ins:
        t[n].copy_(torch.randn(*t[n].shape, generator=gen, device="cuda") * 0.2)
    apart = [t[n].clone() for n in ins]
    y, g, u, h = kdn.kdn_ffn_fwd(*apart[:4])
    want = {"y": y, "g": g, "u": u, "h": h, **kdn.kdn_ffn_bwd(*apart[:4], g, u, h, apart[4])}
    kdn.kdn_ffn_fwd(*[t[n] for n in ins[:4]], g=t["g"], u=t["u"], h=t["h"], y=t["y"])
    kdn.kdn_ffn_bwd(*[t[n] for n in ins[:4]], t["g"], t["u"], t["h"], t["dy"],
                    grads={n: t[n] for n in ("dx", "dwg", "dwu", "dwd")})
    assert all(torch.equal(t[n], w) for n, w in want.items())
    assert all(torch.equal(t[n], w) for n, w in zip(ins, apart))
    # refused: what would be written over what is still read
    kw = {n: t[n] for n in ("dwg", "dwu", "dwd")}
    for dx in (t["x"], t["dy"]):
        with pytest.raises(kdn.KdnError) as e:
            kdn.kdn_ffn_bwd(*[t[n] for n in ins[:4]], t["g"], t["u"], t["h"], t["dy"], grads={"dx": dx, **kw})
        assert e.value.status == kdn.KDN_ERR_INVALID_ARG
    assert all(torch.equal(t[n], w) for n, w in zip(ins, apart))
