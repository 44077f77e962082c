"""A hybrid pair of layers as a model would hold them: a Diagonal KDN mixer, then
sliding-window attention with sinks, each behind the residual RMS norm.

    h = x + res;  y = norm(h) w;  x' = mixer(y Wq, y Wk, ...) Wo;  res' = h

`prefill` runs a padded batch of prompts and leaves what decode continues from (the KDN
memory and uncertainty, and the attention's bounded cache: both of a size that does not
grow with the context), `decode` one token of every sequence, and `gradients` a training
pass.  Projections are plain matrix products; everything else is the library's.

    python examples/hybrid_layer.py        # prefill, decode and gradients, checked
"""
import os
import sys

import torch
import torch.nn.functional as F

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_2609_07816_gb300 as kdn  # noqa: E402

BF = torch.bfloat16


class Hybrid:
    """Weights of the pair: H heads of d for the mixer; H query and Hk kv heads for the attention."""

    def __init__(self, H=4, Hk=2, d=128, window=64, sinks=4, seed=0):
        self.H, self.Hk, self.d, self.window, self.sinks = H, Hk, d, window, sinks
        D = self.D = H * d
        g = torch.Generator(device="cuda").manual_seed(seed)

        def w(*shape, scale=None):
            x = torch.randn(*shape, generator=g, device="cuda") * (scale or shape[0] ** -0.5)
            return x.to(BF)

        self.norm = [1 + w(D, scale=0.1) for _ in range(2)]
        # mixer: q, k, v, the decay, process-noise and observation-noise logits
        self.mixer = {n: w(D, H * (1 if n == "r" else d)) for n in ("q", "k", "v", "g", "omega", "r")}
        self.attn = {"q": w(D, H * d), "k": w(D, Hk * d), "v": w(D, Hk * d)}
        self.out = [w(D, D) for _ in range(2)]

    # ------------------------------------------------------------- the two layers

    def _mixer_inputs(self, y):
        lead, H, d = y.shape[:-1], self.H, self.d
        x = {n: (y @ W).view(*lead, H, -1) for n, W in self.mixer.items()}
        x["q"], x["k"] = F.normalize(x["q"], dim=-1), F.normalize(x["k"], dim=-1)
        x["g"] = F.logsigmoid(x["g"] + 2.0)
        x["omega"] = F.softplus(x["omega"])
        x["r"] = 0.01 + F.softplus(x["r"].squeeze(-1))
        return [x[n].contiguous() for n in ("q", "k", "v", "g", "omega", "r")]

    def _attn_inputs(self, y):
        lead, d = y.shape[:-1], self.d
        return [(y @ self.attn[n]).view(*lead, -1, d) for n in ("q", "k", "v")]

    @property
    def _at(self):
        return dict(window=self.window, sinks=self.sinks)

    # ------------------------------------------------------------- serving

    def state(self, B):
        S = self.sinks + self.window
        cache = [torch.zeros(B, self.Hk, S, self.d, dtype=BF, device="cuda") for _ in range(2)]
        return {"S": None, "p": None, "kc": cache[0], "vc": cache[1],
                "pos": torch.zeros(B, dtype=torch.int32, device="cuda")}

    def prefill(self, x):
        """x [B,T,D]: the pair's output [B,T,D] and the state that decode continues from."""
        B, T, _ = x.shape
        s = self.state(B)
        y, h, _, _ = kdn.kdn_add_rmsnorm_fwd(x, self.norm[0])
        o, s["S"], s["p"] = kdn.kdn_diag_fwd(*self._mixer_inputs(y), out_dtype=BF)
        x, res = o.view(B, T, -1) @ self.out[0], h
        y, h, _, _ = kdn.kdn_add_rmsnorm_fwd(x, self.norm[1], res)
        q, k, v = self._attn_inputs(y)
        o, _ = kdn.kdn_swa_fwd(q, k, v, want_lse=False, **self._at)
        kdn.kdn_swa_cache_fill(k, v, s["kc"], s["vc"], **self._at)
        s["pos"].fill_(T)
        return o.view(B, T, -1) @ self.out[1] + h, s

    def decode(self, x, s):
        """x [B,D], one token of every sequence; the state moves on in place."""
        B = x.shape[0]
        y, h, _, _ = kdn.kdn_add_rmsnorm_fwd(x, self.norm[0], want_rstd=False)
        o = kdn.kdn_diag_decode_step(*self._mixer_inputs(y), s["S"], s["p"], out_dtype=BF)
        x, res = o.view(B, -1) @ self.out[0], h
        y, h, _, _ = kdn.kdn_add_rmsnorm_fwd(x, self.norm[1], res, want_rstd=False)
        o = kdn.kdn_swa_decode_step(*self._attn_inputs(y), s["kc"], s["vc"], s["pos"], **self._at)
        s["pos"] += 1
        return o.view(B, -1) @ self.out[1] + h

    # ------------------------------------------------------------- training

    def gradients(self, x, dout):
        """Gradients of <dout, output> with respect to x and to both norms' weights."""
        B, T, D = x.shape
        flat = lambda t: t.reshape(B, T, -1)
        y0, h0, rstd0, _ = kdn.kdn_add_rmsnorm_fwd(x, self.norm[0])
        y0_ = y0.detach().requires_grad_()
        with torch.enable_grad():
            ins = self._mixer_inputs(y0_)
        o0, _, _, saved = kdn.kdn_diag_fwd_save(*[t.detach() for t in ins], out_dtype=BF)
        x1 = flat(o0) @ self.out[0]
        y1, h1, rstd1, _ = kdn.kdn_add_rmsnorm_fwd(x1, self.norm[1], h0)
        q, k, v = self._attn_inputs(y1)
        o1, lse = kdn.kdn_swa_fwd(q, k, v, **self._at)
        # output = o1 Wo + h1
        do1 = (dout @ self.out[1].T).view_as(o1)
        g = kdn.kdn_swa_bwd(q, k, v, o1, lse, do1, **self._at)
        dy1 = sum(flat(g["d" + n]) @ self.attn[n].T for n in ("q", "k", "v"))
        dx1, dw1 = kdn.kdn_add_rmsnorm_bwd(h1, self.norm[1], rstd1, dy1, dout)
        # dx1 is the gradient of x1 and of the residual h0 alike
        do0 = (dx1 @ self.out[0].T).view_as(o0)
        g = kdn.kdn_diag_bwd_saved(*[t.detach() for t in ins], saved, do0, out_dtype=BF, want_state_grads=False)
        torch.autograd.backward(ins, [g[n].view_as(t) for n, t in zip(("dq", "dk", "dv", "dg", "domega", "dr"), ins)])
        dx, dw0 = kdn.kdn_add_rmsnorm_bwd(h0, self.norm[0], rstd0, y0_.grad, dx1)
        return dx, dw0, dw1


def main(B=2, T=200, n=40):
    """Prefill and decode against a longer prefill, and a directional difference of the
    output against the gradients.  Returns (decode error, gradient error), both relative."""
    m = Hybrid()
    g = torch.Generator(device="cuda").manual_seed(1)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda").to(BF)
    x = rand(B, T + n, m.D)
    whole, _ = m.prefill(x)
    _, s = m.prefill(x[:, :T].contiguous())
    steps = torch.stack([m.decode(x[:, T + t].contiguous(), s) for t in range(n)], 1)
    err = float((steps.float() - whole[:, T:].float()).norm() / whole[:, T:].float().norm())

    dout, step = rand(B, T, m.D), rand(B, T, m.D)
    x = x[:, :T].contiguous()
    dx, _, _ = m.gradients(x, dout)
    e = 0.25  # of bfloat16 inputs: far above their rounding
    f = lambda a: float((m.prefill(a)[0].double() * dout.double()).sum())
    want = (f((x + e * step).to(BF)) - f((x - e * step).to(BF))) / (2 * e)
    got = float((dx.double() * step.double()).sum())
    scale = float(dx.double().norm() * step.double().norm()) / (B * T * m.D) ** 0.5
    return err, abs(want - got) / scale


if __name__ == "__main__":
    from paper_2609_07816_gb300 import build
    build.build()
    err, grad = main()
    print(f"decode against the longer prefill: relative error {err:.2e}")
    print(f"difference against the gradients: {grad:.2e} of a random direction's share")
