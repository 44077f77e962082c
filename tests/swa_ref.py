"""Plain 64-bit definition of the sliding-window attention with sinks and of its
gradients, and the error bounds that the kernels' arithmetic implies.

The bounds are elementwise.  u = 2^-9 is the relative rounding of bfloat16, taken
twice (2^-8) for the stored result and for an operand rounded to bfloat16 (the
weights P, and dS, where products run on the tensor cores); r32 covers float32:
a score's sum of d products and the sums over n keys, as random rounding errors of
2^-24 with a factor of 8 in hand.  delta = sum_d o dO is formed from the stored o, except
for queries that see at most 64 keys, where it is formed from the keys."""
import math

import torch

U24 = 2.0 ** -24


def visible(T, W, ns, n, device):
    i = torch.arange(T, device=device)[:, None]
    j = torch.arange(T, device=device)[None]
    return (j <= i) & ((j > i - W) | (j < ns)) & (i < n)


def attention(q, k, v, W, ns, lens=None, scale=None, dO=None):
    """[B,T,H,d] inputs of any dtype -> dict of float64 o, lse, dq, dk, dv and bounds on
    |result - kernel| (eo, else, edq, edk, edv) for the inputs' dtype."""
    B, T, H, d = q.shape
    Hk, G = k.shape[2], H // k.shape[2]
    c = 1 / math.sqrt(d) if scale is None else scale
    half = q.dtype == torch.bfloat16
    u8 = 2.0 ** -8 if half else 2.0 ** -23
    up = 2.0 ** -8 if half else 0.0
    z = lambda *s: torch.zeros(*s, dtype=torch.float64, device=q.device)
    R = {"o": z(B, T, H, d), "lse": z(B, H, T) - math.inf, "eo": z(B, T, H, d), "else": z(B, H, T)}
    if dO is not None:
        for n in ("dq", "edq"):
            R[n] = z(B, T, H, d)
        for n in ("dk", "dv", "edk", "edv"):
            R[n] = z(B, T, Hk, d)
    for b in range(B):
        n = T if lens is None else int(lens[b])
        if n == 0:
            continue
        see = visible(T, W, ns, n, q.device)[:n, :n]
        for h in range(H):
            hk = h // G
            Q, K, V = q[b, :n, h].double(), k[b, :n, hk].double(), v[b, :n, hk].double()
            s = (c * Q @ K.T).masked_fill(~see, -math.inf)
            lse = torch.logsumexp(s, 1)
            P = torch.exp(s - lse[:, None])
            o = P @ V
            smax = float((c * Q.abs() @ K.abs().T).max())
            r32 = 8 * U24 * (math.sqrt(d) * smax / 2 + math.sqrt(n) + 8)
            R["o"][b, :n, h], R["lse"][b, h, :n] = o, lse
            R["eo"][b, :n, h] = u8 * o.abs() + (up + r32) * (P @ V.abs())
            R["else"][b, h, :n] = r32 * (1 + lse.abs())
            if dO is None:
                continue
            g = dO[b, :n, h].double()
            dP, D = g @ V.T, (o * g).sum(1, keepdim=True)
            Da = (o * g).abs().sum(1, keepdim=True)
            dS = P * (dP - D)
            far = (see.sum(1, keepdim=True) > 64).double()
            E = up * dS.abs() + P * (far * up * Da + r32 * (Da + g.abs() @ V.abs().T))
            R["dq"][b, :n, h] = c * dS @ K
            R["edq"][b, :n, h] = c * (E + r32 * dS.abs()) @ K.abs()
            R["dk"][b, :n, hk] += c * dS.T @ Q
            R["edk"][b, :n, hk] += c * (E + r32 * dS.abs()).T @ Q.abs()
            R["dv"][b, :n, hk] += P.T @ g
            R["edv"][b, :n, hk] += (up + r32) * P.T @ g.abs()
    if dO is not None:
        for n in ("dq", "dk", "dv"):
            R["e" + n] += u8 * R[n].abs()
    return R


def check(name, got, want, bound):
    """|got - want| <= bound elementwise; infinities and zeros of the padding exactly."""
    got = got.double()
    assert got.shape == want.shape, name
    fin = torch.isfinite(want)
    assert torch.equal(torch.isfinite(got), fin), f"{name}: not finite where it has to be"
    over = ((got - want).abs() - bound)[fin]
    if over.numel():
        i = int(over.argmax())
        assert float(over[i]) <= 1e-30, (f"{name}: |err| over its bound by {float(over[i]):.3e} "
                                         f"(err {float((got - want).abs()[fin][i]):.3e})")


def decode(q, kc, vc, k, v, pos, W, ns, scale=None):
    """One token over the cache in float64: (o, bound, new kc, new vc)."""
    B, H, d = q.shape
    Hk, G = k.shape[1], H // k.shape[1]
    c = 1 / math.sqrt(d) if scale is None else scale
    half = q.dtype == torch.bfloat16
    u8, up = (2.0 ** -8, 2.0 ** -8) if half else (2.0 ** -23, 0.0)
    kc, vc = kc.clone(), vc.clone()
    o = torch.zeros(B, H, d, dtype=torch.float64, device=q.device)
    e = torch.zeros_like(o)
    for b in range(B):
        p = int(pos[b])
        if p < 0:
            continue
        at = p if p < ns else ns + (p - ns) % W
        kc[b, :, at], vc[b, :, at] = k[b], v[b]
        n = min(p + 1, W + ns)
        for h in range(H):
            K, V = kc[b, h // G, :n].double(), vc[b, h // G, :n].double()
            s = c * K @ q[b, h].double()
            P = torch.softmax(s, 0)
            smax = float((c * K.abs() @ q[b, h].double().abs()).max())
            r32 = 8 * U24 * (math.sqrt(d) * smax / 2 + math.sqrt(n) + 8)
            o[b, h] = P @ V
            e[b, h] = u8 * o[b, h].abs() + (up + r32) * (P @ V.abs())
    return o, e, kc, vc
