"""The 64-bit definition and error bounds of swa_ref.py for long sequences with a narrow
window: strips of queries against the keys that some query of the strip sees, so that
nothing of size T x T is held."""
import math

import torch

from swa_ref import U24


def head(q, k, v, dO, W, ns, scale=None, rows=1024):
    """One head's [T, d] inputs of any dtype -> dict of float64 o, lse, dq, dk, dv and bounds on
    |result - kernel| (eo, else, edq, edk, edv) for the inputs' dtype.  dk and dv (and their
    bounds) are this query head's share, and the bounds leave out the rounding of the stored
    sum: `stored` adds it."""
    T, d = q.shape
    half = q.dtype == torch.bfloat16
    u8, up = (2.0 ** -8, 2.0 ** -8) if half else (2.0 ** -23, 0.0)
    c = 1 / math.sqrt(d) if scale is None else scale
    Q, K, V, G = (x.double() for x in (q, k, v, dO))
    R = {n: torch.zeros_like(Q) for n in ("o", "dq", "dk", "dv", "eo", "edq", "edk", "edv")}
    R["lse"], R["else"] = (torch.zeros(T, dtype=torch.float64, device=q.device) for _ in range(2))
    for a in range(0, T, rows):
        e = min(T, a + rows)
        lo = max(0, a - W + 1)
        j = torch.cat([torch.arange(min(ns, lo), device=q.device), torch.arange(lo, e, device=q.device)])
        i = torch.arange(a, e, device=q.device)[:, None]
        see = (j <= i) & ((j > i - W) | (j < ns))
        Kj, Vj, Qi, g = K[j], V[j], Q[a:e], G[a:e]
        s = (c * Qi @ Kj.T).masked_fill(~see, -math.inf)
        lse = torch.logsumexp(s, 1)
        P = torch.exp(s - lse[:, None])
        o = P @ Vj
        smax = float((c * Qi.abs() @ Kj.abs().T).max())
        r32 = 8 * U24 * (math.sqrt(d) * smax / 2 + math.sqrt(int(see.sum(1).max())) + 8)
        R["o"][a:e], R["lse"][a:e] = o, lse
        R["eo"][a:e] = u8 * o.abs() + (up + r32) * (P @ Vj.abs())
        R["else"][a:e] = r32 * (1 + lse.abs())
        D, Da = (o * g).sum(1, keepdim=True), (o * g).abs().sum(1, keepdim=True)
        dS = P * (g @ Vj.T - D)
        far = (see.sum(1, keepdim=True) > 64).double()
        E = up * dS.abs() + P * (far * up * Da + r32 * (Da + g.abs() @ Vj.abs().T)) + r32 * dS.abs()
        R["dq"][a:e] = c * dS @ Kj
        R["edq"][a:e] = c * E @ Kj.abs()
        for n, x in (("dk", c * dS.T @ Qi), ("edk", c * E.T @ Qi.abs()), ("dv", P.T @ g),
                     ("edv", (up + r32) * P.T @ g.abs())):
            R[n].index_add_(0, j, x)
    R["edq"] += u8 * R["dq"].abs()
    return R


def group(q, k, v, dO, W, ns, scale=None):
    """The query heads of one kv head: q, dO [T, G, d], k, v [T, d].  o and dq [T, G, d], lse [G, T],
    dk and dv [T, d], with bounds."""
    heads = [head(q[:, g], k, v, dO[:, g], W, ns, scale) for g in range(q.shape[1])]
    R = {n: torch.stack([r[n] for r in heads], 1) for n in ("o", "dq", "eo", "edq")}
    R.update({n: torch.stack([r[n] for r in heads]) for n in ("lse", "else")})
    R.update({n: sum(r[n] for r in heads) for n in ("dk", "dv", "edk", "edv")})
    u8 = 2.0 ** -8 if q.dtype == torch.bfloat16 else 2.0 ** -23
    for n in ("dk", "dv"):
        R["e" + n] += u8 * R[n].abs()
    return R
