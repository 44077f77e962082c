"""Workloads of the hybrid layer's operators: sliding-window attention with sinks
(training, prefill, decode over its bounded cache) and the residual RMS norm
(forward with an output in the activations' type or in 8 bits, and training).

Every case runs either the plain form (``own`` false: elementary torch
operations in 32 bits, rounded once at the end) or the library's entry points
(``own`` true) on the same inputs.

Kinds of a case
  train    one training pass of the attention: forward, then the gradients
  prefill  the forward over a prompt, and the cache that decode continues from
  decode   one token for every sequence of a batch over the cache
  norm     the residual's addition and the norm in front of a layer's projections
  normtr   the same with its gradients
"""
import math

import torch

own = False

EPS = 1e-6
F8_MAX = 448.0  # largest finite value of the 8-bit type (e4m3)
_DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # a training step of the 1.3B-shaped layer: B8, T4096, 16 heads of 128
        _attn("train_b8_t4096", "train", 8, 4096, 16, 16, 128, 2048, 4),
        # grouped heads of 64, an odd length, padded batch (one sequence empty)
        _attn("train_gqa_ragged", "train", 4, 1777, 16, 4, 64, 512, 16, ragged=True),
        # a float32 check run at the small size
        _attn("train_f32_small", "train", 2, 200, 4, 4, 32, 64, 3, dtype="f32"),
        # one long prompt
        _attn("prefill_t65536", "prefill", 1, 65536, 16, 16, 128, 2048, 4),
        # a batch of short prompts of different lengths, eight query heads to a kv head
        _attn("prefill_ragged", "prefill", 8, 1000, 16, 2, 128, 256, 64, ragged=True),
        # a single user's next token: latency
        _decode("decode_b1", 1, 16, 16, 128, 2048, 4, 9999),
        # the serving batch of the decode benchmark: B256, 16 heads of 128
        _decode("decode_b256", 256, 16, 16, 128, 2048, 4, 5000),
        # odd batch and grouping, sequences of every age, one slot of the batch idle
        _decode("decode_gqa_ragged", 61, 18, 2, 64, 1000, 3, 1500, ragged=True),
        # the norm in front of one decoded token
        _norm("norm_one_row", "norm", 1, 2304, True, "bf16"),
        # the 1.3B-shaped layer's tokens, output in 8 bits for 8-bit projections
        _norm("norm_f8_block", "norm", 32768, 2048, True, "f8", block=128),
        # training pass of the norm at the same shape
        _norm("normtr_b8_t4096", "normtr", 32768, 2048, True, "bf16"),
        # an odd number of rows in float32, without a residual
        _norm("normtr_f32", "normtr", 1601, 2304, False, "f32", dtype="f32"),
    ]


def _attn(name, kind, B, T, H, Hk, d, window, sinks, dtype="bf16", ragged=False):
    return {"name": name, "kind": kind, "B": B, "T": T, "H": H, "Hk": Hk, "d": d, "window": window,
            "sinks": sinks, "dtype": dtype, "ragged": ragged}


def _decode(name, B, H, Hk, d, window, sinks, pos, dtype="bf16", ragged=False):
    return {"name": name, "kind": "decode", "B": B, "H": H, "Hk": Hk, "d": d, "window": window,
            "sinks": sinks, "pos": pos, "dtype": dtype, "ragged": ragged}


def _norm(name, kind, rows, D, residual, out, dtype="bf16", block=0):
    return {"name": name, "kind": kind, "rows": rows, "D": D, "residual": residual, "out": out,
            "dtype": dtype, "block": block}


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("train", "train", "prefill", "prefill", "decode", "decode", "norm", "normtr"))
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    if kind in ("norm", "normtr"):
        D = 8 * _log(rng, 8, 1024)
        rows = _log(rng, 1, max(1, min(65536, (32768 * 2048) // D // (2 if dtype == "f32" else 1))))
        out = "f8" if kind == "norm" and rng.random() < 0.5 else dtype
        c = _norm("", kind, rows, D, rng.random() < 0.7, out, dtype, rng.choice((0, 128)) if out == "f8" else 0)
    else:
        d = rng.choice((32, 64, 128, 128))
        Hk = rng.choice((1, 2, 3, 4, 8, 16))
        H = Hk * rng.choice((1, 1, 2, 3, 4, 8) if Hk < 8 else (1, 2))
        window, sinks = _log(rng, 16, 4096), rng.choice((0, 1, 3, 4, 16, 100))
        ragged = rng.random() < 0.4
        if kind == "decode":
            B = _log(rng, 1, 256)
            while B * Hk * (window + sinks) * d * (2 if dtype == "f32" else 1) > 256 * 16 * 2052 * 128:
                window = max(16, window // 2)
            c = _decode("", B, H, Hk, d, window, sinks, _log(rng, 1, 20000), dtype, ragged)
        else:
            T = _log(rng, 1, 65536 if kind == "prefill" else 8192)
            B = _log(rng, 1, 8)
            # no more than the largest listed pass of its kind costs, an eighth of it in float32
            most = 65536 * 16 * 2048 if kind == "prefill" else 8 * 4096 * 16 * 2048
            most = most // 8 if dtype == "f32" else most
            while B * T * H * min(T, window + sinks) > most or B * T * H * d > 8 * 4096 * 16 * 128:
                if B > 1:
                    B = max(1, B // 2)
                else:
                    T = max(1, T * 3 // 4)
            c = _attn("", kind, B, T, H, Hk, d, window, sinks, dtype, ragged)
    del c["name"]
    return c


# ------------------------------------------------------------------ inputs


def _lens(c):
    """Lengths of a padded batch: the full one, none, one token, and others between."""
    B, T = c["B"], c["T"]
    if not c["ragged"]:
        return [T] * B
    return [T - T // 3] if B == 1 else [T, 0, min(T, 1)][:B] + [T * b // B for b in range(3, B)]


def _positions(c):
    """Positions of a decode batch's tokens; a ragged one has an idle slot (-1) and sequences of every age."""
    B, p = c["B"], c["pos"]
    if not c["ragged"]:
        return [p] * B
    return [p * (b + 1) // B if b != 1 else -1 for b in range(B)]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    dt = _DT[case["dtype"]]

    def randn(*shape, scale=1.0, shift=0.0):
        return torch.randn(*shape, generator=g, device="cuda", dtype=dt) * scale + shift

    s = {"case": case}
    if case["kind"] in ("norm", "normtr"):
        n, D = case["rows"], case["D"]
        s["x"] = randn(n, D)
        s["res"] = randn(n, D, scale=2.0) if case["residual"] else None
        s["w"] = randn(D, scale=0.2, shift=1.0)
        if case["kind"] == "normtr":
            s["dy"], s["dh"] = randn(n, D, scale=0.1), randn(n, D, scale=0.1) if case["residual"] else None
        return s
    B, H, Hk, d = case["B"], case["H"], case["Hk"], case["d"]
    S = case["window"] + case["sinks"]
    if case["kind"] == "decode":
        s["q"], s["k"], s["v"] = randn(B, H, d), randn(B, Hk, d), randn(B, Hk, d)
        s["kc"], s["vc"] = randn(B, Hk, S, d), randn(B, Hk, S, d)
        s["pos"] = torch.tensor(_positions(case), dtype=torch.int32, device="cuda")
        return s
    T = case["T"]
    s["q"], s["k"], s["v"] = randn(B, T, H, d), randn(B, T, Hk, d), randn(B, T, Hk, d)
    s["lens"] = torch.tensor(_lens(case), dtype=torch.int32, device="cuda") if case["ragged"] else None
    if case["kind"] == "train":
        s["dO"] = randn(B, T, H, d, scale=0.1)
    else:
        s["kc"], s["vc"] = randn(B, Hk, S, d), randn(B, Hk, S, d)
    return s


# ------------------------------------------------------------------ one pass


def run(s):
    c = s["case"]
    return (_run_own if own else _run_plain)[c["kind"]](s, c)


def _own_train(s, c):
    import paper_2609_07816_gb300 as kdn
    at = dict(window=c["window"], sinks=c["sinks"], lens=s["lens"])
    o, lse = kdn.kdn_swa_fwd(s["q"], s["k"], s["v"], **at)
    return {"o": o, "lse": lse, **kdn.kdn_swa_bwd(s["q"], s["k"], s["v"], o, lse, s["dO"], **at)}


def _own_prefill(s, c):
    import paper_2609_07816_gb300 as kdn
    at = dict(window=c["window"], sinks=c["sinks"], lens=s["lens"])
    o, _ = kdn.kdn_swa_fwd(s["q"], s["k"], s["v"], want_lse=False, **at)
    kdn.kdn_swa_cache_fill(s["k"], s["v"], s["kc"], s["vc"], **at)
    return {"o": o, "kc": s["kc"], "vc": s["vc"]}


def _own_decode(s, c):
    import paper_2609_07816_gb300 as kdn
    o = kdn.kdn_swa_decode_step(s["q"], s["k"], s["v"], s["kc"], s["vc"], s["pos"], window=c["window"],
                                sinks=c["sinks"])
    return {"o": o, "kc": s["kc"], "vc": s["vc"]}


def _own_norm(s, c):
    import paper_2609_07816_gb300 as kdn
    y, h, _, scales = kdn.kdn_add_rmsnorm_fwd(s["x"], s["w"], s["res"], eps=EPS, block=c["block"], want_rstd=False,
                                              out_dtype=torch.float8_e4m3fn if c["out"] == "f8" else None)
    return {"y": y, **({"h": h} if c["residual"] else {}), **({"scales": scales} if c["out"] == "f8" else {})}


def _own_normtr(s, c):
    import paper_2609_07816_gb300 as kdn
    y, h, rstd, _ = kdn.kdn_add_rmsnorm_fwd(s["x"], s["w"], s["res"], eps=EPS)
    dx, dw = kdn.kdn_add_rmsnorm_bwd(h, s["w"], rstd, s["dy"], s["dh"])
    return {"y": y, **({"h": h} if c["residual"] else {}), "rstd": rstd, "dx": dx, "dw": dw}


# ------------------------------------------------------------------ plain forms


def _live(s, T):
    """Which tokens of the padded batch there are: [B or 1, T]."""
    t = torch.arange(T, device=s["q"].device)[None]
    return t < (T if s["lens"] is None else s["lens"][:, None])


def _bands(x, nb, c):
    """[B, h, T, d] in blocks of c tokens: [B, h, nb, c, d]."""
    B, h, T, d = x.shape
    return torch.nn.functional.pad(x, (0, 0, 0, nb * c - T)).view(B, h, nb, c, d)


def _with_previous(x):
    """Each block behind the one before it: the keys that a block's window reaches."""
    return torch.cat([torch.nn.functional.pad(x[:, :, :-1], (0, 0, 0, 0, 1, 0)), x], 3)


def _weights(s, c):
    """Scores of every query block against the sinks and its band of keys, as unnormalised weights."""
    B, T, H, Hk, d, W = (c[n] for n in ("B", "T", "H", "Hk", "d", "window"))
    W, ns, dev = min(W, T), min(c["sinks"], T), s["q"].device
    nb = -(-T // W)
    live = _live(s, T)
    keep = live[:, :, None, None]

    def heads(x):
        return torch.where(keep, x.float(), 0.0).transpose(1, 2)

    q = heads(s["q"]).reshape(B, Hk, H // Hk, T, d)
    q = _bands(q.flatten(1, 2), nb, W).view(B, Hk, H // Hk, nb, W, d)
    k, v = _bands(heads(s["k"]), nb, W), _bands(heads(s["v"]), nb, W)
    ks, vs = (heads(s[x])[:, :, None, None, :ns] for x in ("k", "v"))
    if nb > 1:
        k, v = _with_previous(k), _with_previous(v)
    k, v = k[:, :, None], v[:, :, None]  # over a group's query heads
    i = torch.arange(nb * W, device=dev).view(nb, W, 1)
    j = torch.arange(k.shape[-2], device=dev) + (torch.arange(nb, device=dev) * W - (k.shape[-2] - W)).view(nb, 1, 1)
    band = (j <= i) & (j > i - c["window"]) & (j >= 0)
    sink = torch.arange(ns, device=dev) <= i - c["window"]
    rows = _bands(live[:, None, :, None].float(), nb, W) > 0  # [B or 1, 1, nb, W, 1]
    mask = (torch.cat([sink, band], -1) & rows)[:, :, None]
    scale = 1.0 / math.sqrt(d)
    sc = torch.cat([q @ ks.transpose(-1, -2), q @ k.transpose(-1, -2)], -1) * scale
    sc = sc.masked_fill_(~mask, -math.inf)
    m = sc.amax(-1, keepdim=True).clamp_min(-1e30)
    p = sc.sub_(m).exp_()
    l = p.sum(-1, keepdim=True)
    return q, (ks, k), (vs, v), p, m, l, ns, scale


def _tokens(x, c, dt):
    """[B, Hk, G, nb, W, d] back to [B, T, H, d]."""
    B, T = c["B"], c["T"]
    return x.reshape(B, x.shape[1] * x.shape[2], -1, x.shape[-1])[:, :, :T].transpose(1, 2).to(dt).contiguous()


def _times(p, xs, ns):
    """Weights times the sinks' and the band's rows."""
    return p[..., :ns] @ xs[0] + p[..., ns:] @ xs[1]


def _to_keys(p, x, c, ns):
    """Transposed weights times the queries' rows `x`: the sum over a group's heads and over the blocks that see a key."""
    B, T, Hk = c["B"], c["T"], c["Hk"]
    W, nb, d = x.shape[-2], x.shape[-3], x.shape[-1]
    band = (p[..., ns:].transpose(-1, -2) @ x).sum(2)  # [B, Hk, nb, W or 2W, d]
    own_block = band[..., -W:, :].clone()
    if nb > 1:
        own_block[:, :, :-1] += band[:, :, 1:, :W]
    out = own_block.reshape(B, Hk, nb * W, d)[:, :, :T]
    if ns:
        out[:, :, :ns] += (p[..., :ns].transpose(-1, -2) @ x).sum((2, 3))
    return out.transpose(1, 2)


def _plain_attention(s, c, grads):
    q, ks, vs, p, m, l, ns, scale = _weights(s, c)
    B, T, H, dt = c["B"], c["T"], c["H"], s["q"].dtype
    p = p.div_(torch.where(l > 0, l, 1.0))
    o = _times(p, vs, ns)
    out = {"o": _tokens(o, c, dt)}
    if not grads:
        return out
    lse = torch.where(l > 0, m + torch.log(l), -math.inf)
    out["lse"] = lse.reshape(B, H, -1)[:, :, :T].contiguous()
    dO = torch.where(_live(s, T)[:, :, None, None], s["dO"].float(), 0.0).transpose(1, 2)
    dO = _bands(dO, q.shape[3], q.shape[4]).view(q.shape)
    out["dv"] = _to_keys(p, dO, c, ns).to(dt).contiguous()
    dp = torch.cat([dO @ vs[0].transpose(-1, -2), dO @ vs[1].transpose(-1, -2)], -1)
    ds = dp.sub_((dO * o).sum(-1, keepdim=True)).mul_(p)
    out["dq"] = _tokens(_times(ds, ks, ns) * scale, c, dt)
    out["dk"] = (_to_keys(ds, q, c, ns) * scale).to(dt).contiguous()
    return out


def _plain_train(s, c):
    return _plain_attention(s, c, True)


def _newest(c, T, lens):
    """For every slot of the cache the newest token of the prompt that belongs there, and whether there is one."""
    W, ns, dev = c["window"], c["sinks"], lens.device
    slot = torch.arange(W + ns, device=dev)
    last = lens.long()[:, None] - 1
    ring = last - (last - slot) % W  # the newest t <= last with (t - sinks) % W == slot - sinks
    t = torch.where(slot < ns, slot, ring)
    return t.clamp_min(0), (t <= last) & (t >= torch.where(slot < ns, 0, ns))


def _plain_prefill(s, c):
    out = _plain_attention(s, c, False)
    B, T = c["B"], c["T"]
    lens = s["lens"] if s["lens"] is not None else torch.full((B,), T, dtype=torch.int32, device=s["q"].device)
    t, has = _newest(c, T, lens)
    for cache, x in ((s["kc"], s["k"]), (s["vc"], s["v"])):
        new = x.gather(1, t[:, :, None, None].expand(-1, -1, c["Hk"], c["d"])).transpose(1, 2)
        cache.copy_(torch.where(has[:, None, :, None], new, cache))
    return {**out, "kc": s["kc"], "vc": s["vc"]}


def _plain_decode(s, c):
    B, H, Hk, d, W, ns = (c[n] for n in ("B", "H", "Hk", "d", "window", "sinks"))
    pos = s["pos"].long()
    slot = torch.where(pos < ns, pos, ns + (pos - ns) % W)
    at = torch.arange(W + ns, device=pos.device)
    here = (at == slot[:, None])[:, None, :, None]
    for cache, x in ((s["kc"], s["k"]), (s["vc"], s["v"])):
        cache.copy_(torch.where(here, x[:, :, None], cache))
    q = s["q"].float().view(B, Hk, H // Hk, d)
    seen = (at <= pos[:, None])[:, None, None]
    sc = (q @ s["kc"].float().transpose(-1, -2) / math.sqrt(d)).masked_fill(~seen, -math.inf)
    p = torch.exp(sc - sc.amax(-1, keepdim=True).clamp_min(-1e30))
    l = p.sum(-1, keepdim=True)
    o = (p / torch.where(l > 0, l, 1.0)) @ s["vc"].float()
    return {"o": o.view(B, H, d).to(s["q"].dtype), "kc": s["kc"], "vc": s["vc"]}


def _plain_add_norm(s):
    h = s["x"].float() + s["res"].float() if s["res"] is not None else s["x"].float()
    rstd = 1.0 / torch.sqrt(h.square().mean(-1) + EPS)
    return h, rstd, h * rstd[:, None] * s["w"].float()


def _amax(y, block):
    """Largest magnitude of each row, or of each `block` columns of it: [rows, blocks]."""
    n, D = y.shape
    b = block or D
    return torch.nn.functional.pad(y.abs(), (0, -D % b)).view(n, -1, b).amax(-1)


def _plain_norm(s, c):
    h, rstd, y = _plain_add_norm(s)
    dt, out = s["x"].dtype, {}
    if c["residual"]:
        out["h"] = h.to(dt)
    if c["out"] != "f8":
        return {"y": y.to(dt), **out}
    amax = _amax(y, c["block"])
    scales = torch.where(amax > 0, amax / F8_MAX, 1.0)
    wide = scales.repeat_interleave(c["block"] or c["D"], 1)[:, :c["D"]]
    return {"y": (y / wide).to(torch.float8_e4m3fn), "scales": scales, **out}


def _plain_normtr(s, c):
    h, rstd, y = _plain_add_norm(s)
    dt = s["x"].dtype
    out = {"y": y.to(dt), "rstd": rstd}
    if c["residual"]:
        out["h"] = h.to(dt)
        h = h.to(dt).float()  # the residual stream as it is kept for the backward pass
    dy, xh = s["dy"].float(), h * rstd[:, None]
    g = dy * s["w"].float()
    dx = rstd[:, None] * (g - xh * (g * xh).mean(-1, keepdim=True))
    out["dx"] = (dx if s["dh"] is None else dx + s["dh"].float()).to(dt)
    out["dw"] = (dy * xh).sum(0)
    return out


_run_plain = {"train": _plain_train, "prefill": _plain_prefill, "decode": _plain_decode, "norm": _plain_norm,
              "normtr": _plain_normtr}
_run_own = {"train": _own_train, "prefill": _own_prefill, "decode": _own_decode, "norm": _own_norm,
            "normtr": _own_normtr}


# ------------------------------------------------------------------ cost


def _pairs(n, W, ns):
    """Visible (query, key) pairs of a sequence of n tokens."""
    a = min(n, W)
    total = a * (a + 1) // 2 + (n - a) * W
    far = n - a  # queries whose window leaves tokens behind: 1, 2, ... of them
    b = min(far, ns)
    return total + b * (b + 1) // 2 + (far - b) * ns


def work(case):
    c = case
    es = 4 if c["dtype"] == "f32" else 2
    if c["kind"] in ("norm", "normtr"):
        n, r = c["rows"] * c["D"], int(c["residual"])
        out = 1 if c["out"] == "f8" else es
        b = n * (es * (1 + 2 * r) + out) + c["D"] * es
        f = n * (6 + r)
        if c["out"] == "f8":
            b += c["rows"] * -(-c["D"] // (c["block"] or c["D"])) * 4
        if c["kind"] == "normtr":
            b += n * es * (2 + r) + c["rows"] * 4 + c["D"] * 4
            f += n * 12
        return {"bytes": b, "flops": f}
    B, H, Hk, d, W, ns = (c[n] for n in ("B", "H", "Hk", "d", "window", "sinks"))
    if c["kind"] == "decode":
        pos = [p for p in _positions(c) if p >= 0]
        n = sum(min(p, W + ns - 1) for p in pos)  # rows of the cache read beside the new token's
        live = len(pos)
        return {"bytes": es * d * (2 * n * Hk + live * (4 * Hk + H) + B * H), "flops": 4 * d * H * (n + live)}
    T, lens = c["T"], _lens(c)
    tok = sum(lens)
    pairs = sum(_pairs(n, W, ns) for n in lens)
    qo, kv = tok * H * d * es, tok * Hk * d * es
    full = B * T * H * d * es  # outputs are written whole, padding included
    if c["kind"] == "train":
        return {"bytes": 2 * qo + 2 * kv + 2 * full + 2 * B * T * Hk * d * es + B * H * T * 4,
                "flops": 14 * d * H * pairs}
    kept = sum(min(n, W + ns) for n in lens)
    return {"bytes": qo + 2 * kv + full + 2 * kept * Hk * d * es, "flops": 4 * d * H * pairs}


# ------------------------------------------------------------------ 64 bits


def _exact_head(q, k, v, dO, W, ns, scale, rows=2048):
    """One head of one sequence from the definition, by strips of queries: o, lse and the gradients."""
    n, d = q.shape
    o, lse = torch.zeros_like(q), q.new_full((n,), -math.inf)
    dq, dk, dv = (torch.zeros_like(x) for x in (q, k, v))
    for a in range(0, n, rows):
        e = min(n, a + rows)
        lo = max(0, a - W + 1)
        j = torch.arange(lo, e, device=q.device)
        j = torch.cat([torch.arange(min(ns, lo), device=q.device), j])
        i = torch.arange(a, e, device=q.device)[:, None]
        see = (j <= i) & ((j > i - W) | (j < ns))
        sc = (q[a:e] @ k[j].T * scale).masked_fill(~see, -math.inf)
        lse[a:e] = torch.logsumexp(sc, 1)
        p = torch.exp(sc - lse[a:e, None])
        o[a:e] = p @ v[j]
        if dO is not None:
            dp = dO[a:e] @ v[j].T
            ds = p * (dp - (p * dp).sum(1, keepdim=True)) * scale
            dq[a:e] = ds @ k[j]
            dk.index_add_(0, j, ds.T @ q[a:e])
            dv.index_add_(0, j, p.T @ dO[a:e])
    return o, lse, dq, dk, dv


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["kind"] in ("norm", "normtr"):
        return _exact_norm(s, c)
    B, H, Hk, d, W, ns = (c[n] for n in ("B", "H", "Hk", "d", "window", "sinks"))
    scale = 1.0 / math.sqrt(d)
    if c["kind"] == "decode":
        o = torch.zeros(B, H, d, dtype=torch.float64, device="cuda")
        for b, p in enumerate(_positions(c)):
            if p < 0:
                continue
            at = p if p < ns else ns + (p - ns) % W
            s["kc"][b, :, at], s["vc"][b, :, at] = s["k"][b], s["v"][b]
            n = min(p + 1, W + ns)
            q = s["q"][b].double().view(Hk, H // Hk, d)
            w = torch.softmax(q @ s["kc"][b, :, :n].double().transpose(1, 2) * scale, -1)
            o[b] = (w @ s["vc"][b, :, :n].double()).view(H, d)
        return {"o": o, "kc": s["kc"].double(), "vc": s["vc"].double()}
    train, T = c["kind"] == "train", c["T"]
    if B * T * H * min(T, W) * d * (7 if train else 2) > 8 * 4096 * 16 * 2048 * 128 * 7:
        return None
    out = {"o": torch.zeros(B, T, H, d, dtype=torch.float64, device="cuda")}
    if train:
        out["lse"] = torch.full((B, H, T), -math.inf, dtype=torch.float64, device="cuda")
        out["dq"] = torch.zeros_like(out["o"])
        out["dk"], out["dv"] = (torch.zeros(B, T, Hk, d, dtype=torch.float64, device="cuda") for _ in range(2))
    for b, n in enumerate(_lens(c)):
        for h in range(H if n else 0):
            hk = h // (H // Hk)
            q, k, v = s["q"][b, :n, h].double(), s["k"][b, :n, hk].double(), s["v"][b, :n, hk].double()
            r = _exact_head(q, k, v, s["dO"][b, :n, h].double() if train else None, W, ns, scale)
            out["o"][b, :n, h] = r[0]
            if train:
                out["lse"][b, h, :n], out["dq"][b, :n, h] = r[1], r[2]
                out["dk"][b, :n, hk] += r[3]
                out["dv"][b, :n, hk] += r[4]
    if not train:
        for b, n in enumerate(_lens(c)):
            for t in range(max(0, n - W - ns), n):
                if t >= ns and t < n - W:
                    continue
                at = t if t < ns else ns + (t - ns) % W
                s["kc"][b, :, at], s["vc"][b, :, at] = s["k"][b, t], s["v"][b, t]
            m = min(n, ns)
            s["kc"][b, :, :m] = s["k"][b, :m].transpose(0, 1)
            s["vc"][b, :, :m] = s["v"][b, :m].transpose(0, 1)
        out["kc"], out["vc"] = s["kc"].double(), s["vc"].double()
    return out


def _exact_norm(s, c):
    x = s["x"].double()
    h = x if s["res"] is None else x + s["res"].double()
    out = {}
    rstd = (h.pow(2).sum(1) / c["D"] + EPS).rsqrt()
    y = h * rstd[:, None] * s["w"].double()
    if c["residual"]:
        out["h"] = h
    if c["kind"] == "norm":
        if c["out"] != "f8":
            return {"y": y, **out}
        step = c["block"] or c["D"]
        parts = [y[:, a:a + step] for a in range(0, c["D"], step)]
        amax = [p.abs().amax(1, keepdim=True) for p in parts]
        scales = [torch.where(a > 0, a / F8_MAX, 1.0) for a in amax]
        return {"y": torch.cat([p / a for p, a in zip(parts, scales)], 1), "scales": torch.cat(scales, 1), **out}
    kept = h.to(s["x"].dtype).double()  # what the forward pass stores is what the backward pass is given
    dy, w = s["dy"].double(), s["w"].double()
    xh = kept * rstd[:, None]
    dot = (dy * w * xh).sum(1, keepdim=True) / c["D"]
    dx = rstd[:, None] * (dy * w - xh * dot)
    return {"y": y, "rstd": rstd, **out, "dx": dx if s["dh"] is None else dx + s["dh"].double(),
            "dw": torch.einsum("nd,nd->d", dy, xh)}
