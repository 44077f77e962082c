"""Sliding-window attention with sinks on the GPU against its 64-bit definition:
forward, gradients, cache and decode, at the sizes, windows, sinks, lengths and head
groupings where tiles end raggedly and masks leave rows or tiles empty."""
import ctypes
import math

import pytest
import torch

import swa_ref as ref

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def kdn():
    import paper_2609_07816_gb300 as m
    m.lib()
    return m


def rand(seed, *shapes, dtype=BF, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [(torch.randn(*s, generator=g, device="cuda") * scale).to(dtype) for s in shapes]


def make(seed, B, T, H, Hk, d, dtype):
    return rand(seed, (B, T, H, d), (B, T, Hk, d), (B, T, Hk, d), (B, T, H, d), dtype=dtype)


def bwd_workspace(kdn, q, k, W, ns):
    desc = kdn.make_swa_desc(*q.shape[:3], k.shape[2], q.shape[3], q.dtype, window=W, sinks=ns)
    n = kdn.lib().kdn_swa_bwd_workspace_bytes(ctypes.byref(desc))
    return torch.full((n,), 255, dtype=torch.uint8, device="cuda")  # contents need no initialisation


def run_and_check(kdn, q, k, v, dO, W, ns, lens=None, scale=None):
    kw = dict(window=W, sinks=ns, lens=lens, scale=scale, workspace=bwd_workspace(kdn, q, k, W, ns))
    o, lse = kdn.kdn_swa_fwd(q, k, v, **kw)
    assert kdn.kdn_get_device_status(kw["workspace"]) == kdn.KDN_OK  # no wait of the kernel ran out
    G = kdn.kdn_swa_bwd(q, k, v, o, lse, dO, **kw)
    assert kdn.kdn_get_device_status(kw["workspace"]) == kdn.KDN_OK
    clean = [x if lens is None else torch.where(
        (torch.arange(x.shape[1], device="cuda")[None] < lens[:, None])[:, :, None, None], x, 0) for x in (q, k, v, dO)]
    R = ref.attention(*clean[:3], W, ns, lens, scale, clean[3])
    ref.check("o", o, R["o"], R["eo"])
    ref.check("lse", lse, R["lse"], R["else"])
    for n in ("dq", "dk", "dv"):
        ref.check(n, G[n], R[n], R["e" + n])
    return o, lse, G


SHAPES = [(T, W, ns) for T in (1, 2, 63, 64, 65, 127, 128, 129, 255, 256, 257, 300)
          for W, ns in ((1, 0), (7, 3), (64, 1), (128, 0), (129, 5), (1000000, 0))]


@pytest.mark.parametrize("T,W,ns", SHAPES)
@pytest.mark.parametrize("d,dtype", [(128, BF), (64, BF), (32, BF), (128, F32), (32, F32)])
def test_lengths_windows_and_sinks(kdn, T, W, ns, d, dtype):
    q, k, v, dO = make(T * 7 + W, 1, T, 2, 2, d, dtype)
    run_and_check(kdn, q, k, v, dO, W, ns)


@pytest.mark.parametrize("H,Hk", [(1, 1), (3, 1), (6, 2), (8, 1), (4, 4)])
@pytest.mark.parametrize("d,dtype", [(128, BF), (64, BF), (64, F32)])
def test_grouped_heads(kdn, H, Hk, d, dtype):
    q, k, v, dO = make(H * 10 + Hk, 2, 333, H, Hk, d, dtype)
    run_and_check(kdn, q, k, v, dO, 100, 4)


@pytest.mark.parametrize("T,W,ns", [(900, 64, 130), (700, 50, 700), (520, 256, 200), (1111, 300, 17), (640, 1, 1),
                                    (1500, 128, 128)])
@pytest.mark.parametrize("d,dtype", [(128, BF), (64, BF), (32, F32)])
def test_many_tiles_and_wide_sinks(kdn, T, W, ns, d, dtype):
    q, k, v, dO = make(T + W + ns, 1, T, 2, 1, d, dtype)
    run_and_check(kdn, q, k, v, dO, W, ns)


@pytest.mark.parametrize("d,dtype", [(128, BF), (64, BF), (32, BF), (128, F32), (64, F32)])
def test_padding_is_never_used(kdn, d, dtype):
    """Sequences of many lengths, none and one among them; NaN and infinities past each
    length in q, k, v and dO."""
    T, lens = 400, [400, 0, 1, 399, 128, 129, 255, 257, 64]
    B = len(lens)
    q, k, v, dO = make(5, B, T, 4, 2, d, dtype)
    for b, n in enumerate(lens):
        for x in (q, k, v, dO):
            x[b, n:] = math.nan
            x[b, n + 1::3] = math.inf
            x[b, n + 2::3] = -torch.finfo(dtype).max
    L = torch.tensor(lens, dtype=torch.int32, device="cuda")
    o, lse, G = run_and_check(kdn, q, k, v, dO, 150, 9, L)
    for b, n in enumerate(lens):
        for x in (o, G["dq"], G["dk"], G["dv"]):
            assert not x[b, n:].any()
        assert (lse[b, :, n:] == -math.inf).all()


@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("T,step,empty", [(300, 7, 0), (130, 1, 0), (700, 97, 0), (300, 7, 40), (2000, 1, 44)])
def test_many_short_padded_sequences(kdn, d, T, step, empty):
    """Far more work items than CTAs, nearly all of them with a ragged last tile or with
    nothing at all, one after another in the same CTA; passes that nothing waits between."""
    B, H = 48, 8
    lens = [(b * step + 1) % (T + 1) if b % 48 >= empty else 0 for b in range(B)]
    q, k, v, dO = make(T, B, T, H, 2, d, BF)
    for b, n in enumerate(lens):
        for x in (q, k, v, dO):
            x[b, n:] = math.nan
    L = torch.tensor(lens, dtype=torch.int32, device="cuda")
    ws = torch.empty(256, dtype=torch.uint8, device="cuda")
    kw = dict(window=60, sinks=3, lens=L)
    runs = []
    for _ in range(20):
        o, lse = kdn.kdn_swa_fwd(q, k, v, workspace=ws, **kw)
        runs.append((o, lse, *kdn.kdn_swa_bwd(q, k, v, o, lse, dO, **kw).values()))
    assert kdn.kdn_get_device_status(ws) == kdn.KDN_OK
    for r in runs[1:]:
        assert all(torch.equal(x, y) for x, y in zip(r, runs[0]))
    run_and_check(kdn, q, k, v, dO, 60, 3, L)


def test_lengths_out_of_range_are_clamped(kdn):
    q, k, v, dO = make(6, 3, 70, 2, 2, 128, BF)
    L = torch.tensor([1000, -5, 70], dtype=torch.int32, device="cuda")
    o, lse = kdn.kdn_swa_fwd(q, k, v, window=16, lens=L)
    o2, lse2 = kdn.kdn_swa_fwd(q, k, v, window=16, lens=torch.tensor([70, 0, 70], dtype=torch.int32, device="cuda"))
    assert torch.equal(o, o2) and torch.equal(lse, lse2) and not o[1].any()


@pytest.mark.parametrize("d,dtype", [(128, BF), (64, BF), (64, F32)])
def test_large_scores_and_scales(kdn, d, dtype):
    """Scores whose running maximum grows along a row (the accumulator is rescaled), of
    hundreds in size, and scales other than the default."""
    T = 600
    q, k, v, dO = make(8, 1, T, 2, 2, d, dtype)
    ramp = torch.linspace(0.1, 8, T, device="cuda")[None, :, None, None]
    run_and_check(kdn, (q * 2).to(dtype), (k * ramp).to(dtype), v, dO, 333, 2)
    run_and_check(kdn, q, k, v, dO, 200, 2, scale=0.003)
    run_and_check(kdn, q, (k * ramp.flip(1)).to(dtype), v, dO, 500, 0, scale=0.5)


@pytest.mark.parametrize("d,dtype", [(128, BF), (64, BF), (32, F32)])
@pytest.mark.parametrize("B,T,H,Hk,W,ns", [(1, 3000, 1, 1, 64, 4), (1, 1100, 8, 1, 200, 3), (2, 2600, 2, 1, 130, 140)])
def test_split_key_tiles(kdn, d, dtype, B, T, H, Hk, W, ns):
    """Few heads or far queries of the sinks: a key tile's queries are split and joined."""
    q, k, v, dO = make(T, B, T, H, Hk, d, dtype)
    L = torch.tensor([T - 77] * B, dtype=torch.int32, device="cuda") if B > 1 else None
    run_and_check(kdn, q, k, v, dO, W, ns, L)


@pytest.mark.parametrize("d,dtype", [(128, BF), (64, BF), (32, BF), (128, F32)])
def test_same_call_same_bits(kdn, d, dtype):
    q, k, v, dO = make(11, 2, 1000, 4, 2, d, dtype)
    runs = []
    for _ in range(3):
        o, lse = kdn.kdn_swa_fwd(q, k, v, window=100, sinks=4)
        runs.append([o, lse, *kdn.kdn_swa_bwd(q, k, v, o, lse, dO, window=100, sinks=4).values()])
    for r in runs[1:]:
        assert all(torch.equal(x, y) for x, y in zip(r, runs[0]))


def test_gradients_against_differences(kdn):
    """Central differences along random directions: of the 64-bit definition (which pins
    the formula the kernels are held to), and of the float32 kernel's own forward.  The
    kernel's difference has a truncation error of about eps^2 and a rounding error of
    about 1e-6 sqrt(N) / eps of a loss of N terms near one: 2e-3 of the gradient's norm
    at eps = 2^-6 leaves a factor of ten."""
    B, T, H, Hk, d, W, ns = 1, 150, 4, 2, 32, 40, 3
    q, k, v, dO = make(21, B, T, H, Hk, d, F32)
    R = ref.attention(q, k, v, W, ns, dO=dO)
    o, lse = kdn.kdn_swa_fwd(q, k, v, window=W, sinks=ns)
    G = kdn.kdn_swa_bwd(q, k, v, o, lse, dO, window=W, sinks=ns)
    for seed in range(3):
        D = rand(30 + seed, q.shape, k.shape, v.shape, dtype=F32)
        for only in range(3):
            dirs = [x if n == only else torch.zeros_like(x) for n, x in enumerate(D)]
            name, N = (("dq", q), ("dk", k), ("dv", v))[only]
            norm = float(R[name].norm())

            def loss64(e):
                x = [a.double() + e * t.double() for a, t in zip((q, k, v), dirs)]
                return float((ref.attention(*x, W, ns)["o"] * dO.double()).sum())

            want = float((R[name] * dirs[only].double()).sum())
            assert abs((loss64(1e-5) - loss64(-1e-5)) / 2e-5 - want) <= 1e-6 * norm + 1e-7 * N.numel() ** 0.5

            def loss32(e):
                x = [(a + e * t) for a, t in zip((q, k, v), dirs)]
                return float((kdn.kdn_swa_fwd(*x, window=W, sinks=ns)[0].double() * dO.double()).sum())

            e = 2.0 ** -6
            x = (loss32(e) - loss32(-e)) / (2 * e)
            got = float((G[name].double() * dirs[only].double()).sum())
            assert abs(x - got) <= 2e-3 * norm * N.numel() ** 0.5 / 10


def test_gradients_against_close_differences(kdn):
    """Central differences of the float32 kernel's own forward, each direction to 2e-3 of its
    gradient's norm (of which a random direction's share is about one): a term of the
    gradient that is 1 % off shows.  At e = 2^-7 the loss, N = 19200 terms near one with a
    relative rounding of about 2^-22, is off by 2^-22 sqrt(N) / (2 e) = 2e-3, and the third
    derivative, some ten times the gradient's norm, adds e^2 / 6 of it, 1e-4 of the norm.
    The norms are 33 (q, k) and 41 (v): the bound is 0.066 and more."""
    B, T, H, Hk, d, W, ns = 1, 150, 4, 2, 32, 40, 3
    q, k, v, dO = make(21, B, T, H, Hk, d, F32)
    o, lse = kdn.kdn_swa_fwd(q, k, v, window=W, sinks=ns)
    G = kdn.kdn_swa_bwd(q, k, v, o, lse, dO, window=W, sinks=ns)
    e = 2.0 ** -7

    def loss(x):
        return float((kdn.kdn_swa_fwd(*x, window=W, sinks=ns)[0].double() * dO.double()).sum())

    for seed in range(4):
        D = rand(70 + seed, q.shape, k.shape, v.shape, dtype=F32)
        for only, name in enumerate(("dq", "dk", "dv")):
            at = lambda s: [x + s * e * t if n == only else x for n, (x, t) in enumerate(zip((q, k, v), D))]
            got = float((G[name].double() * D[only].double()).sum())
            assert abs((loss(at(1)) - loss(at(-1))) / (2 * e) - got) <= 2e-3 * float(G[name].norm()), name


def test_caller_buffers_streams_and_graphs(kdn):
    """Outputs and workspace of the caller, another stream than the current one, and a
    captured training pass whose replay sees new inputs."""
    q, k, v, dO = make(40, 1, 260, 4, 2, 128, BF)
    o, lse = torch.empty_like(q), torch.empty(1, 4, 260, device="cuda")
    G = {n: torch.empty_like(x) for n, x in (("dq", q), ("dk", k), ("dv", v))}
    ws = bwd_workspace(kdn, q, k, 64, 2)

    def step(stream=None):
        kdn.kdn_swa_fwd(q, k, v, window=64, sinks=2, o=o, lse=lse, workspace=ws, stream=stream)
        kdn.kdn_swa_bwd(q, k, v, o, lse, dO, window=64, sinks=2, grads=G, workspace=ws, stream=stream)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    torch.cuda.current_stream().wait_stream(side)
    R = ref.attention(q, k, v, 64, 2, dO=dO)
    ref.check("o", o, R["o"], R["eo"])
    for x in ("dq", "dk", "dv"):
        ref.check(x, G[x], R[x], R["e" + x])
    assert kdn.kdn_get_device_status(ws) == kdn.KDN_OK
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for x, y in zip((q, k, v, dO), make(41, 1, 260, 4, 2, 128, BF)):
        x.copy_(y)
    graph.replay()
    R = ref.attention(q, k, v, 64, 2, dO=dO)
    ref.check("o", o, R["o"], R["eo"])
    for x in ("dq", "dk", "dv"):
        ref.check(x, G[x], R[x], R["e" + x])


def test_empty_calls(kdn):
    for B, T, H in ((0, 5, 2), (2, 0, 2), (2, 5, 0)):
        q = torch.empty(B, T, H, 64, dtype=BF, device="cuda")
        k = torch.empty(B, T, H, 64, dtype=BF, device="cuda")
        o, lse = kdn.kdn_swa_fwd(q, k, k, window=4)
        g = kdn.kdn_swa_bwd(q, k, k, o, lse, q, window=4)
        assert o.numel() == 0 and g["dq"].numel() == 0


# ------------------------------------------------------------------ cache and decode


def fill_ref(k, v, kc, vc, W, ns, lens):
    for b, n in enumerate(lens):
        for t in range(n):
            if t < ns or t >= n - W:
                at = t if t < ns else ns + (t - ns) % W
                kc[b, :, at], vc[b, :, at] = k[b, t], v[b, t]


@pytest.mark.parametrize("d,dtype", [(128, BF), (64, BF), (32, BF), (64, F32)])
@pytest.mark.parametrize("W,ns", [(1, 0), (16, 3), (50, 0), (100, 130), (500, 2)])
def test_cache_fill(kdn, d, dtype, W, ns):
    T, lens = 211, [211, 0, 1, 2, 16, 19, 20, 150, 210]
    k, v = rand(3, *[(len(lens), T, 3, d)] * 2, dtype=dtype)
    kc, vc = rand(4, *[(len(lens), 3, W + ns, d)] * 2, dtype=dtype)
    for L in (lens, None):
        a, b, x, y = kc.clone(), vc.clone(), kc.clone(), vc.clone()
        t = None if L is None else torch.tensor(L, dtype=torch.int32, device="cuda")
        kdn.kdn_swa_cache_fill(k, v, a, b, window=W, sinks=ns, lens=t)
        fill_ref(k, v, x, y, W, ns, L or [T] * len(lens))
        assert torch.equal(a, x) and torch.equal(b, y)


@pytest.mark.parametrize("H,Hk", [(1, 1), (4, 4), (6, 2), (8, 1), (9, 1), (16, 1), (18, 2), (40, 2)])
@pytest.mark.parametrize("d,dtype", [(128, BF), (64, BF), (32, BF), (128, F32), (32, F32)])
def test_decode_step(kdn, H, Hk, d, dtype):
    """Sequences of every age, idle ones among them; slots that hold no token hold NaN."""
    W, ns = 70, 5
    pos = [0, 3, -1, 5, 33, 74, 75, 76, 1000, 2**31 - 1, 4, 64]
    B, S = len(pos), W + ns
    q, k, v = rand(H, (B, H, d), (B, Hk, d), (B, Hk, d), dtype=dtype)
    kc, vc = rand(H + 1, *[(B, Hk, S, d)] * 2, dtype=dtype)
    for b, p in enumerate(pos):
        if p < S:
            kc[b, :, max(p, 0):], vc[b, :, max(p, 0):] = math.nan, math.inf
    P = torch.tensor(pos, dtype=torch.int32, device="cuda")
    want, bound, kr, vr = ref.decode(q, kc, vc, k, v, pos, W, ns)
    o = kdn.kdn_swa_decode_step(q, k, v, kc, vc, P, window=W, sinks=ns)
    ref.check("o", o, want, bound)
    same = lambda a, b: torch.equal(a.nan_to_num(9.0), b.nan_to_num(9.0))
    assert same(kc, kr) and same(vc, vr)
    assert not o[2].any()


@pytest.mark.parametrize("W,ns", [(1, 0), (2, 1), (63, 0), (64, 0), (1000, 4), (2048, 4), (5000, 0)])
@pytest.mark.parametrize("d,dtype,H,Hk", [(128, BF, 4, 2), (64, BF, 16, 1), (64, F32, 2, 2)])
def test_decode_windows(kdn, W, ns, d, dtype, H, Hk):
    pos = [W + ns + 17, (W + ns) // 2]
    q, k, v = rand(W, (2, H, d), (2, Hk, d), (2, Hk, d), dtype=dtype)
    kc, vc = rand(W + 1, *[(2, Hk, W + ns, d)] * 2, dtype=dtype)
    want, bound, kr, vr = ref.decode(q, kc, vc, k, v, pos, W, ns)
    o = kdn.kdn_swa_decode_step(q, k, v, kc, vc, torch.tensor(pos, dtype=torch.int32, device="cuda"), window=W,
                                sinks=ns)
    ref.check("o", o, want, bound)
    assert torch.equal(kc, kr) and torch.equal(vc, vr)


@pytest.mark.parametrize("d,dtype", [(128, BF), (64, BF), (32, F32)])
def test_prefill_then_decode_is_the_longer_prefill(kdn, d, dtype):
    """Prompts of several lengths into the cache, then token by token past the window's
    wrap: every step agrees with the attention over the whole sequence."""
    B, T, H, Hk, W, ns, lens = 4, 90, 4, 2, 24, 3, [0, 2, 30, 60]
    q, k, v, _ = make(50, B, T, H, Hk, d, dtype)
    kc, vc = (torch.full((B, Hk, W + ns, d), math.nan, dtype=dtype, device="cuda") for _ in range(2))
    L = torch.tensor(lens, dtype=torch.int32, device="cuda")
    kdn.kdn_swa_cache_fill(k, v, kc, vc, window=W, sinks=ns, lens=L)
    R = ref.attention(q, k, v, W, ns)
    for s in range(30):
        at = [n + s for n in lens]
        pick = lambda x: torch.stack([x[b, t] for b, t in enumerate(at)])
        pos = L + s
        o = kdn.kdn_swa_decode_step(pick(q), pick(k), pick(v), kc, vc, pos, window=W, sinks=ns)
        ref.check(f"step {s}", o, pick(R["o"]), pick(R["eo"]))


def test_decode_in_a_graph(kdn):
    """Positions live on the device: one captured step serves every token."""
    B, H, d, W, ns = 2, 4, 128, 20, 2
    kc, vc = (torch.zeros(B, H, W + ns, d, dtype=BF, device="cuda") for _ in range(2))
    q, k, v = rand(60, *[(B, H, d)] * 3)
    o, pos = torch.empty_like(q), torch.zeros(B, dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    kdn.kdn_swa_decode_step(q, k, v, kc.clone(), vc.clone(), pos, window=W, sinks=ns, o=o)
    with torch.cuda.graph(graph):
        kdn.kdn_swa_decode_step(q, k, v, kc, vc, pos, window=W, sinks=ns, o=o)
        pos.add_(1)
    Q, K, V = rand(61, *[(B, 50, H, d)] * 3)
    R = ref.attention(Q, K, V, W, ns)
    for t in range(50):
        q.copy_(Q[:, t]), k.copy_(K[:, t]), v.copy_(V[:, t])
        graph.replay()
        ref.check(f"t={t}", o, R["o"][:, t], R["eo"][:, t])


def test_cache_beyond_32_bit_offsets(kdn):
    """A cache of more than 2^31 elements: the last sequence's rows lie past 32-bit offsets."""
    B, d, W, ns = 3, 128, 6_000_000, 0
    assert B * W * d > 2 ** 31
    kc, vc = (torch.zeros(B, 1, W, d, dtype=BF, device="cuda") for _ in range(2))
    q, k, v = rand(70, *[(B, 1, d)] * 3)
    pos = [3, W + 5, W - 1]  # the last two see the whole cache
    # one key per sequence that takes a known share: score ln(W) against W - 2 zero scores
    at = [1, W // 2, W - 2]
    for b in range(B):
        u = q[b, 0].double() / q[b, 0].double().norm() ** 2
        kc[b, 0, at[b]] = (u * math.log(W) * math.sqrt(d)).to(BF)
        vc[b, 0, at[b]] = 1
    want, bound, kr, vr = ref.decode(q, kc, vc, k, v, pos, W, ns)
    o = kdn.kdn_swa_decode_step(q, k, v, kc, vc, torch.tensor(pos, dtype=torch.int32, device="cuda"), window=W)
    ref.check("o", o, want, bound)
    assert torch.equal(kc[2, 0, W - 1], k[2, 0]) and torch.equal(vc[1, 0, 5], v[1, 0])
    assert torch.equal(kc, kr)
