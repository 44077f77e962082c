"""Calls on a stream other than the current one, queued behind other work there, while the
current stream allocates and fills memory: no kernel of the call may see it, and an output
may be dropped while the caller's stream still reads it."""
import pytest
import torch

from kdn_inputs import make_inputs

pytestmark = pytest.mark.gpu

BF = torch.bfloat16
CYCLES = 40_000_000  # about 20 ms of queueing; only how long a wrong call has to go wrong in


@pytest.fixture(scope="module")
def kdn():
    import paper_2609_07816_gb300 as m
    m.lib()
    return m


def rand(seed, *shapes):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randn(*s, generator=g, device="cuda").to(BF) for s in shapes]


def passes(kdn):
    q, k, v, dO = rand(1, (2, 700, 8, 128), (2, 700, 2, 128), (2, 700, 2, 128), (2, 700, 8, 128))
    x, r, dy = rand(2, *[(3000, 1024)] * 3)
    w, = rand(3, (1024,))

    def attention(s):
        o, lse = kdn.kdn_swa_fwd(q, k, v, window=90, sinks=4, stream=s)
        return [o, lse, *kdn.kdn_swa_bwd(q, k, v, o, lse, dO, window=90, sinks=4, stream=s).values()]

    def norm(s):
        y, h, rstd, _ = kdn.kdn_add_rmsnorm_fwd(x, w, r, stream=s)
        return [y, *kdn.kdn_add_rmsnorm_bwd(h, w, rstd, dy, stream=s)]  # h and rstd are dropped here

    ins = make_inputs("diag", 2, 500, 2, 128, 128, dtype="bf16", seed=4, s0_std=0.0, p0_range=(0.5, 2.0), with_grad=True)
    t = [torch.tensor(ins[n], dtype=BF, device="cuda") for n in ("q", "k", "v", "g", "omega", "r")]
    dmix = torch.tensor(ins["dO"], dtype=BF, device="cuda")

    def mixer(s):
        o, ST, pT, saved = kdn.kdn_diag_fwd_save(*t, stream=s)
        return [o, ST, pT, *kdn.kdn_diag_bwd_saved(*t, saved, dmix, stream=s).values()]

    return {"attention": attention, "norm": norm, "mixer": mixer}


def fill(sizes):
    """Takes memory of these sizes from the current stream and writes all over it."""
    for n in sizes:
        torch.full((n,), 255, dtype=torch.uint8, device="cuda")


SIZES = [256, 512] + [1 << n for n in range(10, 26)]


@pytest.mark.parametrize("what", ["attention", "norm", "mixer"])
def test_memory_of_a_call_on_another_stream(kdn, what):
    run = passes(kdn)[what]
    want = run(None)
    home, side = torch.cuda.current_stream(), torch.cuda.Stream()
    for _ in range(3):
        torch.cuda.synchronize()
        side.wait_stream(home)
        with torch.cuda.stream(side):
            torch.cuda._sleep(CYCLES)
        got = run(side)
        fill(SIZES * 4 + [t.numel() * t.element_size() for t in want])
        home.wait_stream(side)
        assert all(torch.equal(x, y) for x, y in zip(got, want))


@pytest.mark.parametrize("what", ["attention", "norm", "mixer"])
def test_outputs_are_dropped_while_the_callers_stream_reads_them(kdn, what):
    run = passes(kdn)[what]
    want = run(None)
    home, side = torch.cuda.current_stream(), torch.cuda.Stream()
    side.wait_stream(home)
    got = run(side)
    home.wait_stream(side)
    torch.cuda._sleep(CYCLES)
    copies = [t.clone() for t in got]
    del got
    with torch.cuda.stream(side):
        fill([t.numel() * t.element_size() for t in want] * 2)
    assert all(torch.equal(x, y) for x, y in zip(copies, want))


def test_handles_that_are_not_torch_streams(kdn):
    class Handle:
        def __init__(self, h):
            self.cuda_stream = h

    run = passes(kdn)["attention"]
    want, side = run(None), torch.cuda.Stream()
    for h in (side.cuda_stream, 0):
        torch.cuda.synchronize()
        got = run(Handle(h))
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want))
