"""The kept status word: taken from memory whose last tensor a queued kernel still reads, and written by
calls of another stream."""
import pytest
import torch

pytestmark = pytest.mark.gpu

CYCLES = 40_000_000  # about 20 ms of queueing


def test_a_word_in_another_tensors_memory(monkeypatch):
    import paper_2609_07816_gb300 as kdn
    kdn.lib()
    x, wg, wu, wd = (torch.ones(*s, dtype=torch.bfloat16, device="cuda") for s in ((1, 64), (64, 64), (64, 64), (64, 64)))
    h, y = torch.empty_like(x), torch.empty_like(x)
    run = lambda s=None: kdn.kdn_ffn_fwd(x, wg, wu, wd, h=h, y=y, want_saved=False, stream=s)
    run()
    side = torch.cuda.Stream()
    for _ in range(3):
        monkeypatch.setattr(kdn, "_status_words", {})
        kept = [torch.full((64,), 7.0, device="cuda") for _ in range(64)]
        torch.cuda.synchronize()
        torch.cuda._sleep(CYCLES)
        read = torch.stack(kept)
        at = {t.data_ptr() for t in kept}
        del kept
        run()
        assert kdn._status_words[0].data_ptr() in at  # (else the case is not the one that is meant)
        run(side)
        torch.cuda.synchronize()
        assert bool((read == 7.0).all())
