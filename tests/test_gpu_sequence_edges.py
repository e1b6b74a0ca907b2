"""The sequence operators' handles, streams and ends of range: what a call leaves behind, what runs beside it, and the
largest and smallest values and sizes."""
import pytest
import torch

import seq_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def seq():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    import paper_2205_01435_gb300 as pkg
    return pkg.load_seq()


@pytest.fixture(scope="module")
def ops(seq):
    return seq.SequenceOps()


# ------------------------------------------------------------------ handles and streams
def test_new_handle_beside_a_busy_default_stream(seq):
    """A handle's status words are cleared when it is made, not when the default stream comes to it: a call on a
    stream that does not wait for the default one, made at once, meets on cleared counters."""
    side = torch.cuda.Stream()  # (non-blocking)
    g = torch.ones(2_000_000, device="cuda")
    out = torch.empty_like(g)
    warm = seq.SequenceOps()
    warm.clip_grads([g], 1e9, out=[out], stream=side)  # (the module is loaded, the stream in use)
    warm.sync()
    for _ in range(3):
        done = torch.cuda.Event()
        torch.cuda._sleep(50_000_000)  # about 25 ms
        done.record()
        ops = seq.SequenceOps()
        assert done.query()  # nothing of the handle's making is still queued behind the default stream's work
        norm = ops.clip_grads([g], 1e9, out=[out], stream=side)
        torch.cuda._sleep(1_000_000)
        ops.sync()
        ref.check(norm, *ref.clip([g], 1e9)[:2], "norm")
