"""The sequence operators' C entries without a device: no handle, no call."""
import ctypes as C

import pytest


@pytest.fixture(scope="module")
def seq():
    import paper_2205_01435_gb300 as pkg
    pkg._build.build()
    return pkg.load_seq()


def test_null_handles_are_rejected(seq):
    lib = seq._lib
    assert lib.wm_seq_embed(None, 0, 1, 1, 1, None, None, 1.0, None, None) == 1
    assert lib.wm_seq_embed_backward(None, 0, 1, 1, 1, None, None, 1.0, None, None) == 1
    assert lib.wm_seq_layer_norm(None, 0, 1, 1, None, 1, None, None, 0.0, None, 1, None, None, None) == 1
    assert lib.wm_seq_layer_norm_backward(None, 0, 1, 1, None, 1, *([None] * 4), 1, None, 1, None, None, None) == 1
    assert lib.wm_seq_gated_scan(None, 0, 1, 1, 1, *([None] * 8)) == 1
    assert lib.wm_seq_gated_scan_backward(None, 0, 1, 1, 1, *([None] * 12)) == 1
    assert lib.wm_seq_clip(None, 0, None, 1.0, None, None) == 1
    assert lib.wm_seq_sync(None) == 1
    assert lib.wm_seq_last_error(None) == b"null handle"
    assert lib.wm_seq_last_launches(None) == 0
    lib.wm_seq_destroy(None)
    lib.wm_seq_create.argtypes = [C.POINTER(C.c_void_p)]
    assert lib.wm_seq_create(None) == 1


def test_the_references_agree_with_autograd():
    """The 64-bit definitions that the GPU tests use, against torch's own derivatives of them."""
    import torch

    import seq_reference as ref

    g = torch.Generator().manual_seed(0)
    T, N, H = 9, 3, 4
    gate, x, h0 = (torch.randn(s, generator=g, dtype=torch.float64, requires_grad=True) for s in ((T, N, H), (T, N, H), (N, H)))
    dh, dl = torch.randn(T, N, H, generator=g, dtype=torch.float64), torch.randn(N, H, generator=g, dtype=torch.float64)
    reset = (torch.rand(T, N, generator=g) < 0.3).to(torch.uint8)
    lens = torch.tensor([T, 0, 5], dtype=torch.int32)
    f = ref.scan(gate, x, h0, reset, lens)
    live = torch.arange(T)[:, None, None] < lens.long()[None, :, None]
    ((f["h"][0] * dh * live).sum() + (f["h_last"][0] * dl).sum()).backward()
    b = ref.scan_backward(gate.detach(), x.detach(), f["h"][0].detach(), dh, dl, h0.detach(), reset, lens)
    for k, v in (("dgate", gate), ("dx", x), ("dh0", h0)):
        assert torch.allclose(b[k][0], v.grad, atol=1e-12), k

    x, w, bias = (torch.randn(s, generator=g, dtype=torch.float64, requires_grad=True) for s in ((6, 10), (10,), (10,)))
    dy = torch.randn(6, 10, generator=g, dtype=torch.float64)
    f = ref.norm(x, w, bias, 1e-5)
    assert torch.allclose(f["y"][0], torch.nn.functional.layer_norm(x, (10,), w, bias, 1e-5), atol=1e-12)
    (f["y"][0] * dy).sum().backward()
    b = ref.norm_backward(x.detach(), w.detach(), f["mean"][0].detach(), f["rstd"][0].detach(), dy)
    for k, v in (("dx", x), ("dw", w), ("db", bias)):
        assert torch.allclose(b[k][0], v.grad, atol=1e-12), k


def test_a_closed_handle_is_refused(seq):
    """What a method of a closed SequenceOps comes to."""
    import torch

    x = torch.zeros(2, 3)
    ops = seq.SequenceOps.__new__(seq.SequenceOps)
    ops.h, ops._index = None, 0
    for call in (lambda: ops.layer_norm(x), lambda: ops.gated_step(x, x, None), lambda: ops.clip_grads([x], 1.0),
                 lambda: ops.embed(x, x)):
        with pytest.raises(ValueError, match="closed"):
            call()
