"""The decayed attention's and the head norm's C entries without a device, and the references the GPU tests use."""
import pytest
import torch

import decay_reference as ref


@pytest.fixture(scope="module")
def seq():
    import paper_2205_01435_gb300 as pkg
    pkg._build.build()
    return pkg.load_seq()


def test_null_handles_are_rejected(seq):
    lib, none = seq._lib, None
    assert lib.wm_seq_head_norm(none, 0, 1, 1, 1, 0, 0, 1, none, none, 0, none, none, 0.0, *([none] * 5)) == 1
    assert lib.wm_seq_head_norm_backward(none, 0, 1, 1, 1, 0, 0, 1, none, none, none, 0, none, none, none, 0.0, *([none] * 7)) == 1
    assert lib.wm_seq_decay_attention(none, 0, 1, 1, 1, 1, 1, *([none] * 4), 1.0, *([none] * 6)) == 1
    assert lib.wm_seq_decay_attention_backward(none, 0, 1, 1, 1, 1, 1, *([none] * 4), 1.0, *([none] * 10)) == 1


def test_a_closed_handle_is_refused(seq):
    x, g = torch.zeros(2, 1, 1, 4), torch.zeros(1)
    ops = seq.SequenceOps.__new__(seq.SequenceOps)
    ops.h, ops._index = None, 0
    for call in (lambda: ops.head_norm(x), lambda: ops.head_norm_backward(x, x), lambda: ops.decay_attention(x, x, x, g),
                 lambda: ops.decay_step(x[0], x[0], x[0], g, None), lambda: ops.decay_attention_backward(x, x, x, g, x)):
        with pytest.raises(ValueError, match="closed"):
            call()


def test_the_attention_reference_agrees_with_autograd():
    gen = torch.Generator().manual_seed(0)
    T, N, H, Dk, Dv = 9, 4, 2, 3, 5

    def r(*s):
        return torch.randn(s, generator=gen, dtype=torch.float64)

    leaf = [r(T, N, H, Dk), r(T, N, H, Dk), r(T, N, H, Dv), r(N, H, Dk, Dv)]
    q, k, v, s0 = (x.requires_grad_() for x in leaf)
    do, dl, g, scale = r(T, N, H, Dv), r(N, H, Dk, Dv), torch.tensor([-0.3, -float("inf")], dtype=torch.float64), 0.7
    reset = (torch.rand(T, N, generator=gen) < 0.3).to(torch.uint8)
    reset[0, 3] = 1
    lens = torch.tensor([T, 0, 5, T], dtype=torch.int32)
    live = torch.arange(T)[:, None] < lens[None]
    # the definition as sums over pairs of tokens
    outs, lasts = [], []
    for n in range(N):
        for h in range(H):
            lam = float(torch.exp(g[h]))
            state = s0[n, h]
            for t in range(int(lens[n])):
                keep = 0.0 if reset[t, n] else lam
                state = keep * state + k[t, n, h][:, None] * v[t, n, h][None]
                outs.append((scale * (q[t, n, h] @ state) * do[t, n, h]).sum())
            lasts.append((state * dl[n, h]).sum())
    (sum(outs) + sum(lasts)).backward()
    a = [x.detach() for x in leaf]
    f = ref.attend(a[0], a[1], a[2], g, scale, a[3], reset, lens, factors=True)
    assert torch.allclose((f["o"][0] * do * live[..., None, None]).sum() + (f["s_last"][0] * dl).sum(), (sum(outs) + sum(lasts)).detach(), atol=1e-10)
    b = ref.attend_backward(a[0], a[1], a[2], g, scale, do, dl, a[3], reset, lens, factors=True)
    for name, x in zip(("dq", "dk", "dv", "ds0"), leaf):
        assert torch.allclose(b[name][0], x.grad, atol=1e-11), name
        assert (b[name][1] >= 0).all()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rotary", [0, 4, 6])
def test_the_norm_reference_agrees_with_autograd(interleaved, rotary):
    gen = torch.Generator().manual_seed(1)
    x, w = (torch.randn(s, generator=gen, dtype=torch.float64, requires_grad=True) for s in ((3, 2, 2, 7), (7,)))
    dy = torch.randn(3, 2, 2, 7, generator=gen, dtype=torch.float64)
    pos = torch.randint(-9, 9, (3, 2), generator=gen, dtype=torch.int32)
    f = torch.tensor([1.0, 0.3, 0.1][:rotary // 2]) if rotary else None
    y = x / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-3) * w
    if rotary:
        ang = pos.double()[..., None, None] * f.double()
        parts = list(y.unbind(-1))
        for i in range(rotary // 2):
            ia, ib = (2 * i, 2 * i + 1) if interleaved else (i, i + rotary // 2)
            a, b, c, s = parts[ia], parts[ib], torch.cos(ang[..., i]), torch.sin(ang[..., i])
            parts[ia], parts[ib] = a * c - b * s, b * c + a * s
        y = torch.stack(parts, -1)
    (y * dy).sum().backward()
    got = ref.head_norm(x.detach(), w.detach(), 1e-3, pos, f, interleaved)
    assert torch.allclose(got[0], y.detach(), atol=1e-12)
    b = ref.head_norm_backward(x.detach(), w.detach(), 1e-3, pos, f, interleaved, dy)
    assert torch.allclose(b["dx"][0], x.grad, atol=1e-12) and torch.allclose(b["dw"][0], w.grad, atol=1e-12)
