"""Decayed linear attention and the head norm against their definitions in 64 bits (tests/decay_reference.py, which also gives the
error they may have), at the sizes and masks where they can go wrong, their gradients against differences, and what they refuse."""
import math

import pytest
import torch

import decay_reference as ref
from seq_reference import check

pytestmark = pytest.mark.gpu

DT = {"fp32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def seq():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    import paper_2205_01435_gb300 as pkg
    return pkg.load_seq()


@pytest.fixture(scope="module")
def ops(seq):
    return seq.SequenceOps()


def rnd(*shape, seed, dtype=torch.float32, mean=0.0, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std + mean).to(dtype).cuda()


def place(v, layout):
    """The values of [T, N, H, D] in a layout of their own."""
    T, N, H, D = v.shape
    if layout == "plain":
        return v
    if layout == "columns":  # columns of a wider array
        w = torch.full((T, N, H, D + 8), float("nan"), dtype=v.dtype, device="cuda")
        w[..., 8:] = v
        return w[..., 8:]
    if layout == "batch":  # batch-major storage
        return v.transpose(0, 1).contiguous().transpose(0, 1)
    if layout == "heads":  # a head's sequence in one piece
        return v.permute(1, 2, 0, 3).contiguous().permute(2, 0, 1, 3)
    if layout == "shifted":  # not aligned to more than an element
        w = torch.empty(v.numel() + 1, dtype=v.dtype, device="cuda")
        w[1:] = v.reshape(-1)
        return w[1:].view(v.shape)
    raise AssertionError(layout)


def decays(H):
    """From heads that forget at once to ones that keep hundreds of tokens."""
    return torch.log1p(-torch.exp2(-(0.2 + 8.0 * torch.arange(H) / max(1, H - 1)))).float().cuda()


def inputs(T, N, H, Dk, Dv, dtype, layout="plain", seed=0, reset=False, lengths=False, state=True):
    s = dict(q=place(rnd(T, N, H, Dk, seed=seed + 1, dtype=dtype), layout), k=place(rnd(T, N, H, Dk, seed=seed + 2, dtype=dtype), layout),
             v=place(rnd(T, N, H, Dv, seed=seed + 3, dtype=dtype), layout), do=place(rnd(T, N, H, Dv, seed=seed + 4, dtype=dtype), layout),
             g=decays(H), scale=0.37, s0=None, ds_last=None, reset=None, lengths=None)
    if state:
        s["s0"], s["ds_last"] = rnd(N, H, Dk, Dv, seed=seed + 5), rnd(N, H, Dk, Dv, seed=seed + 6)
    gen = torch.Generator().manual_seed(seed + 7)
    if reset:
        s["reset"] = (torch.rand(T, N, generator=gen) < 0.05).to(torch.uint8).cuda() * 3
        if T > 1 and N > 1:
            s["reset"][0, 0] = 1
            s["reset"][T - 1, N - 1] = 1
    if lengths:
        ln = torch.randint(0, T + 1, (N,), generator=gen, dtype=torch.int32)
        ln[0] = 0
        ln[N - 1] = T
        if N > 2:
            ln[1] = min(1, T)
        s["lengths"] = ln.cuda()
        for key in ("q", "k", "v", "do"):  # nothing in the padding is read
            for n in range(N):
                s[key][int(ln[n]):, n] = float("nan") if n % 2 else float("inf")
    return s


def masks(s):
    return dict(s0=s["s0"], reset=s["reset"], lengths=s["lengths"])


def near(got, value, what, dtype):
    """Errors of independent roundings, against the output's norm: three of 2^-8 / sqrt(3) in bf16 (products, state, output);
    fewer than 1000 of U in fp32."""
    off = float((got.detach().cpu().double() - value).norm() / value.norm().clamp(min=1e-30))
    assert off <= (1.25 * 2.0 ** -8 if dtype == torch.bfloat16 else 32 * ref.U), f"{what}: {off}"


def check_all(ops, s, out=None, grads=(None, None, None)):
    o, last = ops.decay_attention(s["q"], s["k"], s["v"], s["g"], scale=s["scale"], out=out, **masks(s))
    got = ops.decay_attention_backward(s["q"], s["k"], s["v"], s["g"], s["do"], scale=s["scale"], ds_last=s["ds_last"], dq=grads[0], dk=grads[1],
                                       dv=grads[2], **masks(s))
    f = ref.attend(s["q"], s["k"], s["v"], s["g"], s["scale"], **masks(s))
    b = ref.attend_backward(s["q"], s["k"], s["v"], s["g"], s["scale"], s["do"], s["ds_last"], **masks(s))
    for name, value in [("o", o), ("s_last", last)]:
        check(value, *f[name], name)
        if f[name][0].numel() > 1000:
            near(value, f[name][0], name, value.dtype)
    for name, value in zip(("dq", "dk", "dv", "ds0"), got):
        check(value, *b[name], name)
        if b[name][0].numel() > 1000:
            near(value, b[name][0], name, value.dtype)
    ops.sync()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("T,N,H,Dk,Dv", [(1, 1, 1, 1, 1), (1, 4, 2, 64, 64), (2, 3, 2, 5, 3), (9, 2, 3, 16, 16), (31, 2, 1, 64, 64), (64, 1, 2, 32, 64),
                                         (65, 2, 2, 64, 32), (127, 1, 2, 43, 43), (128, 2, 2, 64, 64), (129, 1, 2, 128, 64), (200, 2, 2, 64, 128),
                                         (300, 1, 2, 128, 128), (140, 1, 1, 256, 40), (70, 1, 2, 40, 256), (400, 1, 1, 8, 8), (130, 1, 1, 200, 136)])
def test_sizes(ops, dtype, T, N, H, Dk, Dv):
    check_all(ops, inputs(T, N, H, Dk, Dv, DT[dtype], seed=T))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("layout", ["columns", "batch", "heads", "shifted"])
@pytest.mark.parametrize("T,N,H,Dk,Dv", [(7, 3, 2, 40, 24), (150, 2, 3, 64, 64), (90, 2, 2, 31, 33)])
def test_layouts(ops, dtype, layout, T, N, H, Dk, Dv):
    s = inputs(T, N, H, Dk, Dv, DT[dtype], layout, seed=11)
    # outputs side by side in one wide array, nothing else written
    wide = torch.full((T, N, H * (2 * Dk + Dv) + 8), 7.0, dtype=DT[dtype], device="cuda")
    dq, dk, dv = (p.unflatten(-1, (H, -1)) for p in wide[..., :-8].split([H * Dk, H * Dk, H * Dv], -1))
    o = torch.empty((N, T, H, Dv), dtype=DT[dtype], device="cuda").transpose(0, 1)
    check_all(ops, s, out=o, grads=(dq, dk, dv))
    assert (wide[..., -8:] == 7.0).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("T,N,H,Dk,Dv", [(1, 4, 2, 16, 16), (6, 5, 2, 64, 64), (40, 5, 2, 24, 8), (129, 3, 2, 64, 64), (300, 4, 2, 33, 32), (1500, 3, 1, 32, 48)])
@pytest.mark.parametrize("reset,lengths", [(True, False), (False, True), (True, True)])
def test_resets_and_lengths(ops, dtype, T, N, H, Dk, Dv, reset, lengths):
    check_all(ops, inputs(T, N, H, Dk, Dv, DT[dtype], seed=5 + T, reset=reset, lengths=lengths))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("T,N,H,Dk,Dv,masked", [(2500, 1, 2, 32, 32, False), (2000, 2, 1, 64, 64, True), (1300, 1, 3, 43, 40, True), (1100, 1, 1, 128, 128, False)])
def test_split_over_time(ops, dtype, T, N, H, Dk, Dv, masked):
    """Few sequences: spans of time side by side, resets and padding across their borders."""
    check_all(ops, inputs(T, N, H, Dk, Dv, DT[dtype], seed=T, reset=masked, lengths=masked and N > 1))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("T", [3, 70, 200])
def test_extreme_decays(ops, dtype, T):
    """No decay, decay at once, and only the token itself."""
    s = inputs(T, 2, 4, 32, 32, DT[dtype], seed=3, reset=True)
    s["g"] = torch.tensor([0.0, -1e-6, -90.0, -float("inf")], device="cuda")
    check_all(ops, s)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("T", [5, 100, 1200])
def test_optional_arguments(ops, dtype, T):
    s = inputs(T, 2, 2, 32, 32, DT[dtype], seed=9, state=False)
    check_all(ops, s)
    o, last = ops.decay_attention(s["q"], s["k"], s["v"], s["g"])
    o1, none = ops.decay_attention(s["q"], s["k"], s["v"], s["g"], want_last=False)
    assert none is None and torch.equal(o, o1)
    g = ops.decay_attention_backward(s["q"], s["k"], s["v"], s["g"], s["do"])
    g1 = ops.decay_attention_backward(s["q"], s["k"], s["v"], s["g"], s["do"], want_ds0=False)
    assert g1[3] is None and all(torch.equal(a, b) for a, b in zip(g[:3], g1))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("T", [1, 4, 40, 300, 1500])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_what_is_not_finite_stays_where_it_is_seen(ops, dtype, T, bad):
    """A token's bad values reach the outputs that see it: not the ones before it, not an episode after a reset."""
    dt, N, H, D = DT[dtype], 2, 2, 64
    s = inputs(T, N, H, D, D, dt, seed=21)
    at, cut = T // 3, (2 * T) // 3
    s["reset"] = torch.zeros(T, N, dtype=torch.uint8, device="cuda")
    s["reset"][cut] = 1
    clean = ops.decay_attention(s["q"], s["k"], s["v"], s["g"], **masks(s))
    cleang = ops.decay_attention_backward(s["q"], s["k"], s["v"], s["g"], s["do"], ds_last=s["ds_last"], **masks(s))
    seen = torch.zeros(T, dtype=torch.bool)
    seen[at:cut if cut > at else T] = True
    tol = 4.0 * ref.B if dt == torch.bfloat16 else 1e-5  # (bad sequences go another way, with roundings of their own)

    def same(a, b, what):
        if a.numel() == 0:
            return
        assert torch.isfinite(a).all(), what
        assert float((a.double() - b.double()).abs().max()) <= tol * float(b.double().abs().max()), what

    for name in ("k", "v"):
        t = dict(s)
        t[name] = s[name].clone()
        t[name][at, 0, 1, 3] = bad
        o, last = ops.decay_attention(t["q"], t["k"], t["v"], t["g"], **masks(t))
        same(o[:, 1], clean[0][:, 1], "another sequence")
        same(o[:, 0, 0], clean[0][:, 0, 0], "another head")
        same(o[~seen, 0, 1], clean[0][~seen, 0, 1], "outputs that do not see it")
        assert not torch.isfinite(o[at, 0, 1]).all()
        if cut > at:
            same(last, clean[1], "the state after the next episode")
    if cut <= at:
        return
    t = dict(s, do=s["do"].clone())
    t["do"][at, 0, 1, 3] = bad
    dq, dk, dv, ds0 = ops.decay_attention_backward(t["q"], t["k"], t["v"], t["g"], t["do"], ds_last=t["ds_last"], **masks(t))
    later = torch.arange(T) > at
    for name, got, want in (("dk", dk, cleang[1]), ("dv", dv, cleang[2])):
        same(got[later, 0, 1], want[later, 0, 1], name + " of tokens after it")
        same(got[:, 1], want[:, 1], name + " of another sequence")
    same(dq[torch.arange(T) != at, 0, 1], cleang[0][torch.arange(T) != at, 0, 1], "dq of other tokens")
    assert not torch.isfinite(dq[at, 0, 1]).all()
    ops.sync()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_reset_drops_a_bad_state(ops, dtype):
    for T in (1, 5, 100):
        s = inputs(T, 1, 1, 32, 32, DT[dtype], seed=2)
        s["reset"] = torch.zeros(T, 1, dtype=torch.uint8, device="cuda")
        s["reset"][0] = 1
        want = ops.decay_attention(s["q"], s["k"], s["v"], s["g"], **masks(s))
        s["s0"] = torch.full_like(s["s0"], float("nan"))
        got = ops.decay_attention(s["q"], s["k"], s["v"], s["g"], **masks(s))
        for a, b in zip(got, want):
            assert torch.isfinite(a).all() and float((a - b).abs().max()) <= 0.02 * float(b.abs().max())


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_empty(ops, dtype):
    dt = DT[dtype]
    e = torch.empty(0, 2, 3, 8, dtype=dt, device="cuda")
    s0 = rnd(2, 3, 8, 8, seed=1)
    o, last = ops.decay_attention(e, e, e, decays(3), s0=s0)
    assert o.shape == e.shape and torch.equal(last, s0)
    assert (ops.decay_attention(e, e, e, decays(3))[1] == 0).all()
    g = ops.decay_attention_backward(e, e, e, decays(3), e, ds_last=s0)
    assert torch.equal(g[3], s0)
    e = torch.empty(4, 0, 3, 8, dtype=dt, device="cuda")
    o, last = ops.decay_attention(e, e, e, decays(3))
    assert o.shape == e.shape and last.shape == (0, 3, 8, 8)


def test_lengths_out_of_range(ops, seq):
    for T in (3, 50, 300):
        s = inputs(T, 3, 2, 32, 32, torch.bfloat16, seed=4)
        s["lengths"] = torch.tensor([-5, T + 7, 2], dtype=torch.int32, device="cuda")
        got = ops.decay_attention(s["q"], s["k"], s["v"], s["g"], **masks(s))
        with pytest.raises(seq.WMError):
            ops.sync()
        ops.sync()
        s["lengths"] = torch.tensor([0, T, 2], dtype=torch.int32, device="cuda")
        want = ops.decay_attention(s["q"], s["k"], s["v"], s["g"], **masks(s))
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_step_is_the_attention(ops, dtype):
    """A dream token by token, the state in place, against one call on all."""
    T, N, H, Dk, Dv = 40, 3, 2, 48, 64
    s = inputs(T, N, H, Dk, Dv, DT[dtype], seed=8, reset=True)
    f = ref.attend(s["q"], s["k"], s["v"], s["g"], s["scale"], factors=False, **masks(s))
    state = s["s0"].clone()
    for t in range(T):
        o, st = ops.decay_step(s["q"][t], s["k"][t], s["v"][t], s["g"], state, scale=s["scale"], reset=s["reset"][t], out_state=state)
        assert st is state
        check(o, f["o"][0][t], f["o"][1][t], "o")
    check(state, *f["s_last"], "state")
    # in parts, each entering with the state before it, in place
    for cuts in ((0, 7, 40), (0, 1, 30, 40), (0, 16, 17, 40)):
        state, outs = s["s0"].clone(), []
        for a, b in zip(cuts, cuts[1:]):
            o, st = ops.decay_attention(s["q"][a:b], s["k"][a:b], s["v"][a:b], s["g"], scale=s["scale"], s0=state, reset=s["reset"][a:b].contiguous(),
                                        s_last=state)
            outs.append(o)
        f = ref.attend(s["q"], s["k"], s["v"], s["g"], s["scale"], **masks(s))
        check(torch.cat(outs), *f["o"], "o in parts")
        check(state, *f["s_last"], "state of the parts")


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("T,N,H,D", [(5, 2, 2, 64), (100, 2, 2, 64), (2000, 1, 2, 64), (200, 1, 1, 160)])
def test_states_in_place(ops, dtype, T, N, H, D):
    s = inputs(T, N, H, D, D, DT[dtype], seed=6)
    o, last = ops.decay_attention(s["q"], s["k"], s["v"], s["g"], s0=s["s0"])
    st = s["s0"].clone()
    o1, l1 = ops.decay_attention(s["q"], s["k"], s["v"], s["g"], s0=st, s_last=st)
    assert l1 is st and torch.equal(o, o1) and torch.equal(last, st)
    g = ops.decay_attention_backward(s["q"], s["k"], s["v"], s["g"], s["do"], ds_last=s["ds_last"], s0=s["s0"])
    ds = s["ds_last"].clone()
    g1 = ops.decay_attention_backward(s["q"], s["k"], s["v"], s["g"], s["do"], ds_last=ds, s0=s["s0"], ds0=ds)
    assert g1[3] is ds and all(torch.equal(a, b) for a, b in zip(g, g1))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_broadcast_inputs(ops, dtype):
    """Keys shared by all heads (a stride of 0): as if they were copied."""
    T, N, H, D = 150, 2, 4, 64
    s = inputs(T, N, H, D, D, DT[dtype], seed=14)
    k = s["k"][:, :, :1].expand(T, N, H, D)
    a = ops.decay_attention(s["q"], k, s["v"], s["g"], s0=s["s0"])
    b = ops.decay_attention(s["q"], k.contiguous(), s["v"], s["g"], s0=s["s0"])
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    a = ops.decay_attention_backward(s["q"], k, s["v"], s["g"], s["do"], s0=s["s0"])
    b = ops.decay_attention_backward(s["q"], k.contiguous(), s["v"], s["g"], s["do"], s0=s["s0"])
    assert all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_same_bits_again(ops, dtype):
    s = inputs(700, 3, 2, 64, 64, DT[dtype], seed=30, reset=True, lengths=True)
    runs = [ops.decay_attention(s["q"], s["k"], s["v"], s["g"], **masks(s)) +
            ops.decay_attention_backward(s["q"], s["k"], s["v"], s["g"], s["do"], ds_last=s["ds_last"], **masks(s)) for _ in range(3)]
    for r in runs[1:]:
        assert all(torch.equal(x, y) for x, y in zip(r, runs[0]))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("heads", [1, 304])
def test_a_state_of_many_tokens(ops, D, heads):
    """A state that forgets nothing, of 16,384 products that are all positive: what is lost on the way adds up.  Each chunk of 128
    tokens is 24 sums of 16 products and the sum so far, each of the 17 off by less than the last place of it (2^-23 of a chunk's
    state, of half of one in the mean of positive sums): 24 * 17 * 2^-24; adding the chunks up is 128 roundings of 2^-24 of half the
    state in the mean; the products' factors are exact to 2^-24.  (With a head for every place of 152 processors the sequences are
    not split.)"""
    T = 16384
    k = (0.5 + torch.rand(T, 1, 1, D, generator=torch.Generator().manual_seed(1))).bfloat16().cuda().expand(T, 1, heads, D)
    v = (0.5 + torch.rand(T, 1, 1, D, generator=torch.Generator().manual_seed(2))).bfloat16().cuda().expand(T, 1, heads, D)
    _, last = ops.decay_attention(k, k, v, torch.zeros(heads, device="cuda"))
    value = torch.einsum("tk,tv->kv", k[:, 0, 0].double(), v[:, 0, 0].double())
    off = float(((last[0].double() - value) / value).abs().max())
    assert off <= (24 * 17 + 64 + 1) * 2.0 ** -24, off
    ops.sync()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_split_into_more_spans_than_run_at_once(ops, dtype):
    """The gradients of 16 heads of 16,384 tokens, and of the same sequence twenty times over, which are too many to split: each is as
    far from the exact value as near() allows, so that the two are apart by at most twice that."""
    T, H, D = 16384, 16, 64
    s = inputs(T, 1, H, D, D, DT[dtype], seed=40, reset=True)
    one = lambda v: v
    many = lambda v: None if v is None else v.expand(-1, 20, *v.shape[2:]) if v.shape[0] == T else v.expand(20, *v.shape[1:]).contiguous()
    results = []
    for of in (one, many):
        m = {key: of(s[key]) for key in ("q", "k", "v", "do", "s0", "ds_last")}
        reset = of(s["reset"]).contiguous()
        o, last = ops.decay_attention(m["q"], m["k"], m["v"], s["g"], scale=s["scale"], s0=m["s0"], reset=reset)
        dq, dk, dv, ds0 = ops.decay_attention_backward(m["q"], m["k"], m["v"], s["g"], m["do"], scale=s["scale"], s0=m["s0"], reset=reset,
                                                       ds_last=m["ds_last"])
        results.append([o[:, 19 if of is many else 0], dq[:, -1], dk[:, -1], dv[:, -1], last[-1], ds0[-1]])
    for name, a, b in zip(("o", "dq", "dk", "dv", "s_last", "ds0"), *results):
        off = float((a.double() - b.double()).norm() / b.double().norm())
        assert off <= 2 * (1.25 * 2.0 ** -8 if a.dtype == torch.bfloat16 else 32 * ref.U), f"{name}: {off}"
    ops.sync()


def test_offsets_past_32_bits(ops):
    """A view of an array of more than 2^32 values."""
    T, N, H, D = 130, 2, 2, 64
    far = (1 << 32) // 128 + 12345 * 8
    s = inputs(T, N, H, D, D, torch.bfloat16, seed=12)
    big = torch.empty(far * T + N * H * D, dtype=torch.bfloat16, device="cuda")
    k = big.as_strided((T, N, H, D), (far, H * D, D, 1))
    k.copy_(s["k"])
    o = torch.empty_like(big).as_strided((T, N, H, D), (far, H * D, D, 1))
    a = ops.decay_attention(s["q"], s["k"], s["v"], s["g"])
    b = ops.decay_attention(s["q"], k, s["v"], s["g"], out=o)
    assert torch.equal(a[0], o) and torch.equal(a[1], b[1])
    x = ops.head_norm(k, q_out=o)
    assert torch.equal(x, ops.head_norm(s["k"]))


def test_gradient_against_differences(ops):
    T, N, H, Dk, Dv = 20, 2, 2, 6, 5
    s = inputs(T, N, H, Dk, Dv, torch.float32, seed=17)
    s["reset"] = torch.zeros(T, N, dtype=torch.uint8, device="cuda")
    s["reset"][11, 0] = 1
    s["lengths"] = torch.tensor([T, 13], dtype=torch.int32, device="cuda")
    live = (torch.arange(T)[:, None] < s["lengths"].cpu()[None])[..., None, None].cuda()

    def loss(s):
        f = ref.attend(s["q"], s["k"], s["v"], s["g"], s["scale"], **masks(s))
        return float((f["o"][0] * torch.where(live, s["do"], 0.0).cpu().double()).sum() + (f["s_last"][0] * s["ds_last"].cpu().double()).sum())

    got = ops.decay_attention_backward(s["q"], s["k"], s["v"], s["g"], s["do"], scale=s["scale"], ds_last=s["ds_last"], **masks(s))
    for name, grad in zip(("q", "k", "v", "s0"), got):
        way = rnd(*grad.shape, seed=40)
        if name != "s0":
            way = torch.where(live, way, 0.0)
        h = 2.0 ** -12
        # (the loss is bilinear in each of them: a central difference is exact but for the inputs' rounding to fp32)
        a, b = dict(s), dict(s)
        a[name], b[name] = s[name].double() + h * way.double(), s[name].double() - h * way.double()
        diff = (loss(a) - loss(b)) / (2 * h)
        assert abs(diff - float((grad.double() * way.double()).sum())) <= 1e-5 * float((grad.double() * way.double()).abs().sum()), name


# ------------------------------------------------------------------ head norm
def head_inputs(T, N, Hq, Hk, D, rotary, dtype, layout="plain", seed=0, far=False):
    g = torch.Generator().manual_seed(seed)
    s = dict(q=place(rnd(T, N, Hq, D, seed=seed + 1, dtype=dtype, std=2.0), layout),
             k=place(rnd(T, N, Hk, D, seed=seed + 2, dtype=dtype, std=2.0), layout) if Hk else None,
             dq_out=place(rnd(T, N, Hq, D, seed=seed + 3, dtype=dtype), layout), dk_out=place(rnd(T, N, Hk, D, seed=seed + 4, dtype=dtype), layout) if Hk else None,
             q_weight=rnd(D, seed=seed + 5, mean=1.0, std=0.3), k_weight=rnd(D, seed=seed + 6, mean=1.0, std=0.3) if Hk else None,
             positions=None, freqs=None)
    if rotary:
        most = 2 ** 31 - 1 if far else 1000
        s["positions"] = torch.randint(-most, most, (T, N), generator=g, dtype=torch.int32).cuda()
        s["freqs"] = (10000.0 ** (-torch.arange(rotary // 2, dtype=torch.float64) / max(1, rotary // 2))).float().cuda()
    return s


def check_heads(ops, s, interleaved, eps=1e-6, **outs):
    kw = dict(q_weight=s["q_weight"], k_weight=s["k_weight"], positions=s["positions"], freqs=s["freqs"], eps=eps, interleaved=interleaved)
    got = ops.head_norm(s["q"], s["k"], **kw)
    got = got if s["k"] is not None else (got,)
    back = ops.head_norm_backward(s["q"], s["dq_out"], s["k"], s["dk_out"], **kw, **outs)
    for i, name in enumerate("qk"[:len(got)]):
        args = (s[name], s[name + "_weight"], eps, s["positions"], s["freqs"], interleaved)
        check(got[i], *ref.head_norm(*args), name)
        b = ref.head_norm_backward(*args, s["d" + name + "_out"])
        check(back[i], *b["dx"], "d" + name)
        check(back[2 + i], *b["dw"], "d" + name + "_weight")
    ops.sync()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,rotary", [(1, 0), (2, 2), (3, 2), (8, 8), (16, 8), (43, 22), (43, 42), (64, 64), (64, 0), (64, 36), (96, 96), (128, 128), (128, 20),
                                      (256, 256), (300, 100), (512, 512), (1000, 1000), (1023, 10), (1024, 1024), (1024, 2)])
def test_head_norm(ops, dtype, interleaved, D, rotary):
    check_heads(ops, head_inputs(5, 3, 3, 2, D, rotary, DT[dtype], seed=D + rotary), interleaved)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("T,N,Hq,Hk", [(1, 1, 1, 0), (1, 1, 1, 1), (1, 7, 16, 1), (300, 4, 2, 2), (64, 9, 5, 0), (2000, 3, 4, 1)])
def test_head_norm_heads(ops, dtype, T, N, Hq, Hk):
    check_heads(ops, head_inputs(T, N, Hq, Hk, 64, 64, DT[dtype], seed=T, far=True), T % 2 == 0)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("layout", ["columns", "batch", "heads", "shifted"])
@pytest.mark.parametrize("D,rotary,interleaved", [(64, 64, False), (40, 16, True), (43, 22, False)])
def test_head_norm_layouts(ops, dtype, layout, D, rotary, interleaved):
    T, N = 33, 3
    s = head_inputs(T, N, 4, 2, D, rotary, DT[dtype], layout, seed=3)
    wide = torch.full((T, N, 6 * D + 8), 7.0, dtype=DT[dtype], device="cuda")
    dq, dk = (p.unflatten(-1, (-1, D)) for p in wide[..., :-8].split([4 * D, 2 * D], -1))
    check_heads(ops, s, interleaved, dq=dq, dk=dk)
    assert (wide[..., -8:] == 7.0).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_head_norm_in_place(ops, dtype):
    s = head_inputs(50, 3, 4, 2, 64, 64, DT[dtype], seed=5)
    kw = dict(q_weight=s["q_weight"], k_weight=s["k_weight"], positions=s["positions"], freqs=s["freqs"])
    want = ops.head_norm(s["q"], s["k"], **kw)
    back = ops.head_norm_backward(s["q"], s["dq_out"], s["k"], s["dk_out"], **kw)
    a, b = s["dq_out"].clone(), s["dk_out"].clone()
    got = ops.head_norm_backward(s["q"], a, s["k"], b, dq=a, dk=b, **kw)
    assert got[0] is a and all(torch.equal(x, y) for x, y in zip(got, back))
    q, k = ops.head_norm(s["q"], s["k"], q_out=s["q"], k_out=s["k"], **kw)
    assert q is s["q"] and torch.equal(q, want[0]) and torch.equal(k, want[1])


def test_head_norm_one_step_and_rows(ops):
    """[N, heads, D] of one step is a step of [T, N, heads, D]; a row of zeros, of huge and of tiny values."""
    s = head_inputs(4, 3, 2, 2, 64, 64, torch.float32, seed=6)
    kw = dict(q_weight=s["q_weight"], k_weight=s["k_weight"], freqs=s["freqs"])
    q, k = ops.head_norm(s["q"], s["k"], positions=s["positions"], **kw)
    for t in range(4):
        a, b = ops.head_norm(s["q"][t], s["k"][t], positions=s["positions"][t], **kw)
        assert torch.equal(a, q[t]) and torch.equal(b, k[t])
    s["q"][0, 0, 0] = 0.0
    s["q"][1, 0, 0] *= 1e15
    s["q"][2, 0, 0] *= 1e-12
    check_heads(ops, s, False)


def test_head_norm_not_finite(ops):
    """A bad row is its own; a frequency that is none spoils its pair alone."""
    s = head_inputs(6, 2, 2, 1, 32, 32, torch.float32, seed=7)
    kw = dict(q_weight=s["q_weight"], k_weight=s["k_weight"], positions=s["positions"])
    want = ops.head_norm(s["q"], s["k"], freqs=s["freqs"], **kw)
    q = s["q"].clone()
    q[3, 1, 0, 5] = float("nan")
    got = ops.head_norm(q, s["k"], freqs=s["freqs"], **kw)
    assert torch.isnan(got[0][3, 1, 0]).all()
    got[0][3, 1, 0] = want[0][3, 1, 0]
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    for f in (float("nan"), float("inf")):
        freqs = s["freqs"].clone()
        freqs[4] = f
        got = ops.head_norm(s["q"], s["k"], freqs=freqs, **kw)[0]
        assert torch.isnan(got[..., [4, 20]]).all()
        rest = [i for i in range(32) if i not in (4, 20)]
        assert torch.equal(got[..., rest], want[0][..., rest])


def test_head_norm_empty(ops):
    e = torch.empty(0, 2, 3, 8, device="cuda")
    pos, f = torch.empty(0, 2, dtype=torch.int32, device="cuda"), torch.ones(4, device="cuda")
    assert ops.head_norm(e, positions=pos, freqs=f).shape == e.shape
    dq, none, dw, _ = ops.head_norm_backward(e, e, positions=pos, freqs=f)
    assert dq.shape == e.shape and none is None and (dw == 0).all()


def test_head_norm_gradient_against_differences(ops):
    s = head_inputs(3, 2, 2, 1, 12, 8, torch.float32, seed=8)
    for interleaved in (False, True):
        kw = dict(positions=s["positions"], freqs=s["freqs"], interleaved=interleaved)
        back = ops.head_norm_backward(s["q"], s["dq_out"], s["k"], s["dk_out"], q_weight=s["q_weight"], k_weight=s["k_weight"], **kw)

        def loss(x, w):
            y = ref.head_norm(x, w, 1e-6, s["positions"], s["freqs"], interleaved)[0]
            return float((y * s["dq_out"].cpu().double()).sum())

        x, w = s["q"].double().cpu(), s["q_weight"].double().cpu()
        h = 1e-5
        wx, ww = rnd(*x.shape, seed=50).double().cpu(), rnd(*w.shape, seed=51).double().cpu()
        dx = (loss(x + h * wx, w) - loss(x - h * wx, w)) / (2 * h)
        dw = (loss(x, w + h * ww) - loss(x, w - h * ww)) / (2 * h)
        for diff, grad, way in ((dx, back[0], wx), (dw, back[2], ww)):
            prod = grad.double().cpu() * way
            assert abs(diff - float(prod.sum())) <= 1e-5 * float(prod.abs().sum())


# ------------------------------------------------------------------ both, and around them
def test_a_block_of_them(ops):
    """Norm and rotation, attention over a recording, and all the way back, against torch's derivatives of the definition."""
    T, N, H, D = 70, 2, 2, 16
    x = {n: rnd(T, N, H, D, seed=60 + i) for i, n in enumerate("qkv")}
    wq, wk = rnd(D, seed=64, mean=1.0, std=0.2), rnd(D, seed=65, mean=1.0, std=0.2)
    pos = torch.arange(T, dtype=torch.int32)[:, None].expand(T, N).contiguous().cuda()
    f = (0.1 ** torch.arange(D // 2, dtype=torch.float64)).float().cuda()
    g, do = decays(H), rnd(T, N, H, D, seed=66)
    kw = dict(q_weight=wq, k_weight=wk, positions=pos, freqs=f)
    q, k = ops.head_norm(x["q"], x["k"], **kw)
    o, _ = ops.decay_attention(q, k, x["v"], g, scale=0.25)
    dq, dk, dv, _ = ops.decay_attention_backward(q, k, x["v"], g, do, scale=0.25)
    dq, dk, dwq, dwk = ops.head_norm_backward(x["q"], dq, x["k"], dk, dq=dq, dk=dk, **kw)
    leaf = [t.detach().cpu().double().requires_grad_() for t in (x["q"], x["k"], x["v"], wq, wk)]

    def turned(v, w):
        y = v / torch.sqrt(v.square().mean(-1, keepdim=True) + 1e-6) * w
        ang = pos.cpu().double()[..., None, None] * f.cpu().double()
        a, b = y[..., :D // 2], y[..., D // 2:]
        return torch.cat([a * torch.cos(ang) - b * torch.sin(ang), b * torch.cos(ang) + a * torch.sin(ang)], -1)

    qq, kk = turned(leaf[0], leaf[3]), turned(leaf[1], leaf[4])
    away = torch.arange(T)[:, None] - torch.arange(T)[None]
    w = torch.where(away >= 0, torch.exp(g.cpu().double()[:, None, None] * away.clamp(min=0)), 0.0)
    want = 0.25 * torch.einsum("tnhd,snhd,hts,snhe->tnhe", qq, kk, w, leaf[2])
    want.backward(do.cpu().double())
    for got, ex in ((o, want.detach()), (dq, leaf[0].grad), (dk, leaf[1].grad), (dv, leaf[2].grad), (dwq, leaf[3].grad), (dwk, leaf[4].grad)):
        assert float((got.cpu().double() - ex).norm() / ex.norm()) <= 64 * ref.U


def test_other_stream(ops):
    s = inputs(300, 2, 2, 64, 64, torch.bfloat16, seed=70)
    h = head_inputs(50, 2, 2, 2, 64, 64, torch.bfloat16, seed=71)
    kw = dict(positions=h["positions"], freqs=h["freqs"])
    want = ops.decay_attention(s["q"], s["k"], s["v"], s["g"]) + ops.decay_attention_backward(s["q"], s["k"], s["v"], s["g"], s["do"])
    want += ops.decay_step(s["q"][0], s["k"][0], s["v"][0], s["g"], s["s0"])
    want += ops.head_norm(h["q"], h["k"], **kw) + ops.head_norm_backward(h["q"], h["dq_out"], h["k"], h["dk_out"], **kw)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    got = ops.decay_attention(s["q"], s["k"], s["v"], s["g"], stream=st) + ops.decay_attention_backward(s["q"], s["k"], s["v"], s["g"], s["do"], stream=st)
    got += ops.decay_step(s["q"][0], s["k"][0], s["v"][0], s["g"], s["s0"], stream=st)
    got += ops.head_norm(h["q"], h["k"], stream=st, **kw) + ops.head_norm_backward(h["q"], h["dq_out"], h["k"], h["dk_out"], stream=st, **kw)
    torch.cuda.current_stream().wait_stream(st)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_graph_capture(seq):
    """All calls captured in one graph, replayed on new inputs; the workspace grows in between and the graph stays valid."""
    ops = seq.SequenceOps()
    s = inputs(900, 1, 2, 64, 64, torch.bfloat16, seed=80)
    h = head_inputs(30, 2, 2, 2, 64, 64, torch.bfloat16, seed=81)

    def calls():
        r = ops.decay_attention(s["q"], s["k"], s["v"], s["g"], s0=s["s0"])
        r += ops.decay_attention_backward(s["q"], s["k"], s["v"], s["g"], s["do"], ds_last=s["ds_last"], s0=s["s0"])
        r += ops.decay_step(s["q"][0], s["k"][0], s["v"][0], s["g"], s["s0"])
        r += ops.head_norm(h["q"], h["k"], positions=h["positions"], freqs=h["freqs"])
        return r + ops.head_norm_backward(h["q"], h["dq_out"], h["k"], h["dk_out"], positions=h["positions"], freqs=h["freqs"])

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        calls()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = calls()
    big = inputs(6000, 1, 2, 128, 128, torch.bfloat16, seed=82)
    ops.decay_attention(big["q"], big["k"], big["v"], big["g"])
    for i in range(2):
        for v in (s["q"], s["v"], s["s0"], h["q"]):
            v.copy_(torch.randn(v.shape, generator=torch.Generator().manual_seed(i)).to(v.dtype))
        graph.replay()
        torch.cuda.synchronize()
        want = calls()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
    ops.sync()


def test_two_graphs_share_a_workspace(seq):
    """Captured on one handle and replayed in turn: neither reads what the other left."""
    ops = seq.SequenceOps()
    a, b = (inputs(1500, 1, 2, D, D, torch.bfloat16, seed=85 + D) for D in (64, 128))

    def calls(s):
        return ops.decay_attention(s["q"], s["k"], s["v"], s["g"], s0=s["s0"]) + ops.decay_attention_backward(s["q"], s["k"], s["v"], s["g"], s["do"])

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        want = [calls(s) for s in (b, a)]
    side.synchronize()
    graphs, outs = [], []
    for s in (b, a):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            outs.append(calls(s))
        graphs.append(g)
    for i in (0, 1, 1, 0, 1):
        for v in outs[i]:
            v.fill_(float("nan"))
        graphs[i].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(outs[i], want[i]))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("T", [11, 13, 20, 32, 33])
def test_many_sequences_of_few_tokens(ops, dtype, T):
    """Token by token, or in chunks: by type and by how many there are."""
    check_all(ops, inputs(T, 110, 3, 16, 24, DT[dtype], seed=T, reset=True, lengths=True))


def test_threads_take_turns(ops):
    """Two threads on one handle: each call whole."""
    import threading
    s = inputs(300, 2, 2, 64, 64, torch.bfloat16, seed=33)
    want = ops.decay_attention(s["q"], s["k"], s["v"], s["g"], s0=s["s0"])
    bad = []

    def work():
        for _ in range(20):
            got = ops.decay_attention(s["q"], s["k"], s["v"], s["g"], s0=s["s0"])
            if not all(torch.equal(x, y) for x, y in zip(got, want)):
                bad.append(1)

    threads = [threading.Thread(target=work) for _ in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not bad


def test_capture_needs_a_workspace(seq):
    ops = seq.SequenceOps()
    s = inputs(3000, 1, 1, 64, 64, torch.bfloat16, seed=83)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with pytest.raises(seq.WMError, match="capture"):
        with torch.cuda.graph(graph, stream=side):
            ops.decay_attention(s["q"], s["k"], s["v"], s["g"])
    torch.cuda.synchronize()


def test_refusals(ops, seq):
    s = inputs(4, 2, 2, 8, 8, torch.float32, seed=90)
    q, k, v, g = s["q"], s["k"], s["v"], s["g"]
    for args in ((q.half(), k, v, g), (q, k.bfloat16(), v, g), (q, k[..., :4], v, g), (q, k, v[:2], g), (q, k, v, g[:1]), (q, k, v, g.double()),
                 (q[0], k[0], v[0], g), (q.transpose(2, 3).contiguous().transpose(2, 3), k, v, g)):
        with pytest.raises(ValueError):
            ops.decay_attention(*args)
    for kw in (dict(s0=s["s0"][0]), dict(s0=s["s0"].transpose(-1, -2)[:, :, :4]), dict(reset=torch.zeros(4, 2, device="cuda")), dict(lengths=torch.zeros(2, device="cuda")),
               dict(out=torch.empty(4, 2, 2, 9, device="cuda")), dict(s_last=torch.empty(1, device="cuda"))):
        with pytest.raises(ValueError):
            ops.decay_attention(q, k, v, g, **kw)
    with pytest.raises(seq.WMError, match="overlap"):
        ops.decay_attention(q, k, v, g, out=torch.empty(4, 1, 2, 8, device="cuda").expand(4, 2, 2, 8))
    with pytest.raises(seq.WMError, match="scale"):
        ops.decay_attention(q, k, v, g, scale=float("nan"))
    with pytest.raises(seq.WMError, match="device"):
        ops.decay_attention(q, k, v, g.cpu())
    wide = torch.empty(1, 1, 1, 257, device="cuda")
    with pytest.raises(seq.WMError, match="256"):
        ops.decay_attention(wide, wide, wide, g[:1])
    with pytest.raises(ValueError):
        ops.decay_step(q, k, v, g, s["s0"])
    with pytest.raises(ValueError):
        ops.decay_attention_backward(q, k, v, g, s["do"][:2])
    h = head_inputs(4, 2, 2, 1, 8, 8, torch.float32, seed=91)
    kw = dict(positions=h["positions"], freqs=h["freqs"])
    for bad in (dict(positions=h["positions"]), dict(freqs=h["freqs"]), dict(kw, freqs=torch.ones(5, device="cuda")), dict(kw, positions=h["positions"].long()),
                dict(q_weight=torch.ones(7, device="cuda")), dict(k_weight=torch.ones(8, device="cuda")), dict(k=h["k"].bfloat16()),
                dict(k=h["k"][0]), dict(q_out=torch.empty(1, device="cuda"))):
        with pytest.raises(ValueError):
            ops.head_norm(h["q"], **bad)
    with pytest.raises(seq.WMError, match="eps"):
        ops.head_norm(h["q"], eps=-1.0)
    with pytest.raises(seq.WMError, match="strides"):
        x = torch.empty(8 * 2 * 2 * 8, device="cuda")
        ops.head_norm(x.as_strided((4, 2, 2, 8), (32, 16, 8, 1)), q_out=x.as_strided((4, 2, 2, 8), (64, 16, 8, 1)))
    with pytest.raises(seq.WMError, match="1024"):
        ops.head_norm(torch.empty(1, 1, 1, 1025, device="cuda"))
    with pytest.raises(ValueError):
        ops.head_norm_backward(h["q"], h["dq_out"], h["k"], None)
    ops.sync()
