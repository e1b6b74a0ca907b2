"""Decayed linear attention: what runs side by side in its kernels, states at the edge of their precision, decays and values that
are not finite, waits that give up, calls that are refused; angles of the head norm."""
import pytest
import torch

import decay_reference as ref
from seq_reference import check
from test_gpu_decay import DT, inputs, masks, near, ops, rnd, seq  # noqa: F401  (fixtures among them)

pytestmark = pytest.mark.gpu


def both_ways(ops, s):
    """Outputs and gradients of a call, by name."""
    o, last = ops.decay_attention(s["q"], s["k"], s["v"], s["g"], scale=s["scale"], **masks(s))
    g = ops.decay_attention_backward(s["q"], s["k"], s["v"], s["g"], s["do"], scale=s["scale"], ds_last=s["ds_last"], **masks(s))
    return dict(zip(("o", "s_last", "dq", "dk", "dv", "ds0"), (o, last, *g)))


def copies(s, n):
    """The same sequence n times over (N = 1)."""
    out = dict(s)
    for key in ("q", "k", "v", "do"):
        out[key] = s[key].expand(-1, n, -1, -1).contiguous()
    for key in ("s0", "ds_last"):
        out[key] = s[key].expand(n, -1, -1, -1).contiguous()
    return out


# ------------------------------------------------------------------ side by side
@pytest.mark.parametrize("T,H,Dk,Dv,n", [(130, 8, 128, 128, 60), (13, 8, 128, 128, 60), (300, 4, 128, 64, 100), (200, 4, 72, 128, 100),
                                         (1100, 2, 128, 128, 1), (2600, 1, 96, 128, 1)])
def test_wide_heads_take_their_states_whole(ops, T, H, Dk, Dv, n):
    """States of more than 64 values that enter without resets, more heads of sequences than run at once or spans of time: each copy of
    a sequence, and each call again, gives the same bits, and what the definition gives."""
    s = inputs(T, 1, H, Dk, Dv, torch.bfloat16, seed=T)
    got = both_ways(ops, copies(s, n))
    f = ref.attend(s["q"], s["k"], s["v"], s["g"], s["scale"], **masks(s))
    b = ref.attend_backward(s["q"], s["k"], s["v"], s["g"], s["scale"], s["do"], s["ds_last"], **masks(s))
    for name, value in got.items():
        axis = 0 if name in ("s_last", "ds0") else 1
        first = value.narrow(axis, 0, 1)
        assert torch.equal(value, first.expand_as(value)), name
        check(first, *{**f, **b}[name], name)
        near(first, {**f, **b}[name][0], name, value.dtype)
    for _ in range(3 if n > 1 else 12):
        again = both_ways(ops, copies(s, n))
        for name, value in got.items():
            assert torch.equal(value, again[name]), name
    ops.sync()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T,state", [(14, False), (128, True), (257, False)])
def test_keys_are_there_when_they_are_weighted(ops, D, T, state):
    """Items of one to three chunks, one after the other on each processor: what the keys give the states (and, by them, the outputs)
    is the same in each copy of a sequence and in each call, and what the definition gives."""
    s = inputs(T, 1, 4, D, D, torch.bfloat16, seed=100 + T, state=state)
    if not state:
        s["s0"] = s["ds_last"] = torch.zeros(1, 4, D, D, device="cuda")
    c = copies(s, 300)
    if not state:
        for v in (s, c):
            v["s0"] = v["ds_last"] = None
    got = both_ways(ops, c)
    f = ref.attend(s["q"], s["k"], s["v"], s["g"], s["scale"], **masks(s))
    b = ref.attend_backward(s["q"], s["k"], s["v"], s["g"], s["scale"], s["do"], s["ds_last"], **masks(s))
    for name, value in got.items():
        first = value.narrow(0 if name in ("s_last", "ds0") else 1, 0, 1)
        assert torch.equal(value, first.expand_as(value)), name
        check(first, *{**f, **b}[name], name)
        near(first, {**f, **b}[name][0], name, value.dtype)
    again = both_ways(ops, c)
    assert all(torch.equal(v, again[name]) for name, v in got.items())
    ops.sync()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("N,Dk,Dv", [(1, 1, 1), (2, 3, 5), (3, 43, 43), (1, 256, 31), (2, 33, 64), (200, 20, 66), (400, 64, 72), (1, 7, 256)])
def test_steps_of_any_width(ops, dtype, N, Dk, Dv):
    """Single tokens whose values fill a CTA's columns in part, 32 and 64 columns wide, with the state in place."""
    s = inputs(3, N, 2, Dk, Dv, DT[dtype], seed=Dk + Dv)
    f = ref.attend(s["q"], s["k"], s["v"], s["g"], s["scale"], s["s0"], factors=False)
    state = s["s0"].clone()
    for t in range(3):
        o, _ = ops.decay_step(s["q"][t], s["k"][t], s["v"][t], s["g"], state, scale=s["scale"], out_state=state)
        check(o, f["o"][0][t], f["o"][1][t], "o")
    check(state, *f["s_last"], "state")
    ops.sync()


# ------------------------------------------------------------------ waits that give up
@pytest.mark.parametrize("layout,masked", [("plain", False), ("plain", True), ("shifted", False), ("shifted", True)])
@pytest.mark.parametrize("T,N,H,D", [(70, 3, 2, 64), (300, 2, 2, 64), (500, 1, 3, 128), (300, 250, 2, 128), (2000, 1, 2, 64), (1500, 1, 1, 128)])
def test_a_wait_gives_up(seq, T, N, H, D, layout, masked):
    """A wait that nothing completes, with copies and products on their way: the call ends by its limit with all its warps, the
    timeout is reported once, and the same call then gives what it gave before.  Copies and plain loads, one span and several."""
    ops = seq.SequenceOps()
    s = inputs(T, N, H, D, D, torch.bfloat16, layout, seed=T + D, reset=masked, lengths=masked and N > 1)
    want = both_ways(ops, s)
    ops.sync()
    calls = (lambda: ops.decay_attention(s["q"], s["k"], s["v"], s["g"], **masks(s)),
             lambda: ops.decay_attention_backward(s["q"], s["k"], s["v"], s["g"], s["do"], ds_last=s["ds_last"], **masks(s)))
    for call in calls:
        ops.inject_wait_timeout(1000)
        call()
        with pytest.raises(seq.WMError) as e:
            ops.sync()
        assert e.value.status == 4
        ops.sync()
    got = both_ways(ops, s)
    ops.sync()
    assert all(torch.equal(v, got[name]) for name, v in want.items())


# ------------------------------------------------------------------ decays and values that are not finite
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("T", [5, 20, 100, 300, 1500])
def test_a_decay_that_is_no_number(ops, dtype, T):
    """It spoils all tokens of its head that see another one, with states and without, and no other head."""
    s = inputs(T, 2, 2, 64, 64, DT[dtype], seed=50, state=False)
    args = s["q"], s["k"], s["v"]
    want = ops.decay_attention(*args, s["g"], want_last=False)[0], *ops.decay_attention_backward(*args, s["g"], s["do"], want_ds0=False)[:3]
    g = s["g"].clone()
    g[0] = float("nan")
    got = ops.decay_attention(*args, g, want_last=False)[0], *ops.decay_attention_backward(*args, g, s["do"], want_ds0=False)[:3]
    for name, value, clean in zip(("o", "dq", "dk", "dv"), got, want):
        assert torch.isnan(value[:-1, :, 0] if name in ("dk", "dv") else value[1:, :, 0]).all(), name
        assert torch.equal(value[:, :, 1], clean[:, :, 1]), name
    ops.sync()


def same(got, want, what, dtype):
    """As good as equal: what is not finite is taken again another way, with roundings of its own."""
    if got.numel():
        assert torch.isfinite(got).all(), what
        off = float((got.double() - want.double()).abs().max())
        assert off <= (4.0 * ref.B if dtype == torch.bfloat16 else 1e-5) * float(want.double().abs().max()), f"{what}: {off}"


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("T", [2, 5, 40, 300, 1500])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
@pytest.mark.parametrize("reset", [False, True])
def test_only_the_token_itself(ops, dtype, T, bad, reset):
    """A head that keeps nothing (log_decay = -inf): a token's bad values, and a bad state, reach no other token."""
    dt = DT[dtype]
    s = inputs(T, 2, 2, 64, 64, dt, seed=51, reset=reset)
    s["g"] = torch.tensor([-float("inf"), -0.01], device="cuda")
    want, at = both_ways(ops, s), T // 3
    assert (want["ds0"][:, 0] == 0).all()
    others, not_last = torch.arange(T) != at, torch.arange(T) != T - 1

    def spoiled(name, *where):
        t = dict(s)
        t[name] = s[name].clone()
        t[name][where] = bad
        return both_ways(ops, t)

    for name, alone in (("q", ("o", "dk")), ("k", ("o", "dq", "dv")), ("v", ("o", "dq", "dk")), ("do", ("dq", "dk", "dv"))):
        got = spoiled(name, at, 0, 0, 3)
        for out in ("o", "dq", "dk", "dv"):
            same(got[out][others, 0, 0], want[out][others, 0, 0], f"{out} of {name}", dt)
            same(got[out][:, 1], want[out][:, 1], f"{out} of {name}, another sequence", dt)
            if out in alone:
                assert not torch.isfinite(got[out][at, 0, 0]).all(), f"{out} of {name}"
        if at < T - 1:
            same(got["s_last"][:, 0], want["s_last"][:, 0], f"s_last of {name}", torch.float32)
        assert (got["ds0"][:, 0] == 0).all(), name
    got = spoiled("s0", 0, 0)
    for out in ("o", "s_last", "dq", "dk", "dv"):
        axis = 1 if out == "s_last" else 2
        same(got[out].select(axis, 0), want[out].select(axis, 0), f"{out} of s0", dt)
    got = spoiled("ds_last", 0, 0)
    for out in ("o", "dq"):
        same(got[out][:, :, 0], want[out][:, :, 0], f"{out} of ds_last", dt)
    for out in ("dk", "dv"):
        same(got[out][not_last, :, 0], want[out][not_last, :, 0], f"{out} of ds_last", dt)
        assert not torch.isfinite(got[out][T - 1, 0, 0]).any(), out
    assert (got["ds0"][:, 0] == 0).all()
    ops.sync()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("T,N", [(5, 2), (40, 2), (200, 2), (2600, 1)])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_what_is_not_finite_does_not_wear_off(ops, dtype, T, N, bad):
    """However small its weight has become (0 in fp32): what is not finite reaches all that sees it, and the state."""
    s = inputs(T, N, 2, 64, 64, DT[dtype], seed=52)
    s["g"] = torch.tensor([-2.0, -30.0], device="cuda")

    def spoiled(name, *where):
        t = dict(s)
        t[name] = s[name].clone()
        t[name][where] = bad
        return both_ways(ops, t)

    def none(x, what):
        assert not torch.isfinite(x).any(), what

    for h in range(2):
        got = spoiled("k", 1, 0, h, 3)
        none(got["o"][1:, 0, h], "o of k")
        none(got["s_last"][0, h, 3], "s_last of k")
        none(got["dq"][1:, 0, h, 3], "dq of k")
        got = spoiled("v", 1, 0, h, 3)
        none(got["o"][1:, 0, h, 3], "o of v")
        none(got["s_last"][0, h, :, 3], "s_last of v")
        none(got["dq"][1:, 0, h], "dq of v")
        got = spoiled("s0", 0, h, 3, 3)
        none(got["o"][:, 0, h, 3], "o of s0")
        none(got["s_last"][0, h, 3, 3], "s_last of s0")
        none(got["dq"][:, 0, h, 3], "dq of s0")
        got = spoiled("do", T - 2, 0, h, 3)
        none(got["dk"][:T - 1, 0, h], "dk of do")
        none(got["dv"][:T - 1, 0, h, 3], "dv of do")
        none(got["ds0"][0, h, :, 3], "ds0 of do")
        got = spoiled("q", T - 2, 0, h, 3)
        none(got["dk"][:T - 1, 0, h, 3], "dk of q")
        none(got["dv"][:T - 1, 0, h], "dv of q")
        none(got["ds0"][0, h, 3], "ds0 of q")
        got = spoiled("ds_last", 0, h, 3, 3)
        none(got["dk"][:, 0, h, 3], "dk of ds_last")
        none(got["dv"][:, 0, h, 3], "dv of ds_last")
        none(got["ds0"][0, h, 3, 3], "ds0 of ds_last")
    ops.sync()


# ------------------------------------------------------------------ the state's precision
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T,tail,rate", [(192, 64, -0.05), (320, 190, -0.05), (384, 128, -0.5), (2000, 300, -0.02)])
def test_a_state_after_tokens_that_write_nothing(ops, dtype, D, T, tail, rate):
    """Keys that are zeros at the end (and queries at the start, for the gradient of the entering state): the state that leaves has decayed
    and is as good as it was.  Beside what near() allows it its factors are off by U / 2 of their exponents, which are rate * tail in all,
    and the exponential and the product by 3 U each of the chunks that it lay still: of 64 tokens at least.  One call, and two that are cut
    where the keys end, are each as good as that."""
    N, H = 1, 2
    s = inputs(T, N, H, D, D, DT[dtype], seed=53, state=False)
    s["g"] = torch.tensor([rate, rate / 3], device="cuda")
    s["k"][T - tail:] = 0
    s["q"][:tail] = 0
    s["ds_last"] = None
    f = ref.attend(s["q"], s["k"], s["v"], s["g"], s["scale"], **masks(s))["s_last"][0]
    b = ref.attend_backward(s["q"], s["k"], s["v"], s["g"], s["scale"], s["do"], **masks(s))["ds0"][0]
    got = both_ways(ops, s)
    _, first = ops.decay_attention(s["q"][:T - tail], s["k"][:T - tail], s["v"][:T - tail], s["g"])
    _, parts = ops.decay_attention(s["q"][T - tail:], s["k"][T - tail:], s["v"][T - tail:], s["g"], s0=first)
    for h in range(H):
        most = (32 + 0.5 * abs(float(s["g"][h])) * (tail + 128) + 3 * (tail // 64 + 2)) * ref.U
        for what, value, exact in (("s_last", got["s_last"], f), ("s_last of parts", parts, f), ("ds0", got["ds0"], b)):
            off = float((value[:, h].cpu().double() - exact[:, h]).norm() / exact[:, h].norm())
            assert off <= most, f"{what}, head {h}: {off} of {most}"
    ops.sync()


# ------------------------------------------------------------------ refusals
def test_an_output_is_no_other_array(ops, seq):
    """Three passes read what one writes, and a sequence may be taken again: refused, with the outputs as they were."""
    for T, dtype in ((8, torch.float32), (40, torch.bfloat16)):
        s = inputs(T, 2, 2, 8, 8, dtype, seed=70)
        q, k, v, do, g = s["q"], s["k"], s["v"], s["do"], s["g"]
        given = {name: x.clone() for name, x in s.items() if torch.is_tensor(x)}
        for x in (q, k, v):
            with pytest.raises(seq.WMError, match="another array"):
                ops.decay_attention(q, k, v, g, out=x)
        if dtype == torch.float32:
            with pytest.raises(seq.WMError, match="another array"):
                ops.decay_attention(q, k, v, g, s_last=q.flatten()[:256].view(2, 2, 8, 8))
        for x in (q, k, v, do):
            for name in ("dq", "dk", "dv"):
                with pytest.raises(seq.WMError, match="another array"):
                    ops.decay_attention_backward(q, k, v, g, do, **{name: x})
        x = torch.empty_like(q)
        for a, b in (("dq", "dk"), ("dq", "dv"), ("dk", "dv")):
            with pytest.raises(seq.WMError, match="another array"):
                ops.decay_attention_backward(q, k, v, g, do, **{a: x, b: x})
        with pytest.raises(seq.WMError, match="another array"):
            ops.decay_attention_backward(q, k, v, g, do, s0=s["s0"], ds_last=s["ds_last"], ds0=s["s0"])
        for name, x in given.items():
            assert torch.equal(s[name], x), name
        # side by side in one buffer is not the same array
        wide = torch.empty(T, 2, 2, 24, dtype=dtype, device="cuda")
        dq, dk, dv = wide.split(8, -1)
        got = ops.decay_attention_backward(q, k, v, g, do, dq=dq, dk=dk, dv=dv)
        assert all(torch.equal(a, b) for a, b in zip(got[:3], ops.decay_attention_backward(q, k, v, g, do)))
    x, y, dx, dy = (rnd(4, 2, 2, 8, seed=71 + i) for i in range(4))
    given = [t.clone() for t in (x, y, dx, dy)]
    z = torch.empty_like(x)
    for kw in (dict(q_out=y), dict(k_out=x), dict(q_out=z, k_out=z), dict(q_out=x, k_out=x)):
        with pytest.raises(seq.WMError, match="another array"):
            ops.head_norm(x, y, **kw)
    for kw in (dict(dq=y), dict(dk=x), dict(dq=dy), dict(dk=dx), dict(dq=z, dk=z)):
        with pytest.raises(seq.WMError, match="another array|must not be"):
            ops.head_norm_backward(x, dx, y, dy, **kw)
    assert all(torch.equal(a, b) for a, b in zip((x, y, dx, dy), given))
    ops.sync()


# ------------------------------------------------------------------ head norm
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
def test_angles_of_negative_frequencies(ops, dtype, interleaved):
    """A turn back is a turn by the negative position: the same bits, at any position and frequency."""
    T, N, H, D = 40, 3, 2, 64
    q, dy = rnd(T, N, H, D, seed=60, dtype=DT[dtype]), rnd(T, N, H, D, seed=61, dtype=DT[dtype])
    pos = torch.randint(-2 ** 31 + 1, 2 ** 31 - 1, (T, N), generator=torch.Generator().manual_seed(62), dtype=torch.int32).cuda()
    pos[0] = 2 ** 31 - 1
    f = (10.0 ** -torch.linspace(0, 12, D // 2, dtype=torch.float64)).float().cuda()
    a = ops.head_norm(q, positions=pos, freqs=-f, interleaved=interleaved)
    b = ops.head_norm(q, positions=-pos, freqs=f, interleaved=interleaved)
    assert torch.equal(a, b)
    a = ops.head_norm_backward(q, dy, positions=pos, freqs=-f, interleaved=interleaved)
    b = ops.head_norm_backward(q, dy, positions=-pos, freqs=f, interleaved=interleaved)
    assert torch.equal(a[0], b[0]) and torch.equal(a[2], b[2])


def test_angles_next_to_a_quarter_turn(ops):
    """Where a cosine or a sine is below 1e-4 its error is the angle's: |position * frequency| 2^-53 by the frequency as a fraction of a turn,
    2^-33 turns of fixed point, and in all 16 U of the value itself by the functions, the norm and the products (the other side of
    the pair is 0, so that there is one product)."""
    import math
    pos, near_0 = [], []
    for p in range(1, 400000):
        for k, f in enumerate((math.cos, math.sin)):
            if abs(f(float(p))) < 1e-4:
                pos.append(p)
                near_0.append(k)
    pos, near_0 = torch.tensor(pos, dtype=torch.int32), torch.tensor(near_0)
    assert len(pos) > 40 and 0 < int(near_0.sum()) < len(pos)
    x = torch.zeros(len(pos), 1, 1, 2, device="cuda")
    x[..., 0] = 1.0
    for sign in (1.0, -1.0):
        y = ops.head_norm(x, positions=pos[:, None].cuda(), freqs=torch.full((1,), sign, device="cuda"), eps=0.0).cpu().double()[:, 0, 0]
        # (x / sqrt(1 / 2): off by 4 U)
        got = torch.where(near_0 == 0, y[:, 0], y[:, 1]) / math.sqrt(2.0)
        want = torch.where(near_0 == 0, torch.cos(pos.double()), sign * torch.sin(pos.double()))
        most = pos.double() * 2.0 ** -53 + 2 * math.pi * 2.0 ** -33 + 16 * ref.U * want.abs() + 1e-11  # (cosines of 64 bits in the last)
        off = (got - want).abs()
        assert (off <= most).all(), float((off / most).max())
    ops.sync()
