"""The sequence operators against their definitions in 64 bits (tests/seq_reference.py, which also
gives the error an fp32 evaluation may have), at the sizes and masks where they can go wrong, their
gradients against differences, and what they refuse."""
import math

import pytest
import torch

import seq_reference as ref

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


def scan_inputs(T, N, H, dtype, layout="plain", seed=0, reset=False, lengths=False, mean=2.0):
    """gate, x, dh [T, N, H] in a layout, with what a call may leave out."""
    def place(i, mean, std=1.0):
        v = rnd(T, N, H, seed=seed + i, dtype=dtype, mean=mean, std=std)
        if layout == "plain":
            return v
        if layout == "columns":  # columns of a wider array
            w = torch.full((T, N, 2 * H + 8), float("nan"), dtype=dtype, device="cuda")
            w[..., 8:8 + H] = v
            return w[..., 8:8 + H]
        if layout == "batch":  # batch-major storage
            return v.transpose(0, 1).contiguous().transpose(0, 1)
        if layout == "shifted":  # not aligned to more than an element
            w = torch.empty(T * N * H + 1, dtype=dtype, device="cuda")
            w[1:] = v.reshape(-1)
            return w[1:].view(T, N, H)
        raise AssertionError(layout)

    s = dict(gate=place(1, mean, 1.5), x=place(2, 0.0), dh=place(3, 0.0), h0=rnd(N, H, seed=seed + 4),
             dh_last=rnd(N, H, seed=seed + 5), reset=None, lengths=None)
    g = torch.Generator().manual_seed(seed + 6)
    if reset:
        s["reset"] = (torch.rand(T, N, generator=g) < 0.05).to(torch.uint8).cuda() * 3
        if T > 1 and N > 1:
            s["reset"][0, 0] = 1
            s["reset"][T - 1, N - 1] = 1
    if lengths:
        ln = torch.randint(0, T + 1, (N,), generator=g, dtype=torch.int32)
        ln[0] = 0
        ln[N - 1] = T
        if N > 2:
            ln[1] = min(1, T)
        s["lengths"] = ln.cuda()
        for k in ("gate", "x", "dh"):  # nothing in the padding is read
            for n in range(N):
                s[k][int(ln[n]):, n] = float("nan") if n % 2 else float("inf")
    return s


def run_scan(ops, s, out=None, dgate=None, dx=None):
    h, last = ops.gated_scan(s["gate"], s["x"], h0=s["h0"], reset=s["reset"], lengths=s["lengths"], out=out)
    g = ops.gated_scan_backward(s["gate"], s["x"], h, s["dh"], dh_last=s["dh_last"], h0=s["h0"], reset=s["reset"],
                                lengths=s["lengths"], dgate=dgate, dx=dx)
    return (h, last) + g


def check_scan(ops, s, **out):
    h, last, dgate, dx, dh0 = run_scan(ops, s, **out)
    f = ref.scan(s["gate"], s["x"], s["h0"], s["reset"], s["lengths"])
    b = ref.scan_backward(s["gate"], s["x"], h, s["dh"], s["dh_last"], s["h0"], s["reset"], s["lengths"])
    ref.check(h, *f["h"], "h")
    ref.check(last, *f["h_last"], "h_last")
    ref.check(dgate, *b["dgate"], "dgate")
    ref.check(dx, *b["dx"], "dx")
    ref.check(dh0, *b["dh0"], "dh0")
    ops.sync()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("T,N,H", [(1, 1, 1), (1, 16, 256), (2, 3, 5), (31, 2, 64), (64, 1, 8), (65, 3, 33), (127, 1, 301),
                                   (200, 5, 96), (1000, 1, 256), (1025, 2, 7), (4099, 1, 24), (33, 40, 512)])
def test_scan_sizes(ops, dtype, T, N, H):
    check_scan(ops, scan_inputs(T, N, H, DT[dtype], seed=T))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("layout", ["columns", "batch", "shifted"])
@pytest.mark.parametrize("T,N,H", [(7, 3, 40), (300, 2, 64), (90, 4, 31)])
def test_scan_layouts(ops, dtype, layout, T, N, H):
    s = scan_inputs(T, N, H, DT[dtype], layout, seed=11)
    check_scan(ops, s)
    # outputs in that layout too: two gradients side by side, nothing else written
    wide = torch.full((T, N, 2 * H + 3), 7.0, dtype=DT[dtype], device="cuda")
    hs = torch.empty((N, T, H), dtype=DT[dtype], device="cuda").transpose(0, 1)
    check_scan(ops, s, out=hs, dgate=wide[..., :H], dx=wide[..., H:2 * H])
    assert (wide[..., 2 * H:] == 7.0).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("T,N,H", [(1, 4, 16), (40, 5, 24), (129, 3, 64), (2000, 3, 48), (700, 6, 5)])
@pytest.mark.parametrize("reset,lengths", [(True, False), (False, True), (True, True)])
def test_scan_resets_and_lengths(ops, dtype, T, N, H, reset, lengths):
    check_scan(ops, scan_inputs(T, N, H, DT[dtype], seed=5 + T, reset=reset, lengths=lengths))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("T,N,H,layout", [(9, 90, 512, "plain"), (33, 160, 301, "plain"), (70, 100, 512, "columns"),
                                          (40, 48, 1000, "batch"), (11, 95, 514, "plain"), (14, 200, 1024, "plain"),
                                          (9, 365, 504, "columns")])
@pytest.mark.parametrize("masks", [False, True])
def test_scan_many_channels(ops, dtype, T, N, H, layout, masks):
    check_scan(ops, scan_inputs(T, N, H, DT[dtype], layout, seed=T, reset=masks, lengths=masks))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("T,N,H", [(5000, 1, 20), (3000, 2, 130), (6000, 1, 66), (2500, 1, 33), (1500, 3, 700)])
def test_scan_long(ops, dtype, T, N, H):
    """Several stretches of time, one channel tile to many, resets and padding across their borders."""
    check_scan(ops, scan_inputs(T, N, H, DT[dtype], seed=T, reset=True, lengths=N > 1))


@pytest.mark.parametrize("T,N,H", [(600, 1, 64), (20, 2, 32)])
def test_scan_slow_gates(ops, T, N, H):
    """Gates that keep nearly everything: errors must not grow beyond the bound that follows them."""
    check_scan(ops, scan_inputs(T, N, H, torch.float32, seed=3, mean=8.0))
    check_scan(ops, scan_inputs(T, N, H, torch.bfloat16, seed=3, mean=8.0))


@pytest.mark.parametrize("T", [5, 640])
def test_scan_optional_arguments(ops, T):
    s = scan_inputs(T, 3, 32, torch.float32, seed=21)
    s["h0"] = s["dh_last"] = None
    check_scan(ops, s)
    h, last = ops.gated_scan(s["gate"], s["x"], want_last=False)
    assert last is None
    ref.check(h, *ref.scan(s["gate"], s["x"])["h"], "h")
    dgate, dx, dh0 = ops.gated_scan_backward(s["gate"], s["x"], h, s["dh"], want_dh0=False)
    assert dh0 is None
    b = ref.scan_backward(s["gate"], s["x"], h, s["dh"])
    ref.check(dgate, *b["dgate"], "dgate")
    ref.check(dx, *b["dx"], "dx")


@pytest.mark.parametrize("T", [9, 512])
def test_scan_reset_drops_what_came_before(ops, T):
    """A state of inf or NaN before an episode's first step does not reach it, forward or backward."""
    s = scan_inputs(T, 2, 16, torch.float32, seed=8)
    cut = T // 2
    s["reset"] = torch.zeros(T, 2, dtype=torch.uint8, device="cuda")
    s["reset"][cut] = 1
    clean = run_scan(ops, s)
    bad = dict(s, h0=torch.full_like(s["h0"], float("inf")), x=s["x"].clone(), gate=s["gate"].clone())
    bad["x"][1] = float("nan")
    got = run_scan(ops, bad)
    assert torch.isnan(got[0][1:cut]).all()
    for i in (0, 2, 3):  # h, dgate, dx from the reset on
        ref.check(got[i][cut:], clean[i][cut:].cpu().double(), torch.zeros_like(clean[i][cut:].cpu().double()) + 1e-6, str(i))
    ref.check(got[1], clean[1].cpu().double(), torch.full(clean[1].shape, 1e-6, dtype=torch.float64), "h_last")
    # a gradient of NaN after a reset does not reach the steps before it
    bad = dict(s, dh=s["dh"].clone(), dh_last=torch.full_like(s["dh_last"], float("nan")))
    got = run_scan(ops, bad)
    for i in (2, 3):
        ref.check(got[i][:cut], clean[i][:cut].cpu().double(), torch.zeros_like(clean[i][:cut].cpu().double()) + 1e-6, str(i))
    assert torch.isfinite(got[4]).all()


def test_scan_saturated_gates(ops):
    """Gates at the ends of their range: all kept, or all written, exactly."""
    T, N, H = 130, 1, 8
    x = rnd(T, N, H, seed=1)
    h0 = rnd(N, H, seed=2)
    for g, want in ((float("inf"), h0.expand(T, N, H)), (200.0, h0.expand(T, N, H)), (float("-inf"), x), (-200.0, x),
                    (torch.finfo(torch.float32).min, x)):
        h, last = ops.gated_scan(torch.full((T, N, H), g, device="cuda"), x, h0=h0)
        assert torch.equal(h, want.contiguous()), g
        assert torch.equal(last, h[-1])


def test_scan_empty(ops):
    z = torch.empty(0, 3, 8, device="cuda")
    h0 = rnd(3, 8, seed=1)
    h, last = ops.gated_scan(z, z, h0=h0)
    assert h.shape == (0, 3, 8) and torch.equal(last, h0)
    _, last = ops.gated_scan(z, z)
    assert torch.equal(last, torch.zeros(3, 8, device="cuda"))
    dg, dx, dh0 = ops.gated_scan_backward(z, z, z, z, dh_last=h0)
    assert dg.shape == (0, 3, 8) and torch.equal(dh0, h0)
    e = torch.empty(5, 0, 8, device="cuda")
    h, last = ops.gated_scan(e, e)
    assert h.shape == (5, 0, 8) and last.shape == (0, 8)


def test_scan_length_out_of_range(ops, seq):
    s = scan_inputs(6, 3, 8, torch.float32)
    h, _ = ops.gated_scan(s["gate"], s["x"], lengths=torch.tensor([6, 9, -2], dtype=torch.int32, device="cuda"))
    with pytest.raises(seq.WMError) as e:
        ops.sync()
    assert e.value.status == 1
    ops.sync()  # cleared
    want, _ = ops.gated_scan(s["gate"], s["x"], lengths=torch.tensor([6, 6, 0], dtype=torch.int32, device="cuda"))
    assert torch.equal(h, want)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_step_is_the_scan(ops, dtype):
    """A dream's steps one by one, the state in place, against one call."""
    T, N, H = 12, 16, 256
    s = scan_inputs(T, N, H, DT[dtype], reset=True, seed=4)
    f = ref.scan(s["gate"], s["x"], s["h0"], s["reset"])
    state = s["h0"].clone()
    for t in range(T):
        h, got = ops.gated_step(s["gate"][t], s["x"][t], state, reset=s["reset"][t], out_state=state)
        assert got is state
        ref.check(h, f["h"][0][t], f["h"][1][t], f"h {t}")
    ref.check(state, *f["h_last"], "state")
    assert ops.last_launches == 1


@pytest.mark.parametrize("T,N,H", [(3, 2, 8), (40, 100, 512), (100, 2, 40), (20000, 1, 96), (5000, 4, 33)])
def test_scan_state_in_place(ops, T, N, H):
    """h_last may be h0, whichever kernel runs and however many CTAs read the state entering the call."""
    s = scan_inputs(T, N, H, torch.bfloat16, seed=6)
    want, last = ops.gated_scan(s["gate"], s["x"], h0=s["h0"])
    for _ in range(3):
        state = s["h0"].clone()
        h, got = ops.gated_scan(s["gate"], s["x"], h0=state, h_last=state)
        assert got is state and torch.equal(h, want) and torch.equal(state, last)


@pytest.mark.parametrize("T,N,H,far", [(5, 2, 64, 2 ** 31 + 64), (12, 2, 64, 2 ** 29 + 64), (12, 90, 512, 2 ** 29 + 64)])
def test_scan_offsets_past_32_bits(ops, T, N, H, far):
    """Arrays whose last steps begin past 2^32 values: 64-bit offsets in every kernel."""
    big = torch.empty((T - 1) * far + 6 * N * H, dtype=torch.bfloat16, device="cuda")
    s = scan_inputs(T, N, H, torch.bfloat16, seed=9)
    views = [torch.as_strided(big, (T, N, H), (far, H, 1), i * N * H) for i in range(6)]
    for v, k in zip(views, ("gate", "x", "dh")):
        v.copy_(s[k])
        s[k] = v
    check_scan(ops, s, out=views[3], dgate=views[4], dx=views[5])


def test_norm_offsets_past_32_bits(ops):
    far = 2 ** 31 + 24
    big = torch.empty(2 * far + 3 * 64, dtype=torch.bfloat16, device="cuda")
    x, y, dx = (torch.as_strided(big, (3, 64), (far, 1), i * 64) for i in range(3))
    x.copy_(rnd(3, 64, seed=1, dtype=torch.bfloat16))
    _, mean, rstd = ops.layer_norm(x, out=y, want_stats=True)
    ref.check(y, *ref.norm(x, None, None, 1e-5)["y"], "y")
    g = ref.norm_backward(x, None, mean, rstd, y)
    ops.layer_norm_backward(x, None, mean, rstd, y, dx=dx)
    ref.check(dx, *g["dx"], "dx")


def test_embed_and_clip_past_32_bits(ops):
    """More than 2^31 values: lookup, gradient (whole numbers, so that the sums are exact) and norm."""
    n, V, D = 4_300_000, 1000, 512
    t = ((torch.arange(n, device="cuda") * 7919) % (V + 1) - 1).to(torch.int32)
    table = rnd(V, D, seed=1, dtype=torch.bfloat16)
    out = ops.embed(table, t, scale=2.0)
    at = torch.arange(n - 3000, n, 7, device="cuda")
    assert torch.equal(out[at], torch.where((t[at] >= 0)[:, None], table[t[at].clamp(min=0).long()] * 2, 0))
    part = torch.arange(n, device="cuda") % 3
    out.copy_(part[:, None].expand(n, D))
    got = ops.embed_backward(t, out, V, scale=0.25)
    want = torch.zeros(V + 1, dtype=torch.float64, device="cuda").index_add_(0, (t + 1).long(), part.double())[1:] * 0.25
    assert torch.equal(got, want.to(torch.bfloat16)[:, None].expand(V, D))
    flat = out.view(-1)
    flat.fill_(1.0)
    norm = ops.clip_grads([flat], 1.0)
    assert abs(float(norm) - math.sqrt(n * D)) <= 1e-6 * math.sqrt(n * D)
    assert torch.equal(flat[-5:], torch.full_like(flat[-5:], 1.0 / float(norm)))
    ops.sync()


def test_scan_gradient_against_differences(ops):
    T, N, H = 70, 2, 6
    s = scan_inputs(T, N, H, torch.float32, seed=31, reset=True, lengths=True)
    for k in ("gate", "x", "dh"):
        s[k] = torch.nan_to_num(s[k], nan=0.5, posinf=0.5)
    _, _, dgate, dx, dh0 = run_scan(ops, s)

    def loss(gate, x, h0):
        f = ref.scan(gate, x, h0, s["reset"], s["lengths"])
        live = torch.arange(T)[:, None, None] < s["lengths"].cpu().long()[None, :, None]
        return float((f["h"][0] * s["dh"].cpu().double() * live).sum() + (f["h_last"][0] * s["dh_last"].cpu().double()).sum())

    base = [s[k].cpu().double() for k in ("gate", "x", "h0")]
    for i, g in enumerate((dgate, dx, dh0)):
        d = torch.randn(base[i].shape, generator=torch.Generator().manual_seed(i), dtype=torch.float64)
        eps = 1e-5
        hi, lo = (loss(*[b + (sgn * eps * d if j == i else 0) for j, b in enumerate(base)]) for sgn in (1, -1))
        want, got = (hi - lo) / (2 * eps), float((g.cpu().double() * d).sum())
        # the difference quotient: eps^2 and 1e-16 / eps; the gradient: fp32 over its terms
        tol = 1e-5 * float((g.cpu().double() * d).abs().sum()) + 1e-6
        assert abs(want - got) <= tol, (i, want, got, tol)


# ------------------------------------------------------------------ layer norm
NORM_D = [1, 2, 7, 33, 128, 256, 300, 301, 512, 1000, 1024, 1025, 2048, 4096, 5000, 8192, 8193, 16384, 20000]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("D", NORM_D)
def test_norm(ops, dtype, D):
    for rows in (1, 5, 37):
        x = rnd(rows, D, seed=D, dtype=DT[dtype], mean=0.7, std=2.0)
        w, b = rnd(D, seed=D + 1, mean=1.0), rnd(D, seed=D + 2)
        dy = rnd(rows, D, seed=D + 3, dtype=DT[dtype])
        y, mean, rstd = ops.layer_norm(x, w, b, eps=1e-5, want_stats=True)
        f = ref.norm(x, w, b, 1e-5)
        for k, v in (("y", y), ("mean", mean), ("rstd", rstd)):
            ref.check(v, *f[k], f"{k} {rows}")
        dx, dw, db = ops.layer_norm_backward(x, w, mean, rstd, dy)
        g = ref.norm_backward(x, w, mean, rstd, dy)
        for k, v in (("dx", dx), ("dw", dw), ("db", db)):
            ref.check(v, *g[k], f"{k} {rows}")


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,D", [(3000, 64), (5001, 301), (700, 2048)])
def test_norm_many_rows(ops, dtype, rows, D):
    x, dy = (rnd(rows, D, seed=i, dtype=DT[dtype]) for i in (1, 2))
    y, mean, rstd = ops.layer_norm(x, None, None, want_stats=True)
    ref.check(y, *ref.norm(x, None, None, 1e-5)["y"], "y")
    g = ref.norm_backward(x, None, mean, rstd, dy)
    got = ops.layer_norm_backward(x, None, mean, rstd, dy)
    for k, v in zip(("dx", "dw", "db"), got):
        ref.check(v, *g[k], k)
    again = ops.layer_norm_backward(x, None, mean, rstd, dy)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,D", [(1, 9001), (3, 8200), (333, 9000), (333, 9002), (200, 9001), (310, 12288), (310, 12289)])
def test_norm_long_rows(ops, dtype, rows, D):
    """Around the longest rows that a CTA's registers hold, of every width, with more rows than CTAs; dx over dy."""
    x, dy, w = rnd(rows, D, seed=1, dtype=DT[dtype], mean=0.2), rnd(rows, D, seed=2, dtype=DT[dtype]), rnd(D, seed=3, mean=1.0)
    y, mean, rstd = ops.layer_norm(x, w, None, want_stats=True)
    ref.check(y, *ref.norm(x, w, None, 1e-5)["y"], "y")
    g = ref.norm_backward(x, w, mean, rstd, dy)
    got = ops.layer_norm_backward(x, w, mean, rstd, dy)
    for k, v in zip(("dx", "dw", "db"), got):
        ref.check(v, *g[k], k)
    again = ops.layer_norm_backward(x, w, mean, rstd, dy, dx=dy)
    assert again[0] is dy and all(torch.equal(a, b) for a, b in zip(got, again))


def test_norm_strides_and_in_place(ops):
    wide = rnd(40, 3 * 96 + 1, seed=1)
    for at in (0, 96, 97):  # aligned and not
        x = wide[:, at:at + 96]
        w, b = rnd(96, seed=2), rnd(96, seed=3)
        f = ref.norm(x, w, b, 1e-3)
        out = torch.full((40, 200), 5.0, device="cuda")
        ops.layer_norm(x, w, b, eps=1e-3, out=out[:, 3:99])
        ref.check(out[:, 3:99], *f["y"], "y")
        assert (out[:, 99:] == 5.0).all() and (out[:, :3] == 5.0).all()
    x = rnd(4, 10, 64, seed=4)
    f = ref.norm(x, None, None, 1e-5)
    y, mean, rstd = ops.layer_norm(x, None, None, out=x, want_stats=True)
    assert y is x and mean.shape == (4, 10)
    ref.check(x, *f["y"], "in place")
    x, dy = rnd(50, 64, seed=5), rnd(50, 64, seed=6)
    _, mean, rstd = ops.layer_norm(x, None, None, want_stats=True)
    g = ref.norm_backward(x, None, mean, rstd, dy)
    dx, dw, db = ops.layer_norm_backward(x, None, mean, rstd, dy, dx=dy, want_params=False)
    assert dx is dy and dw is None and db is None
    ref.check(dy, *g["dx"], "dx in place")


def test_norm_hard_rows(ops):
    """Rows far from 0 (no cancellation in the variance), constant rows, rows of inf or NaN beside others."""
    x = rnd(6, 256, seed=1)
    x[1] = x[1] * 1e-3 + 1000.0
    x[2] = 3.0
    x[3, 17] = float("inf")
    x[4, 200] = float("nan")
    y, mean, rstd = ops.layer_norm(x, None, None, want_stats=True)
    ok = [0, 1, 2, 5]
    f = ref.norm(x[ok], None, None, 1e-5)
    ref.check(y[ok], *f["y"], "y")
    assert torch.isnan(y[3:5]).all()
    assert torch.equal(y[2], torch.zeros_like(y[2]))


def test_norm_rows_of_any_stride(ops):
    """Rows that are one row repeated, every other row, and runs of rows within wider arrays."""
    row, dy = rnd(64, seed=1), rnd(5, 64, seed=2)
    base = rnd(6, 4, 128, seed=3)
    for x in (row.expand(5, 64), rnd(10, 64, seed=4)[::2], base[1:, 2, 32:96], base[:, :, 64:].flatten(0, 1)[:5], base[2:3, 1:2, :64].expand(5, 1, 64)):
        y, mean, rstd = ops.layer_norm(x, want_stats=True)
        ref.check(y, *ref.norm(x, None, None, 1e-5)["y"], str(x.stride()))
        d = dy.view(x.shape)
        got = ops.layer_norm_backward(x, None, mean, rstd, d)
        for k, v in zip(("dx", "dw", "db"), got):
            ref.check(v, *ref.norm_backward(x, None, mean, rstd, d)[k], k)
    with pytest.raises(ValueError):  # not one run of rows
        ops.layer_norm(base[:, :3, :64])
    with pytest.raises(seq_error()):  # an output's rows may not be one row
        ops.layer_norm(rnd(5, 64, seed=1), out=row.clone().expand(5, 64))


def seq_error():
    import paper_2205_01435_gb300 as pkg
    return pkg.load().WMError


def test_norm_empty(ops):
    x = torch.empty(0, 32, device="cuda")
    y, mean, rstd = ops.layer_norm(x, None, None, want_stats=True)
    assert y.shape == (0, 32)
    dx, dw, db = ops.layer_norm_backward(x, None, mean, rstd, x)
    assert dx.shape == (0, 32) and not dw.any() and not db.any()


def test_norm_gradient_against_differences(ops):
    x, w, dy = rnd(9, 24, seed=1), rnd(24, seed=2, mean=1.0), rnd(9, 24, seed=3)
    _, mean, rstd = ops.layer_norm(x, w, None, want_stats=True)
    got = ops.layer_norm_backward(x, w, mean, rstd, dy)
    base = [x.cpu().double(), w.cpu().double(), torch.zeros(24, dtype=torch.float64)]

    def loss(*a):
        return float((ref.norm(*a, 1e-5)["y"][0] * dy.cpu().double()).sum())

    for i, g in enumerate(got):
        d = torch.randn(base[i].shape, generator=torch.Generator().manual_seed(i), dtype=torch.float64)
        hi, lo = (loss(*[b + (sgn * 1e-5 * d if j == i else 0) for j, b in enumerate(base)]) for sgn in (1, -1))
        tol = 1e-5 * float((g.cpu().double() * d).abs().sum()) + 1e-6
        assert abs((hi - lo) / 2e-5 - float((g.cpu().double() * d).sum())) <= tol, i


# ------------------------------------------------------------------ embedding
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n,V,D", [(1, 1, 1), (1, 300, 8), (5, 3, 7), (31, 64, 33), (32, 64, 256), (33, 1, 64), (257, 255, 40),
                                   (1000, 256, 301), (4096, 257, 64), (4097, 70000, 24), (5000, 2, 72), (20000, 17, 128)])
def test_embed(ops, dtype, n, V, D):
    g = torch.Generator().manual_seed(n)
    tokens = torch.randint(0, V, (n,), generator=g, dtype=torch.int32)
    tokens[torch.rand(n, generator=g) < 0.1] = -1
    tokens = tokens.cuda()
    table, dout = rnd(V, D, seed=1, dtype=DT[dtype]), rnd(n, D, seed=2, dtype=DT[dtype])
    ref.check(ops.embed(table, tokens, scale=1.7), *ref.embed(table, tokens, 1.7), "out")
    got = ops.embed_backward(tokens, dout, V, scale=1.7)
    ref.check(got, *ref.embed_backward(tokens, dout, V, 1.7), "dtable")
    assert torch.equal(got, ops.embed_backward(tokens, dout, V, scale=1.7))
    ops.sync()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n,V,D", [(700, 40, 300), (700, 40, 302), (900, 1000, 1001), (3000, 9, 516), (300, 2, 2050)])
def test_embed_widths(ops, dtype, n, V, D):
    """Rows whose length allows 16-, 8-, 4- and 2-byte accesses, in one slice of columns and several."""
    t = torch.randint(-1, V, (n,), generator=torch.Generator().manual_seed(D), dtype=torch.int32).cuda()
    table, dout = rnd(V, D, seed=1, dtype=DT[dtype]), rnd(n, D, seed=2, dtype=DT[dtype])
    ref.check(ops.embed(table, t, scale=0.3), *ref.embed(table, t, 0.3), "out")
    ref.check(ops.embed_backward(t, dout, V, scale=0.3), *ref.embed_backward(t, dout, V, 0.3), "dtable")


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("D", [12, 258, 302, 380, 516, 700, 1002, 2050, 4100, 8194])
def test_norm_widths(ops, dtype, D):
    rows = 50
    x, dy = rnd(rows, D, seed=D, dtype=DT[dtype], std=2.0), rnd(rows, D, seed=D + 3, dtype=DT[dtype])
    w, b = rnd(D, seed=D + 1, mean=1.0), rnd(D, seed=D + 2)
    y, mean, rstd = ops.layer_norm(x, w, b, want_stats=True)
    ref.check(y, *ref.norm(x, w, b, 1e-5)["y"], "y")
    g = ref.norm_backward(x, w, mean, rstd, dy)
    for k, v in zip(("dx", "dw", "db"), ops.layer_norm_backward(x, w, mean, rstd, dy)):
        ref.check(v, *g[k], k)


@pytest.mark.parametrize("n,V", [(1023, 255), (1025, 256), (16384, 30000), (70001, 513), (196608, 100), (196609, 300), (250000, 70000)])
def test_embed_backward_sort_sizes(ops, n, V):
    """One CTA, a cluster, its last size, and beyond it; one digit to three."""
    g = torch.Generator().manual_seed(V)
    t = (float(V) ** torch.rand(n, generator=g, dtype=torch.float64)).long() - torch.randint(0, 2, (n,), generator=g)
    t = torch.randperm(V + 1, generator=g)[t.clamp(0, V)] - 1
    dout = rnd(n, 16, seed=2)
    got = ops.embed_backward(t.to(torch.int32).cuda(), dout, V)
    ref.check(got, *ref.embed_backward(t, dout, V, 1.0), "dtable")


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n", [31, 255, 256, 257])
@pytest.mark.parametrize("V,D", [(3, 1000), (5000, 301), (1, 64)])
def test_embed_backward_few_tokens(ops, dtype, n, V, D):
    """Up to 256 tokens go without a sort: rows that nearly all tokens took, and none."""
    g = torch.Generator().manual_seed(n)
    t = torch.where(torch.rand(n, generator=g) < 0.7, 0, torch.randint(-1, V, (n,), generator=g)).to(torch.int32).cuda()
    dout = rnd(n, D, seed=2, dtype=DT[dtype])
    out = torch.full((V, D), 5.0, dtype=DT[dtype], device="cuda")
    ref.check(ops.embed_backward(t, dout, V, scale=3.0, out=out), *ref.embed_backward(t, dout, V, 3.0), "dtable")
    assert ops.last_launches == (1 if n <= 256 else 3)


@pytest.mark.parametrize("kind", ["one token", "none", "sorted", "reversed", "common"])
def test_embed_token_orders(ops, kind):
    n, V, D = 9000, 1000, 48
    g = torch.Generator().manual_seed(1)
    t = {"one token": torch.full((n,), 7), "none": torch.full((n,), -3), "sorted": torch.arange(n) * V // n,
         "reversed": (torch.arange(n) * V // n).flip(0),
         "common": torch.where(torch.rand(n, generator=g) < 0.5, 999, torch.randint(0, V, (n,), generator=g))}[kind]
    t = t.to(torch.int32).cuda()
    dout = rnd(n, D, seed=2)
    ref.check(ops.embed_backward(t, dout, V, scale=0.5), *ref.embed_backward(t, dout, V, 0.5), kind)


def test_embed_bad_tokens_and_nan_elsewhere(ops, seq):
    table = rnd(10, 16, seed=1)
    t = torch.tensor([[3, 10, -1], [2 ** 31 - 1, -2 ** 31, 9]], dtype=torch.int32, device="cuda")
    out = ops.embed(table, t, scale=2.0)
    assert out.shape == (2, 3, 16)
    assert torch.equal(out[0, 0], table[3] * 2) and torch.equal(out[1, 2], table[9] * 2)
    assert not out[0, 1:].any() and not out[1, :2].any()
    with pytest.raises(seq.WMError):
        ops.sync()
    dout = torch.full((2, 3, 16), float("nan"), device="cuda")  # gradients of rows that were not taken are not read
    dout[0, 0] = 1.0
    dout[1, 2] = 2.0
    g = ops.embed_backward(t, dout, 10, scale=2.0)
    want = torch.zeros(10, 16, device="cuda")
    want[3], want[9] = 2.0, 4.0
    assert torch.equal(g, want)
    with pytest.raises(seq.WMError) as e:
        ops.sync()
    assert e.value.status == 1


def test_embed_empty(ops):
    t = torch.empty(0, dtype=torch.int32, device="cuda")
    assert ops.embed(rnd(4, 8, seed=1), t).shape == (0, 8)
    g = ops.embed_backward(t, torch.empty(0, 8, device="cuda"), 4, out=torch.ones(4, 8, device="cuda"))
    assert not g.any()


# ------------------------------------------------------------------ clipping
def grads_of(sizes, dtypes, seed=0, std=1.0):
    return [rnd(n, seed=seed + i, dtype=DT[d], std=std) for i, (n, d) in enumerate(zip(sizes, dtypes))]


@pytest.mark.parametrize("sizes,dtypes", [([1], ["fp32"]), ([0, 3, 0], ["fp32", "bf16", "bf16"]), ([5000], ["bf16"]),
                                          ([4096, 1, 7, 8192, 8193, 300001], ["fp32", "bf16"] * 3),
                                          ([33] * 1500, ["bf16", "fp32"] * 750)])
@pytest.mark.parametrize("ratio", [0.3, 3.0])
def test_clip(ops, sizes, dtypes, ratio):
    grads = grads_of(sizes, dtypes)
    bound = ratio * float(ref.clip(grads, 1.0)[0])
    norm, ne, want = ref.clip(grads, bound)
    out = [torch.full_like(g, 9.0) for g in grads]
    got = ops.clip_grads(grads, bound, out=out)
    ref.check(got, norm, ne, "norm")
    for o, g, (v, e) in zip(out, grads, want):
        ref.check(o, v, e, "out") if ratio < 1 else None
        assert ratio < 1 or torch.equal(o, g)
    got2 = ops.clip_grads(grads, bound)  # in place
    assert torch.equal(got, got2) and all(torch.equal(a, b) for a, b in zip(grads, out))


def test_clip_unaligned_and_shaped(ops):
    flat = rnd(20000, seed=1)
    half = rnd(20000, seed=2, dtype=torch.bfloat16)
    grads = [flat[1:1 + 63 * 65].view(63, 65), flat[5001:5003], half[3:9000], half[9001:9002].view(1, 1, 1)]
    norm, ne, want = ref.clip(grads, 2.0)
    out = [torch.empty(g.numel() + 1, dtype=g.dtype, device="cuda")[1:].view(g.shape) for g in grads]
    ref.check(ops.clip_grads(grads, 2.0, out=out), norm, ne, "norm")
    for o, (v, e) in zip(out, want):
        ref.check(o, v, e, "out")


@pytest.mark.parametrize("total", [100, 8_400_000, 8_700_000, 20_000_000])
def test_clip_one_launch_and_two(ops, total):
    """Around the size up to which the gradients are held on the SMs, and beyond it."""
    grads = grads_of([total // 2, 3, total // 4 + 1], ["fp32", "bf16", "bf16"], seed=5)
    grads.append(grads[0].new_zeros(total // 4))
    norm, ne, want = ref.clip(grads, 100.0)
    for _ in range(2):
        out = [torch.empty_like(g) for g in grads]
        ref.check(ops.clip_grads(grads, 100.0, out=out), norm, ne, "norm")
        for o, (v, e) in zip(out, want):
            ref.check(o, v, e, "out")
    assert ops.last_launches == (1 if total <= 8_400_000 else 2)


def test_clip_wait_gives_up(seq):
    ops = seq.SequenceOps()
    g = grads_of([3_000_000], ["fp32"])
    ops.inject_wait_timeout(1000)
    ops.clip_grads(g, 1e9)
    with pytest.raises(seq.WMError) as e:
        ops.sync()
    assert e.value.status == 4
    ops.sync()
    norm, ne, _ = ref.clip(g, 1.0)
    ref.check(ops.clip_grads(g, 1e9), norm, ne, "norm")


@pytest.mark.parametrize("std", [1e-30, 1e-20, 1e18, 1e25])
def test_clip_range(ops, std):
    """Values whose squares leave fp32's range, with zeros between them."""
    grads = grads_of([1001, 64], ["fp32", "bf16"], seed=3, std=std)
    grads[0][100:300] = 0
    norm, ne, want = ref.clip(grads, std)
    ref.check(ops.clip_grads(grads, std), norm, ne, "norm")
    for o, (v, e) in zip(grads, want):
        ref.check(o, v, e, "out")


@pytest.mark.parametrize("bad", [float("inf"), float("nan"), 3e38])
def test_clip_norm_not_finite(ops, bad):
    """The gradients stay as they are, and the norm says so."""
    grads = grads_of([100, 5000], ["fp32", "fp32"])
    grads[1][4000:4003] = bad
    before = [g.clone() for g in grads]
    norm = ops.clip_grads(grads, 1.0)
    assert not math.isfinite(float(norm))
    assert all(torch.equal(a.nan_to_num(), b.nan_to_num()) for a, b in zip(grads, before))


def test_clip_zero_and_none(ops):
    z = [torch.zeros(1000, device="cuda"), torch.zeros(9, device="cuda", dtype=torch.bfloat16)]
    assert float(ops.clip_grads(z, 1.0)) == 0 and float(ops.clip_grads(z, 0.0)) == 0
    assert float(ops.clip_grads([], 1.0)) == 0
    g = [rnd(100, seed=1)]
    want = float(g[0].double().norm())
    assert abs(float(ops.clip_grads(g, float("inf"))) - want) <= 1e-6 * want
    ops.clip_grads(g, 0.0)
    assert not g[0].any()


# ------------------------------------------------------------------ streams, graphs, refusals
def test_other_stream(ops):
    s = scan_inputs(300, 2, 64, torch.bfloat16, seed=2)
    want = run_scan(ops, s)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    h, last = ops.gated_scan(s["gate"], s["x"], h0=s["h0"], stream=side)
    g = ops.gated_scan_backward(s["gate"], s["x"], h, s["dh"], dh_last=s["dh_last"], h0=s["h0"], stream=side)
    n = ops.clip_grads([g[0].clone()], 1.0, stream=side.cuda_stream)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(want, (h, last) + g))
    assert math.isfinite(float(n))


def test_graph_capture(seq):
    ops = seq.SequenceOps()
    s = scan_inputs(400, 1, 64, torch.bfloat16, seed=2)
    t = (torch.arange(3000, device="cuda") % 50).to(torch.int32)
    dout = rnd(3000, 32, seed=1)
    def calls():
        clipped = [torch.empty_like(dout), torch.empty_like(big_grad)]
        norms = [ops.clip_grads([dout], 1.0, out=clipped[:1]), ops.clip_grads([big_grad], 1.0, out=clipped[1:])]
        _, mean, rstd = ops.layer_norm(dout, want_stats=True)
        return run_scan(ops, s) + (ops.embed_backward(t, dout, 50), *clipped, *norms,
                                   *ops.layer_norm_backward(dout, None, mean, rstd, dout))

    big_grad = rnd(9_000_000, seed=3)
    want = calls()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = calls()
    graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    # the workspace grows; the graph still has its own
    big = (torch.arange(200000, device="cuda") % 50).to(torch.int32)
    ops.embed_backward(big, rnd(200000, 32, seed=1), 50)
    for v in got:
        v.zero_()
    graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    # growing under capture is refused
    fresh = seq.SequenceOps()
    with pytest.raises(seq.WMError) as e:
        with torch.cuda.graph(torch.cuda.CUDAGraph(), stream=side):
            fresh.embed_backward(t, dout, 50)
    assert e.value.status == 3
    fresh.embed_backward(t, dout, 50)
    ops.close()
    ops.close()


def test_refusals(ops, seq):
    f, b = rnd(4, 2, 8, seed=1), rnd(4, 2, 8, seed=1, dtype=torch.bfloat16)
    h0 = rnd(2, 8, seed=1)
    i32 = torch.zeros(4, dtype=torch.int32, device="cuda")
    bad = [
        lambda: ops.gated_scan(f, b), lambda: ops.gated_scan(f.half(), f.half()), lambda: ops.gated_scan(f, f[:3]),
        lambda: ops.gated_scan(f.cpu(), f.cpu()), lambda: ops.gated_scan(f, f, h0=h0[:1]),
        lambda: ops.gated_scan(f, f, h0=h0.bfloat16()), lambda: ops.gated_scan(f, f, reset=torch.zeros(4, 2, device="cuda")),
        lambda: ops.gated_scan(f, f, lengths=i32), lambda: ops.gated_scan(f[0], f[0]),
        lambda: ops.gated_scan(f.transpose(1, 2), f.transpose(1, 2)),
        lambda: ops.gated_scan(f, f, out=torch.empty(1, 2, 8, device="cuda").expand(4, 2, 8)),
        lambda: ops.gated_scan_backward(f, f, f, b), lambda: ops.gated_scan_backward(f, f, f, f, dx=f[:2]),
        lambda: ops.layer_norm(f, h0[0, :4]), lambda: ops.layer_norm(f, None, None, eps=-1.0),
        lambda: ops.layer_norm(f.double()), lambda: ops.layer_norm(f.cpu()), lambda: ops.layer_norm(f, out=b),
        lambda: ops.layer_norm_backward(f, None, h0[:, 0], h0[:, 0], f),
        lambda: ops.layer_norm(torch.empty(3, 0, device="cuda")),
        lambda: ops.embed(f[0], i32.long()), lambda: ops.embed(f, i32), lambda: ops.embed(f[0].cpu(), i32),
        lambda: ops.embed_backward(i32, f[:3, 0], 5), lambda: ops.embed_backward(i32, f[:, 0].contiguous(), 0),
        lambda: ops.clip_grads([f.transpose(0, 1)], 1.0), lambda: ops.clip_grads([f], -1.0),
        lambda: ops.clip_grads([f], float("nan")), lambda: ops.clip_grads([f], 1.0, out=[b]),
        lambda: ops.clip_grads([f.double()], 1.0), lambda: ops.clip_grads([f], 1.0, out=[]),
    ]
    for k, call in enumerate(bad):
        with pytest.raises((ValueError, seq.WMError)):
            call()
            raise AssertionError(f"call {k} was taken")
    ops.sync()


def test_refusals_of_the_c_entries(ops, seq):
    """What the binding does not look at: addresses, alignment, sizes, types."""
    lib, h = seq._lib, ops.h
    t = torch.empty(64, device="cuda")
    host = torch.empty(64)
    p, hp = t.data_ptr(), host.data_ptr()
    bad = [
        lib.wm_seq_layer_norm(h, 7, 1, 8, p, 8, None, None, 0.1, p, 8, None, None, None),
        lib.wm_seq_layer_norm(h, 0, 1, 8, hp, 8, None, None, 0.1, p, 8, None, None, None),
        lib.wm_seq_layer_norm(h, 0, 1, 8, p + 2, 8, None, None, 0.1, p, 8, None, None, None),
        lib.wm_seq_layer_norm(h, 0, 1, 8, None, 8, None, None, 0.1, p, 8, None, None, None),
        lib.wm_seq_layer_norm(h, 0, 2, 8, p, 8, None, None, 0.1, p + 128, 7, None, None, None),
        lib.wm_seq_layer_norm(h, 0, 1, 8, p, 8, None, None, 0.1, p + 128, 8, p, None, None),
        lib.wm_seq_layer_norm(h, 0, -1, 8, p, 8, None, None, 0.1, p, 8, None, None, None),
        lib.wm_seq_embed(h, 0, 1, 0, 8, p, p, 1.0, p, None),
        lib.wm_seq_embed(h, 0, 1, 1, 8, p, None, 1.0, p, None),
        lib.wm_seq_embed_backward(h, 0, 2 ** 31, 1, 8, p, p, 1.0, p, None),
        lib.wm_seq_gated_scan(h, 0, 1, 1, 8, None, None, None, None, None, None, None, None),
        lib.wm_seq_gated_scan(h, 0, -1, 1, 8, None, None, None, None, None, None, None, None),
        lib.wm_seq_clip(h, 1, None, 1.0, p, None), lib.wm_seq_clip(h, 0, None, 1.0, None, None),
        lib.wm_seq_clip(h, -1, None, 1.0, p, None),
    ]
    assert bad == [1] * len(bad)
    assert lib.wm_seq_last_error(h)
    assert lib.wm_seq_layer_norm(h, 0, 1, 8, p, 8, None, None, 0.1, p, 8, None, None, None) == 0
    assert lib.wm_seq_last_error(h) == b""


def test_wait_gives_up(seq):
    """A wait that nothing completes ends by its limit, is reported once, and leaves the handle usable."""
    ops = seq.SequenceOps()
    s = scan_inputs(3000, 1, 64, torch.float32, seed=1)
    ops.inject_wait_timeout(1000)
    run_scan(ops, s)
    with pytest.raises(seq.WMError) as e:
        ops.sync()
    assert e.value.status == 4
    ops.sync()
    check_scan(ops, s)


# ------------------------------------------------------------------ the operators together
def block_module():
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "gated_block.py")
    spec = importlib.util.spec_from_file_location("gated_block", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_block_gradients_against_autograd():
    """A training step's gradients, every operator in it, against torch's derivative of the plain block in 64 bits."""
    m = block_module()
    T, N, Z, A, D, H = 37, 6, 8, 11, 40, 24
    z, actions = m.recordings(T, N, Z, A, "fp32")
    block = m.GatedBlock(Z, A, D, H)
    g = torch.Generator().manual_seed(3)
    starts = (torch.rand(T, N, generator=g) < 0.1).to(torch.uint8).cuda()
    lengths = torch.tensor([T, 0, 5, T, 20, 1], dtype=torch.int32, device="cuda")
    pred, saved = block.forward(z[:-1], actions, starts, lengths)
    dpred = torch.randn(T, N, Z, generator=g).cuda()
    dpred = dpred * (torch.arange(T, device="cuda")[:, None] < lengths[None, :])[..., None]
    got = block.backward(saved, dpred)
    p = {k: v.double().cpu().requires_grad_() for k, v in block.p.items()}
    e = torch.nn.functional.embedding(actions.cpu().long(), p["embed"]) * block.scale
    y = torch.nn.functional.layer_norm(e + z[:-1].double().cpu() @ p["w_in"], (D,), p["ln_weight"], p["ln_bias"], 1e-5)
    proj = y @ p["w_proj"] + p["b_proj"]
    h = ref.scan(proj[..., :H], proj[..., H:], None, starts, lengths)["h"][0]
    want = h @ p["w_out"]
    # fp32 through five operators and six products (torch's products in fp32: tf32 is off)
    assert float((pred.double().cpu() - want).abs().max()) <= 1e-4 * float(want.abs().max())
    (want * dpred.double().cpu()).sum().backward()
    for k, v in p.items():
        assert float((got[k].double().cpu() - v.grad).norm()) <= 1e-4 * float(v.grad.norm()), k


@pytest.mark.parametrize("precision", ["fp32", "bf16"])
def test_block_trains_and_dreams(precision):
    m = block_module()
    T, N, Z, A, H = 64, 32, 16, 20, 64
    z, actions = m.recordings(T, N, Z, A, precision)
    block = m.GatedBlock(Z, A, 64, H, precision)
    losses = [float(block.train_step(z, actions, lr=1.0)[0]) for _ in range(60)]
    assert losses[-1] < 0.5 * losses[0], losses[::10]
    # step by step, the state in hand, the block predicts what the scan over the recording does
    pred, _ = block.forward(z[:-1], actions)
    state = torch.zeros(N, H, device="cuda")
    steps = torch.stack([block.dream(z[t], actions[t], state) for t in range(T)])
    tol = 1e-4 if precision == "fp32" else 3e-2
    assert float((steps.float() - pred.float()).abs().max()) <= tol * float(pred.float().abs().max())
    block.ops.sync()
