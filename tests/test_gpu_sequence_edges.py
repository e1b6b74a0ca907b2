"""The sequence operators' handles, streams and ends of range: what a call leaves behind, what runs beside it, and the
largest and smallest values and sizes."""
import ctypes as C
import threading
import time

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


def test_an_error_is_reported_once(seq):
    """A CUDA call that fails inside a call is that call's error, and nobody else's: here the device cannot be waited
    for, so that the workspace cannot grow, while a stream is being captured."""
    rt = C.CDLL("libcudart.so.13")
    stream, graph = C.c_void_p(), C.c_void_p()
    assert rt.cudaStreamCreateWithFlags(C.byref(stream), 1) == 0
    ops = seq.SequenceOps()
    t = (torch.arange(3000, device="cuda") % 50).to(torch.int32)
    dout, table = torch.ones(3000, 32, device="cuda"), torch.empty(50, 32, device="cuda")
    torch.cuda.synchronize()
    assert rt.cudaStreamBeginCapture(stream, 0) == 0
    try:
        with pytest.raises(seq.WMError) as e:
            ops.embed_backward(t, dout, 50, out=table)
        left = rt.cudaPeekAtLastError()
    finally:
        rt.cudaStreamEndCapture(stream, C.byref(graph))
        rt.cudaGetLastError()
    assert e.value.status == 2 and left == 0
    assert torch.equal(ops.embed_backward(t, dout, 50, out=table), torch.full_like(table, 60.0))
    rt.cudaStreamDestroy(stream)


@pytest.mark.parametrize("T,chunks", [(130, (2, 3)), (4100, (33, 65))])
def test_scan_workspace(seq, T, chunks):
    """Scratch of a scan in spans: 8 bytes a chunk and channel, a 16th more for groups of chunks, a 256th for theirs
    (and an 8th of it in hand, in blocks of 2 MB), however few the chunks and narrow the rows."""
    N, H, lanes = 200_000 // T * 40, 1, 32
    v = [torch.randn(T, N, H, device="cuda").bfloat16() for _ in range(6)]
    for k, call in enumerate((lambda o: o.gated_scan(v[0], v[1], out=v[2], want_last=False),
                              lambda o: o.gated_scan_backward(v[0], v[1], v[2], v[3], dgate=v[4], dx=v[5], want_dh0=False))):
        ops = seq.SequenceOps()
        call(warm := seq.SequenceOps())
        warm.sync()
        free = torch.cuda.mem_get_info()[0]
        call(ops)
        ops.sync()
        took = free - torch.cuda.mem_get_info()[0]
        assert took <= N * lanes * 8 * chunks[k] * (1 + 1 / 16 + 1 / 256) * 1.125 + (4 << 20), took


@pytest.mark.parametrize("D,rows_of_cta,at_once", [(500, 4, 3), (1000, 4, 2), (4096, 1, 2)])
def test_norm_sums_of_ctas_that_run_at_once(seq, D, rows_of_cta, at_once):
    """Partial column sums of as many CTAs as an SM's 228 KB hold (fp32: three to four rows of x and dy on their way in each),
    and the gradients from them, with more rows than all CTAs take at a time."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    rows = 4 * sms * rows_of_cta * 2 + 3
    x, dy = (torch.randn(rows, D, generator=torch.Generator().manual_seed(i)).cuda() for i in (1, 2))
    ops = seq.SequenceOps()
    _, mean, rstd = ops.layer_norm(x, want_stats=True)
    dx = torch.empty_like(x)
    ops.layer_norm_backward(x, None, mean, rstd, dy, dx=dx)  # (the outputs' memory is in torch's hands from here on)
    ops = seq.SequenceOps()
    torch.cuda.synchronize()
    free = torch.cuda.mem_get_info()[0]
    got = ops.layer_norm_backward(x, None, mean, rstd, dy, dx=dx)
    ops.sync()
    assert free - torch.cuda.mem_get_info()[0] <= sms * at_once * 2 * D * 4 * 1.125 + (4 << 20)
    want = ref.norm_backward(x, None, mean, rstd, dy)
    for k, v in zip(("dx", "dw", "db"), got):
        ref.check(v, *want[k], k)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("D", [301, 1000, 1023, 4097, 9001, 16383, 20001])
def test_norm_in_place_is_the_norm(ops, dtype, D):
    """y over x gives the same bits, at every width of access, rows lying unaligned beside one another."""
    x = torch.randn(700, D, generator=torch.Generator().manual_seed(D)).to(dtype).cuda()
    w = torch.linspace(0.5, 1.5, D, device="cuda")
    want, *stats = ops.layer_norm(x, w, w, want_stats=True)
    y, *got = ops.layer_norm(x, w, w, out=x, want_stats=True)
    assert y is x and torch.equal(x, want) and all(torch.equal(a, b) for a, b in zip(stats, got))


def test_other_threads_run_while_a_call_waits(seq):
    """A call that waits for the device (its workspace grows) does not keep the interpreter's lock meanwhile."""
    ops = seq.SequenceOps()
    t = (torch.arange(3000, device="cuda") % 50).to(torch.int32)
    dout, table = torch.ones(3000, 32, device="cuda"), torch.empty(50, 32, device="cuda")
    torch.cuda.synchronize()
    stop, ticks = threading.Event(), []

    def other():
        while not stop.wait(0.001):
            ticks.append(time.perf_counter())

    thread = threading.Thread(target=other)
    thread.start()
    try:
        torch.cuda._sleep(600_000_000)  # about 0.3 s
        start = time.perf_counter()
        ops.embed_backward(t, dout, 50, out=table)
        end = time.perf_counter()
    finally:
        stop.set()
        thread.join()
    assert end - start > 0.1  # (it did wait)
    assert sum(start < v < end for v in ticks) > 20
    assert torch.equal(table, torch.full_like(table, 60.0))


@pytest.mark.parametrize("kind", [list, tuple, dict.values, iter])
def test_clip_on_another_stream_keeps_its_gradients(ops, kind):
    """Gradients that the caller lets go of after a call on another stream are not used again before it is done, whatever
    held them."""
    n, side = 4_000_000, torch.cuda.Stream()
    grads, out = {"a": torch.ones(n, device="cuda")}, [torch.empty(n, device="cuda")]
    given = kind(grads) if kind is dict.values else kind(grads.values())
    ops.clip_grads([out[0].fill_(1.0)], 1e9, out=out)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(100_000_000)
    norm = ops.clip_grads(given, 1e9, out=out, stream=side)
    del grads, given
    other = torch.full((n,), 7.0, device="cuda")  # (the memory is free for it)
    torch.cuda.synchronize()
    assert float(norm) == 2000.0 and bool((out[0] == 1.0).all()) and bool((other == 7.0).all())


def test_a_stream_of_another_device_is_refused(seq):
    ops, x = seq.SequenceOps(), torch.ones(2, 8, device="cuda")
    ops.device = torch.device("cuda", 1)  # as if the handle were there
    with pytest.raises(ValueError, match="stream"):
        ops.layer_norm(x, stream=torch.cuda.Stream(0))


def test_threads_take_turns_on_a_handle(seq):
    """Several threads' calls on one handle and stream, with workspaces that grow between them."""
    ops = seq.SequenceOps()
    wrong = []

    def work(k):
        for i in range(12):
            n, V = 300 + 700 * i * (k + 1), 17 + k
            t = (torch.arange(n, device="cuda") % V).to(torch.int32)
            g = ops.embed_backward(t, torch.full((n, 24), float(k + 1), device="cuda"), V)
            want = torch.bincount(t, minlength=V)[:, None].float() * (k + 1)
            if not torch.equal(g, want.expand(V, 24)):
                wrong.append((k, i))

    threads = [threading.Thread(target=work, args=(k,)) for k in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    ops.sync()
    assert not wrong


@pytest.mark.parametrize("T,N,H", [(3, 2, 8), (40, 100, 512), (100, 2, 40), (20000, 1, 96), (5000, 4, 33)])
def test_scan_backward_state_in_place(ops, T, N, H):
    """dh0 may be dh_last, whichever kernel runs and however many CTAs read what enters the last step; on another stream too."""
    from test_gpu_sequence import scan_inputs
    s = scan_inputs(T, N, H, torch.bfloat16, seed=6)
    h, _ = ops.gated_scan(s["gate"], s["x"], h0=s["h0"])
    want = ops.gated_scan_backward(s["gate"], s["x"], h, s["dh"], dh_last=s["dh_last"], h0=s["h0"])
    side = torch.cuda.Stream()
    for stream in (None, None, side):
        state = s["dh_last"].clone()
        side.wait_stream(torch.cuda.current_stream())
        got = ops.gated_scan_backward(s["gate"], s["x"], h, s["dh"], dh_last=state, h0=s["h0"], dh0=state, stream=stream)
        torch.cuda.current_stream().wait_stream(side)
        assert got[2] is state and all(torch.equal(a, b) for a, b in zip(want, got))
    with pytest.raises(ValueError):
        ops.gated_scan_backward(s["gate"], s["x"], h, s["dh"], dh0=s["h0"][:, :1])


# ------------------------------------------------------------------ the ends of the range
def test_norm_of_rows_past_2_30(ops):
    """One row whose weight and bias gradients together pass 2^31 columns.  Whole numbers whose sums over the row are 0
    (D is a multiple of 15): every gradient is exact."""
    D = 2 ** 30 + 11
    x, dy = ((torch.arange(15) % m - m // 2).to(torch.bfloat16).cuda().repeat(D // 15)[None] for m in (5, 3))
    y, mean, rstd = ops.layer_norm(x, eps=0.0, want_stats=True)
    assert float(mean) == 0.0 and abs(float(rstd) - 0.5 ** 0.5) <= 1e-6  # (the mean of 0, 1 and 4 squared: 2)
    assert torch.equal(y[0, -15:], (x[0, -15:].float() * rstd).to(torch.bfloat16))
    del y
    one = torch.ones_like(rstd)
    dx, dw, db = ops.layer_norm_backward(x, None, mean, one, dy)
    assert torch.equal(dx, dy)
    assert torch.equal(db, dy[0].float())
    assert torch.equal(dw, (dy * x)[0].float())
    ops.sync()


def test_axes_that_the_kernels_cannot_index_are_refused(ops, seq):
    """32-bit column and step indices go a little past the end: axes that end within that of 2^31 are refused."""
    lib, h, p = seq._lib, ops.h, torch.empty(64, device="cuda").data_ptr()
    for big in (2 ** 31 - 65535, 2 ** 31 - 1):
        assert lib.wm_seq_embed(h, 0, 1, 1, big, p, p, 1.0, p, None) == 1
        assert lib.wm_seq_embed_backward(h, 0, 1, 1, big, p, p, 1.0, p, None) == 1
        assert lib.wm_seq_layer_norm(h, 0, 1, big, p, big, None, None, 0.1, p, big, None, None, None) == 1
        assert lib.wm_seq_layer_norm_backward(h, 0, 1, big, p, big, None, p, p, p, big, p, big, None, None, None) == 1
        for T, H in ((1, big), (big, 1)):
            assert lib.wm_seq_gated_scan(h, 0, T, 1, H, *([None] * 8)) == 1
            assert b"65536" in lib.wm_seq_last_error(h)
            assert lib.wm_seq_gated_scan_backward(h, 0, T, 1, H, *([None] * 12)) == 1
            assert b"65536" in lib.wm_seq_last_error(h)


def test_embed_backward_of_wide_rows(ops):
    """More than 65,535 times 512 columns, in runs that cross blocks of tokens (whole numbers: every sum is exact)."""
    n, V, D = 260, 3, 33_554_432 + 40
    t = (torch.arange(n, device="cuda") % (V + 1) - 1).to(torch.int32)
    part = (torch.arange(n, device="cuda") % 7).to(torch.bfloat16)
    got = ops.embed_backward(t, part[:, None].expand(n, D).contiguous(), V, scale=0.5)
    want = torch.zeros(V + 1, device="cuda").index_add_(0, (t + 1).long(), part.float())[1:] * 0.5
    assert torch.equal(got, want.to(torch.bfloat16)[:, None].expand(V, D))
    ops.sync()


def test_scan_of_several_sections(ops):
    """More than 256 chunks a tile, in both directions: a state published every 256 chunks."""
    from test_gpu_sequence import check_scan, scan_inputs
    check_scan(ops, scan_inputs(33_100, 1, 8, torch.bfloat16, seed=12, reset=True))


@pytest.mark.parametrize("scale", [float("inf"), float("nan"), 3e38])
@pytest.mark.parametrize("n", [3, 300])
def test_embed_scale_reaches_taken_rows_only(ops, n, scale):
    """Rows that no token took are 0 whatever the scale, with a sort and without."""
    t = torch.tensor([1, -1, 3], dtype=torch.int32, device="cuda").repeat(n // 3)
    g = ops.embed_backward(t, torch.full((n, 8), 100.0, device="cuda"), 5, scale=scale)
    assert torch.equal(g[[0, 2, 4]], torch.zeros(3, 8, device="cuda"))
    want = torch.full((2, 8), 100.0 * (n // 3), device="cuda") * torch.tensor(scale, dtype=torch.float32, device="cuda")
    assert torch.equal(g[[1, 3]], want) or (scale != scale and g[[1, 3]].isnan().all())
    table = torch.ones(5, 8, device="cuda")
    assert torch.equal(ops.embed(table, t, scale=scale)[1], torch.zeros(8, device="cuda"))


@pytest.mark.parametrize("n", [5000, 9_000_000])
@pytest.mark.parametrize("bound", [1e-12, 1e-9, 1e-42])
def test_clip_by_more_than_fp32_holds(ops, n, bound):
    """A factor below fp32's normal range: the clipped values keep their precision, in one launch and two."""
    g = [torch.randn(n, generator=torch.Generator().manual_seed(n)).cuda() * 1e30, torch.ones(3, dtype=torch.bfloat16, device="cuda")]
    norm, ne, want = ref.clip(g, bound)
    out = [torch.empty_like(v) for v in g]
    ref.check(ops.clip_grads(g, bound, out=out), norm, ne, "norm")
    for o, (v, e) in zip(out, want):
        ref.check(o, v, e, "out")


@pytest.mark.parametrize("T,N,H", [(1, 2, 16), (200, 1, 16), (20, 100, 512)])
@pytest.mark.parametrize("gate", [-79.0, -82.0, -84.0, -86.5])
def test_scan_bf16_gates_near_the_range_of_fp32(ops, T, N, H, gate):
    """Gates that keep 1e-35 of a state, and less: large states and gradients show it, forward and backward."""
    g = torch.full((T, N, H), gate).bfloat16().cuda()
    x = torch.zeros(T, N, H, dtype=torch.bfloat16, device="cuda")
    h0 = torch.linspace(1e34, 3e36, N * H).view(N, H).cuda()
    dh = torch.full((T, N, H), 1e25, dtype=torch.bfloat16, device="cuda")
    h, last = ops.gated_scan(g, x, h0=h0)
    f = ref.scan(g, x, h0)
    ref.check(h, *f["h"], "h")
    ref.check(last, *f["h_last"], "h_last")
    got = ops.gated_scan_backward(g, x + 1, h, dh)
    want = ref.scan_backward(g, x + 1, h, dh)
    for k, v in zip(("dgate", "dx", "dh0"), got):
        ref.check(v, *want[k], k)


@pytest.mark.parametrize("T,N,H", [(3, 2, 16), (200, 1, 16), (20, 100, 512)])
@pytest.mark.parametrize("gate", [-100.0, torch.finfo(torch.bfloat16).min, float("-inf")])
def test_scan_bf16_gates_that_keep_nothing(ops, T, N, H, gate):
    """A gate below that range takes the value and drops a large state."""
    g = torch.full((T, N, H), gate, dtype=torch.bfloat16, device="cuda")
    x = torch.linspace(1, 2, T * N * H).view(T, N, H).bfloat16().cuda()
    h, last = ops.gated_scan(g, x, h0=torch.full((N, H), 1e30, device="cuda"))
    assert torch.equal(h, x)
    ref.check(last, x[-1].cpu().double(), torch.full((N, H), 2e-8, dtype=torch.float64), "h_last")
