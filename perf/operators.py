"""The sequence operators, as a training loop or a dream calls them, with their plain forms.

A gated recurrent block over recorded episodes embeds the actions, normalises its input, projects
it (a matrix product), and runs a gated linear recurrence over time; its training step goes back
through the same operators and clips the gradients by their global norm.  Each case is one of these
operators on device arrays, at the sizes of the library's workloads or at general ones, forward or
(``train``) forward and backward.  ``own`` selects the library's kernels; otherwise the operators
run in their plain form, in 32 bits, rounded once at the end.
"""
from __future__ import annotations

import functools
import math

import torch

own = False

_DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
_EPS = 1e-5


# ------------------------------------------------------------------ cases
def _scan(dtype, T, N, H, **flags):
    return dict(dict(op="scan", dtype=dtype, T=T, N=N, H=H, train=False, carried=False, ragged=False, resets=0.0,
                     batch_first=False), **flags)


def _norm(dtype, rows, D, train):
    return dict(op="norm", dtype=dtype, rows=rows, D=D, train=train)


def _embed(dtype, n, V, D, zipf):
    return dict(op="embed", dtype=dtype, n=n, V=V, D=D, zipf=zipf)


def _clip(kind, tensors, total, clipped):
    return dict(op="clip", kind=kind, tensors=tensors, total=total, clipped=clipped)


def listed():
    return [
        # one step of a dream of 16 episodes: state in, state out; latency is all of it
        dict(_scan("bf16", 1, 16, 256, carried=True), name="scan_step_bf16"),
        # scoring a minibatch of recorded trajectories: forward only
        dict(_scan("bf16", 128, 512, 512, ragged=True), name="scan_score_bf16"),
        # the training step of the largest model on a minibatch
        dict(_scan("bf16", 128, 512, 1024, train=True, carried=True), name="scan_train_bf16"),
        # one stream of many episodes recorded back to back: all the parallelism is in time
        dict(_scan("bf16", 65536, 1, 256, train=True, carried=True, resets=0.002), name="scan_long_bf16"),
        # trajectories of different lengths, a model that is a multiple of nothing, batch-major logs
        dict(_scan("fp32", 100, 200, 301, train=True, ragged=True, batch_first=True), name="scan_odd_fp32"),
        # the normalisation inside one step of a dream
        dict(_norm("fp32", 16, 256, False), name="norm_step_fp32"),
        # and inside the training step of the largest model
        dict(_norm("bf16", 65536, 1024, True), name="norm_train_bf16"),
        dict(_norm("fp32", 20000, 301, True), name="norm_odd_fp32"),
        # the actions of a minibatch, drawn evenly from the rule set: few rows, each taken often
        dict(_embed("bf16", 65536, 512, 1024, False), name="embed_actions_bf16"),
        # tokens of a large vocabulary, a few of them common and most of them absent
        dict(_embed("fp32", 16384, 30000, 512, True), name="embed_tokens_fp32"),
        # the gradients of the scoring workload's model: W_lstm, b_lstm, W_mdn, b_mdn
        dict(_clip("model", 4, 0, True), name="clip_model_fp32"),
        # the gradients of a deep model, of both types and all sizes
        dict(_clip("many", 60, 200_000_000, True), name="clip_many_mixed"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: one token to long sequences, odd and regular sizes, both types and directions."""
    op = rng.choice(["scan", "scan", "scan", "norm", "norm", "embed", "embed", "clip"])
    dtype = rng.choice(["fp32", "bf16"])
    if op == "scan":
        H = rng.choice([256, 512, 1024, _log_int(rng, 33, 2000)])
        N = rng.choice([1, _log_int(rng, 1, 64), _log_int(rng, 16, 2048)])
        most = 60_000_000 // (N * H)
        T = 1 if rng.random() < 0.15 else _log_int(rng, 2, max(2, min(65536, most)))
        return _scan(dtype, T, N, H, train=rng.random() < 0.5, carried=T == 1 or rng.random() < 0.5,
                     ragged=N > 1 and rng.random() < 0.3, resets=rng.choice([0.0, 0.0, 0.01]),
                     batch_first=rng.random() < 0.3)
    if op == "norm":
        D = rng.choice([256, 512, 1024, 4096, _log_int(rng, 33, 10000)])
        return _norm(dtype, _log_int(rng, 1, 60_000_000 // D), D, rng.random() < 0.6)
    if op == "embed":
        V = _log_int(rng, 60, 60000)
        D = rng.choice([256, 512, 1024, _log_int(rng, 33, 2000)])
        n = _log_int(rng, 1, min(200_000, 60_000_000 // D))
        return _embed(dtype, n, V, D, rng.random() < 0.5)
    return _clip("many", rng.randint(1, 60), _log_int(rng, 1000, 150_000_000), rng.random() < 0.7)


# ------------------------------------------------------------------ inputs
def _sizes(c):
    """[(values, type)] of a case's gradients."""
    if c["kind"] == "model":  # Z, A, H, K = 64, 256, 512, 5
        return [(n, "fp32") for n in ((64 + 256 + 512) * 2048, 2048, 512 * 960, 960)]
    n, total = c["tensors"], c["total"]
    weight = [math.exp(6.0 * ((i * 0.6180339887) % 1.0)) for i in range(n)]  # sizes over a factor of 400
    return [(max(1, int(total * w / sum(weight))), "bf16" if i % 3 else "fp32") for i, w in enumerate(weight)]


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))

    def normal(*shape, dtype=torch.float32, mean=0.0, std=1.0):
        return (torch.randn(shape, generator=gen, device="cuda") * std + mean).to(dtype)

    if c["op"] == "scan":
        T, N, H, dt = c["T"], c["N"], c["H"], _DTYPES[c["dtype"]]
        # one projection gives the gate's pre-activations and the values, side by side
        lead = (N, T) if c["batch_first"] else (T, N)
        proj = normal(*lead, 2 * H, dtype=dt)
        proj[..., :H] += 2.0
        view = proj.transpose(0, 1) if c["batch_first"] else proj
        s = dict(c, proj=proj, gate=view[..., :H], x=view[..., H:], h0=None, reset=None, lengths=None, dh=None,
                 dh_last=None)
        if c["carried"]:
            s["h0"] = normal(N, H, std=0.5)
        if c["resets"] > 0:
            s["reset"] = (torch.rand(T, N, generator=gen, device="cuda") < c["resets"]).to(torch.uint8)
        if c["ragged"]:
            s["lengths"] = torch.randint(1, T + 1, (N,), generator=gen, device="cuda", dtype=torch.int32)
            s["lengths"][N // 2] = 0  # an episode of which nothing was recorded
        if c["train"]:
            dh = normal(*lead, H, dtype=dt, std=0.1)
            s["dh"] = dh.transpose(0, 1) if c["batch_first"] else dh
            if c["carried"]:
                s["dh_last"] = normal(N, H, std=0.1)
        return s
    if c["op"] == "norm":
        dt = _DTYPES[c["dtype"]]
        s = dict(c, x=normal(c["rows"], c["D"], dtype=dt, mean=0.3, std=2.0), weight=normal(c["D"], mean=1.0, std=0.2),
                 bias=normal(c["D"], std=0.2))
        if c["train"]:
            s["dy"] = normal(c["rows"], c["D"], dtype=dt, std=0.1)
        return s
    if c["op"] == "embed":
        n, V, D, dt = c["n"], c["V"], c["D"], _DTYPES[c["dtype"]]
        u = torch.rand(n, generator=gen, device="cuda")
        if c["zipf"]:  # the r-th most common token about 1/r as often as the first
            ranks = (torch.pow(float(V), u) - 1.0).long().clamp_(0, V - 1)
            tokens = torch.randperm(V, generator=gen, device="cuda")[ranks]
        else:
            tokens = (u * V).long().clamp_(0, V - 1)
        tokens[torch.rand(n, generator=gen, device="cuda") < 0.02] = -1  # steps that took no action
        return dict(c, table=normal(V, D, dtype=dt), tokens=tokens.to(torch.int32), scale=math.sqrt(D),
                    dout=normal(n, D, dtype=dt, std=0.1))
    grads = [normal(n, dtype=_DTYPES[t], std=0.02) for n, t in _sizes(c)]
    n = sum(g.numel() for g in grads)
    return dict(c, grads=grads, out=[torch.empty_like(g) for g in grads],
                max_norm=0.02 * math.sqrt(n) * (0.3 if c["clipped"] else 4.0))


# ------------------------------------------------------------------ the operators in their plain form
def _linear_scan(a, b):
    """h_t = a_t h_{t-1} + b_t along the first axis from h = 0, joining spans of doubling length."""
    span = 1
    while span < a.shape[0]:
        b = torch.cat([b[:span], b[span:] + a[span:] * b[:-span]])
        a = torch.cat([a[:span], a[span:] * a[:-span]])
        span *= 2
    return b


def _gates(s):
    """The factors of the carried state and of the value at every step, and which steps count, in 32 bits."""
    p = s["gate"].float()
    keep, write = 1.0 / (1.0 + torch.exp(-p)), 1.0 / (1.0 + torch.exp(p))
    carry = keep if s["reset"] is None else keep * (s["reset"] == 0)[..., None]
    if s["lengths"] is None:
        return keep, write, carry, None
    live = (torch.arange(s["T"], device=p.device)[:, None] < s["lengths"][None, :])[..., None]
    return keep, write, torch.where(live, carry, 1.0), live


def _plain_scan(s):
    keep, write, carry, live = _gates(s)
    b = write * s["x"].float()
    if live is not None:
        b = torch.where(live, b, 0.0)
    if s["h0"] is not None:
        b[0] += carry[0] * s["h0"]
    h = _linear_scan(carry, b)
    h_last = h[-1].clone()
    return (h if live is None else torch.where(live, h, 0.0)).to(s["gate"].dtype), h_last


def _plain_scan_backward(s, h):
    keep, write, carry, live = _gates(s)
    first = torch.zeros_like(h[:1], dtype=torch.float32) if s["h0"] is None else s["h0"][None]
    before = torch.cat([first, h[:-1].float()])
    if s["reset"] is not None:
        before = before * (s["reset"] == 0)[..., None]
    dh = s["dh"].float()
    if live is not None:
        dh = torch.where(live, dh, 0.0)
    dh = dh.clone()
    if s["dh_last"] is not None:
        dh[-1] += s["dh_last"]
    into = torch.cat([carry[1:], torch.zeros_like(carry[:1])])
    lam = _linear_scan(into.flip(0), dh.flip(0)).flip(0)
    dgate, dx = lam * (before - s["x"].float()) * keep * write, lam * write
    if live is not None:
        dgate, dx = torch.where(live, dgate, 0.0), torch.where(live, dx, 0.0)
    return dgate.to(h.dtype), dx.to(h.dtype), carry[0] * lam[0]


def _plain_norm(s):
    x = s["x"].float()
    mean = x.mean(-1)
    rstd = 1.0 / torch.sqrt((x - mean[:, None]).square().mean(-1) + _EPS)
    xhat = (x - mean[:, None]) * rstd[:, None]
    return (xhat * s["weight"] + s["bias"]).to(s["x"].dtype), mean, rstd


def _plain_norm_backward(s, mean, rstd):
    xhat = (s["x"].float() - mean[:, None]) * rstd[:, None]
    dy = s["dy"].float()
    g = dy * s["weight"]
    dx = rstd[:, None] * (g - g.mean(-1, keepdim=True) - xhat * (g * xhat).mean(-1, keepdim=True))
    return dx.to(s["x"].dtype), (dy * xhat).sum(0), dy.sum(0)


def _plain_embed(s):
    taken = (s["tokens"] >= 0)[:, None]
    index = s["tokens"].clamp(min=0).long()
    out = torch.where(taken, s["table"].float()[index] * s["scale"], 0.0).to(s["table"].dtype)
    dout = torch.where(taken, s["dout"].float() * s["scale"], 0.0)
    dtable = torch.zeros(s["table"].shape, device=dout.device).index_add_(0, index, dout)
    return out, dtable.to(s["table"].dtype)


def _plain_clip(s):
    norm = torch.sqrt(torch.stack([g.float().square().sum() for g in s["grads"]]).sum())
    scale = torch.clamp(s["max_norm"] / norm, max=1.0)
    return [(g.float() * scale).to(g.dtype) for g in s["grads"]], norm


# ------------------------------------------------------------------ one pass
@functools.cache
def _ops():
    import paper_2205_01435_gb300 as pkg

    return pkg.load_seq().SequenceOps()


def run(state):
    s = state
    if s["op"] == "scan":
        if not own:
            h, h_last = _plain_scan(s)
            if not s["train"]:
                return {"h": h, "h_last": h_last}
            dgate, dx, dh0 = _plain_scan_backward(s, h)
            return {"h": h, "h_last": h_last, "dproj": torch.cat([dgate, dx], -1), "dh0": dh0}
        ops, H = _ops(), s["H"]
        if s["T"] == 1 and not s["train"] and s["lengths"] is None:
            h, h_last = ops.gated_step(s["gate"][0], s["x"][0], s["h0"], reset=None if s["reset"] is None else s["reset"][0])
            return {"h": h[None], "h_last": h_last}
        out = None
        if s["batch_first"]:
            out = torch.empty((s["N"], s["T"], H), dtype=s["gate"].dtype, device="cuda").transpose(0, 1)
        h, h_last = ops.gated_scan(s["gate"], s["x"], h0=s["h0"], reset=s["reset"], lengths=s["lengths"], out=out)
        if not s["train"]:
            return {"h": h, "h_last": h_last}
        # the gradients side by side, as the projection's backward product takes them
        dproj = torch.empty_like(s["proj"])
        d = dproj.transpose(0, 1) if s["batch_first"] else dproj
        _, _, dh0 = ops.gated_scan_backward(s["gate"], s["x"], h, s["dh"], dh_last=s["dh_last"], h0=s["h0"], reset=s["reset"],
                                            lengths=s["lengths"], dgate=d[..., :H], dx=d[..., H:])
        return {"h": h, "h_last": h_last, "dproj": d, "dh0": dh0}
    if s["op"] == "norm":
        if not own:
            y, mean, rstd = _plain_norm(s)
            if not s["train"]:
                return {"y": y}
            dx, dw, db = _plain_norm_backward(s, mean, rstd)
            return {"y": y, "dx": dx, "dweight": dw, "dbias": db}
        ops = _ops()
        if not s["train"]:
            return {"y": ops.layer_norm(s["x"], s["weight"], s["bias"], eps=_EPS)}
        y, mean, rstd = ops.layer_norm(s["x"], s["weight"], s["bias"], eps=_EPS, want_stats=True)
        dx, dw, db = ops.layer_norm_backward(s["x"], s["weight"], mean, rstd, s["dy"])
        return {"y": y, "dx": dx, "dweight": dw, "dbias": db}
    if s["op"] == "embed":
        if not own:
            out, dtable = _plain_embed(s)
        else:
            out = _ops().embed(s["table"], s["tokens"], scale=s["scale"])
            dtable = _ops().embed_backward(s["tokens"], s["dout"], s["V"], scale=s["scale"])
        return {"out": out, "dtable": dtable}
    if not own:
        grads, norm = _plain_clip(s)
    else:
        norm = _ops().clip_grads(s["grads"], s["max_norm"], out=s["out"])
        grads = s["out"]
    return {"grads": grads, "norm": norm}


# ------------------------------------------------------------------ what a pass has to move and compute
def work(case):
    c = case
    b = {"fp32": 4, "bf16": 2}.get(c.get("dtype"), 0)
    if c["op"] == "scan":
        n, state = c["T"] * c["N"] * c["H"], c["N"] * c["H"] * 4
        states = (2 if c["carried"] else 1) + ((2 if c["carried"] else 1) if c["train"] else 0)
        marks = (c["T"] * c["N"] if c["resets"] > 0 else 0) + (4 * c["N"] if c["ragged"] else 0)
        # padded steps are not read but their outputs are written: about half of the steps count
        live = 0.5 if c["ragged"] and c["T"] > 1 else 1.0
        bytes_ = n * b * (2 * live + 1) + states * state + marks
        flops = 8 * n * live
        if c["train"]:
            bytes_ += n * b * (live + 2)
            flops += 14 * n * live
        return {"bytes": bytes_, "flops": flops}
    if c["op"] == "norm":
        n = c["rows"] * c["D"]
        if not c["train"]:
            return {"bytes": 2 * n * b + 8 * c["D"], "flops": 8 * n}
        return {"bytes": 4 * n * b + 16 * c["D"], "flops": 22 * n}
    if c["op"] == "embed":
        read = min(c["n"], c["V"])  # rows of the table that are read at all, at most
        return {"bytes": c["D"] * b * (2 * c["n"] + read + c["V"]) + 4 * c["n"], "flops": 3 * c["n"] * c["D"]}
    sizes = _sizes(c)
    return {"bytes": sum(2 * n * (4 if t == "fp32" else 2) for n, t in sizes) + 4, "flops": 3 * sum(n for n, _ in sizes)}


# ------------------------------------------------------------------ the definitions, in 64 bits
def _exact_scan(s):
    T, N, H = s["T"], s["N"], s["H"]
    dev = s["gate"].device
    zero = torch.zeros(N, H, dtype=torch.float64, device=dev)
    sig = torch.sigmoid(s["gate"].double())
    v = s["x"].double()
    one_minus = torch.sigmoid(-s["gate"].double())
    entry = torch.ones(T, N, 1, dtype=torch.float64, device=dev)
    counts = torch.ones(T, N, 1, dtype=torch.bool, device=dev)
    if s["reset"] is not None:
        entry = entry.masked_fill((s["reset"] != 0)[..., None], 0.0)
    if s["lengths"] is not None:
        counts = (torch.arange(T, device=dev)[:, None] < s["lengths"][None].long())[..., None]
    a = (sig * entry).masked_fill(~counts, 1.0)
    u = (one_minus * v).masked_fill(~counts, 0.0)
    start = zero if s["h0"] is None else s["h0"].double()
    states = torch.empty(T + 1, N, H, dtype=torch.float64, device=dev)
    states[0] = start
    for prev, nxt, at, ut in zip(states.unbind(0), states.unbind(0)[1:], a.unbind(0), u.unbind(0)):
        torch.addcmul(ut, at, prev, out=nxt)
    out = {"h": states[1:].masked_fill(~counts, 0.0), "h_last": states[T]}
    if not s["train"]:
        return out
    lam = s["dh"].double().masked_fill(~counts, 0.0)
    if s["dh_last"] is not None:
        lam[T - 1] += s["dh_last"].double()
    rows, factors = lam.unbind(0), a.unbind(0)
    for t in range(T - 2, -1, -1):
        rows[t].addcmul_(factors[t + 1], rows[t + 1])
    dgate = (lam * (states[:-1] * entry - v) * sig * one_minus).masked_fill(~counts, 0.0)
    dx = (lam * one_minus).masked_fill(~counts, 0.0)
    return dict(out, dproj=torch.cat([dgate, dx], -1), dh0=a[0] * lam[0])


def exact(case, seed):
    s = prepare(case, seed)
    if s["op"] == "scan":
        return _exact_scan(s)
    if s["op"] == "norm":
        x, w = s["x"].double(), s["weight"].double()
        var, mean = torch.var_mean(x, dim=1, correction=0, keepdim=True)
        r = torch.rsqrt(var + _EPS)
        xh = (x - mean) * r
        out = {"y": xh * w + s["bias"].double()}
        if s["train"]:
            dy = s["dy"].double()
            g = dy * w
            D = x.shape[1]
            out["dx"] = r / D * (D * g - g.sum(1, keepdim=True) - xh * (g * xh).sum(1, keepdim=True))
            out["dweight"], out["dbias"] = torch.einsum("rd,rd->d", dy, xh), dy.sum(0)
        return out
    if s["op"] == "embed":
        V = s["V"]
        padded = torch.cat([s["table"].double(), torch.zeros(1, s["D"], dtype=torch.float64, device="cuda")])
        at = torch.where(s["tokens"] < 0, V, s["tokens"]).long()
        acc = torch.zeros_like(padded).index_add_(0, at, s["dout"].double())
        return {"out": padded[at] * s["scale"], "dtable": acc[:V] * s["scale"]}
    total = math.sqrt(math.fsum(float(g.double().pow(2).sum()) for g in s["grads"]))
    f = min(1.0, s["max_norm"] / total)
    return {"grads": [g.double() * f for g in s["grads"]], "norm": torch.tensor(total, dtype=torch.float64)}
