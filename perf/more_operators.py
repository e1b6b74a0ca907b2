"""Decayed linear attention and the norm of its heads, as a training step or a dream calls them, with their plain forms.

A block whose memory is a matrix for each head: the heads of its queries and keys are normalised
and rotated by their positions, then a linear attention whose weights fall off with the distance
reads the episode so far.  Over a recording it runs in chunks, in a dream one token at a time on a
state in hand.  Each case is one of the two on device arrays, forward or (``train``) forward and
backward.  ``own`` selects the library's kernels; otherwise the operators run in their plain form,
in 32 bits (angles in 64), rounded once at the end.
"""
from __future__ import annotations

import functools
import math

import torch

own = False

_DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
_EPS = 1e-6
_CHUNK = 64


# ------------------------------------------------------------------ cases
def _attend(dtype, T, N, heads, dk, dv, **flags):
    return dict(dict(op="attend", dtype=dtype, T=T, N=N, heads=heads, dk=dk, dv=dv, train=False, carried=False,
                     ragged=False, resets=0.0, batch_first=False), **flags)


def _heads(dtype, T, N, q_heads, k_heads, d, rotary, **flags):
    return dict(dict(op="heads", dtype=dtype, T=T, N=N, q_heads=q_heads, k_heads=k_heads, d=d, rotary=rotary, train=False,
                     interleaved=False, batch_first=False, far=False), **flags)


def listed():
    return [
        # one token of a dream of 16 episodes: state in, state out; latency is all of it
        dict(_attend("bf16", 1, 16, 16, 64, 64, carried=True), name="attend_step_bf16"),
        # one token for each of 1024 episodes: the states are read and written once
        dict(_attend("bf16", 1, 1024, 16, 64, 64, carried=True), name="attend_serve_bf16"),
        # scoring a minibatch of recorded trajectories: forward only
        dict(_attend("bf16", 128, 512, 16, 64, 64, ragged=True), name="attend_score_bf16"),
        # the training step of the largest model, on longer recordings
        dict(_attend("bf16", 1024, 64, 16, 64, 64, train=True, carried=True), name="attend_train_bf16"),
        # two prompts of wide heads: few heads, so that the work has to be split over time
        dict(_attend("bf16", 8192, 2, 8, 128, 128), name="attend_prompt_bf16"),
        # one stream of many episodes recorded back to back
        dict(_attend("bf16", 65536, 1, 8, 128, 64, train=True, carried=True, resets=0.002), name="attend_long_bf16"),
        # a training step in full precision
        dict(_attend("fp32", 128, 128, 8, 64, 64, train=True), name="attend_train_fp32"),
        # trajectories of different lengths, heads that are multiples of nothing, batch-major logs
        dict(_attend("fp32", 100, 200, 7, 43, 43, train=True, ragged=True, batch_first=True), name="attend_odd_fp32"),
        # the heads of one dreamt token of 16 episodes
        dict(_heads("bf16", 1, 16, 16, 16, 64, 64, far=True), name="heads_step_bf16"),
        # and of the training step of the largest model
        dict(_heads("bf16", 1024, 64, 16, 16, 64, 64, train=True), name="heads_train_bf16"),
        # long prompts far into their episodes, keys shared by groups of queries, neighbours rotated
        dict(_heads("bf16", 8192, 2, 16, 4, 128, 128, interleaved=True, far=True), name="heads_prompt_bf16"),
        # heads that are multiples of nothing, rotated in part, batch-major logs
        dict(_heads("fp32", 100, 200, 7, 7, 43, 22, train=True, batch_first=True), name="heads_odd_fp32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: one token to long sequences, odd and regular sizes, both types and directions."""
    dtype = rng.choice(["fp32", "bf16", "bf16"])
    if rng.random() < 0.6:
        dk = rng.choice([32, 64, 128, _log_int(rng, 8, 128)])
        dv = rng.choice([dk, dk, 64, _log_int(rng, 8, 128)])
        heads = rng.choice([4, 8, 16, _log_int(rng, 1, 24)])
        if rng.random() < 0.25:  # single tokens
            n = _log_int(rng, 1, max(1, min(1024, 60_000_000 // (heads * dk * dv))))
            return _attend(dtype, 1, n, heads, dk, dv, carried=True, resets=rng.choice([0.0, 0.05]))
        most = (15_000_000 if dtype == "fp32" else 30_000_000) // (heads * (dk + dv))
        T = _log_int(rng, 2, min(65536, most))
        N = _log_int(rng, 1, max(1, min(512, most // T, 60_000_000 // (heads * dk * dv))))
        return _attend(dtype, T, N, heads, dk, dv, train=rng.random() < 0.5, carried=rng.random() < 0.5,
                       ragged=N > 1 and rng.random() < 0.3, resets=rng.choice([0.0, 0.0, 0.01]),
                       batch_first=rng.random() < 0.3)
    d = rng.choice([32, 64, 128, 256, _log_int(rng, 8, 256)])
    rotary = rng.choice([d - d % 2, d - d % 2, 2 * (d // 4), 0])
    q_heads = rng.choice([4, 8, 16, _log_int(rng, 1, 24)])
    k_heads = rng.choice([q_heads, q_heads, 1, max(1, q_heads // 4)])
    most = 60_000_000 // ((q_heads + k_heads) * d)
    T = 1 if rng.random() < 0.2 else _log_int(rng, 2, min(65536, most))
    N = _log_int(rng, 1, max(1, min(1024, most // T)))
    return _heads(dtype, T, N, q_heads, k_heads, d, rotary, train=rng.random() < 0.5, interleaved=rng.random() < 0.4,
                  batch_first=rng.random() < 0.3, far=rng.random() < 0.5)


# ------------------------------------------------------------------ inputs
def _wide(c, widths):
    """The columns of one wide array [T, N, sum of widths] (or batch-major) as [T, N, heads, d] views."""
    def split(a):
        a = a.transpose(0, 1) if c["batch_first"] else a
        return [p.unflatten(-1, w) for p, w in zip(a.split([h * d for h, d in widths], -1), widths)]
    return split


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    T, N, dt = c["T"], c["N"], _DTYPES[c["dtype"]]
    lead = (N, T) if c["batch_first"] else (T, N)

    def normal(*shape, dtype=torch.float32, mean=0.0, std=1.0):
        return (torch.randn(shape, generator=gen, device="cuda") * std + mean).to(dtype)

    if c["op"] == "attend":
        H, dk, dv = c["heads"], c["dk"], c["dv"]
        widths = [(H, dk), (H, dk), (H, dv)]
        split = _wide(c, widths)
        # one projection gives queries, keys and values side by side
        proj = normal(*lead, H * (2 * dk + dv), dtype=dt)
        q, k, v = split(proj)
        # heads that forget within a few tokens, up to ones that keep hundreds
        halves = 1.0 + 7.0 * torch.arange(H, device="cuda") / max(1, H - 1)
        s = dict(c, proj=proj, q=q, k=k, v=v, split=split, scale=dk ** -0.5, s0=None, reset=None, lengths=None, do=None, ds_last=None,
                 log_decay=torch.log1p(-torch.exp2(-halves.double() - 0.01 * torch.rand(H, generator=gen, device="cuda"))).float())
        if c["carried"]:
            s["s0"] = normal(N, H, dk, dv)
        if c["resets"] > 0:
            s["reset"] = (torch.rand(T, N, generator=gen, device="cuda") < c["resets"]).to(torch.uint8)
        if c["ragged"]:
            s["lengths"] = torch.randint(1, T + 1, (N,), generator=gen, device="cuda", dtype=torch.int32)
            s["lengths"][N // 2] = 0  # an episode of which nothing was recorded
        if c["train"]:
            do = normal(*lead, H, dv, dtype=dt, std=0.1)
            s["do"] = do.transpose(0, 1) if c["batch_first"] else do
            if c["carried"]:
                s["ds_last"] = normal(N, H, dk, dv, std=0.1)
        return s
    Hq, Hk, d = c["q_heads"], c["k_heads"], c["d"]
    split = _wide(c, [(Hq, d), (Hk, d)])
    proj = normal(*lead, (Hq + Hk) * d, dtype=dt, std=2.0)
    q, k = split(proj)
    start = torch.randint(0, 1_000_000 if c["far"] else 1, (N,), generator=gen, device="cuda", dtype=torch.int32)
    s = dict(c, proj=proj, q=q, k=k, split=split, q_weight=normal(d, mean=1.0, std=0.2), k_weight=normal(d, mean=1.0, std=0.2),
             positions=(start[None, :] + torch.arange(T, device="cuda", dtype=torch.int32)[:, None]).contiguous(), freqs=None)
    if c["rotary"]:
        pair = torch.arange(c["rotary"] // 2, device="cuda", dtype=torch.float64)
        s["freqs"] = torch.exp(-math.log(10000.0) * 2.0 * pair / c["rotary"]).float()
    if c["train"]:
        s["dout"] = split(normal(*lead, (Hq + Hk) * d, dtype=dt, std=0.1))
    return s


# ------------------------------------------------------------------ the operators in their plain form
def _chunked(a, b, c, g, cut, live, state, early):
    """y_i = sum over j <= i of exp(g (p_i - p_j)) (a_i b_j) c_j and what the entering state gives, in steps that are live, where
    p counts them and sums do not reach past a cut; the state after the last.  With `early` the first token sees the entering
    state as it is, and the state that comes out has decayed once more.  All [T, N, H, .], in 32 bits."""
    T, N, H, _ = a.shape
    pad = -T % _CHUNK
    n_chunks = (T + pad) // _CHUNK

    def chunks(x):  # [N, H, chunk, token, .]
        x = torch.where(live[..., None, None], x.float(), 0.0)
        x = torch.nn.functional.pad(x, (0, 0, 0, 0, 0, 0, 0, pad))
        return x.view(n_chunks, _CHUNK, N, H, x.shape[-1]).permute(2, 3, 0, 1, 4)

    def marks(x):  # [N, 1, chunk, token]
        return torch.nn.functional.pad(x, (0, 0, 0, pad)).view(n_chunks, _CHUNK, N).permute(2, 0, 1)[:, None]

    a, b, c = chunks(a), chunks(b), chunks(c)
    count = torch.cumsum(marks(live.long()), -1)
    seg = torch.cumsum(marks(cut.long()), -1)
    n, last, g = count[..., -1:], seg[..., -1:], g.view(1, H, 1, 1)

    def power(e):  # exp(g e), 1 for e = 0 whatever g
        e = e.clamp(min=0)
        return torch.where(e == 0, 1.0, torch.exp(g.view(g.shape + (1,) * (e.dim() - 4)) * e))

    away = count[..., :, None] - count[..., None, :]
    order = torch.ones(_CHUNK, _CHUNK, dtype=torch.bool, device=a.device).tril()
    w = torch.where(order & (seg[..., :, None] == seg[..., None, :]), power(away), 0.0)
    y = ((a @ b.transpose(-1, -2)) * w) @ c
    seen = torch.where(seg == 0, power(count - early), 0.0)
    kept = torch.where(seg == last, power(n - count + early), 0.0)
    local = (b * kept[..., None]).transpose(-1, -2) @ c
    carry = torch.where(last == 0, power(n), 0.0)
    if state is None:
        state = torch.zeros(N, H, b.shape[-1], c.shape[-1], device=a.device)
    entering = torch.empty_like(local)
    for i in range(n_chunks):
        entering[:, :, i] = state
        state = torch.where(carry[:, :, i, :, None] == 0, 0.0, state * carry[:, :, i, :, None]) + local[:, :, i]
    y = y + (a @ entering) * seen[..., None]
    return y.permute(2, 3, 0, 1, 4).reshape(T + pad, N, H, -1)[:T], state


def _marks(s):
    dev = s["q"].device
    live = torch.ones(s["T"], s["N"], dtype=torch.bool, device=dev)
    if s["lengths"] is not None:
        live = torch.arange(s["T"], device=dev)[:, None] < s["lengths"][None, :]
    cut = torch.zeros_like(live) if s["reset"] is None else (s["reset"] != 0) & live
    return cut, live


def _plain_attend(s):
    if s["T"] == 1 and s["lengths"] is None:
        q, k, v = s["q"][0].float(), s["k"][0].float(), s["v"][0].float()
        state = k[..., :, None] * v[..., None, :]
        if s["s0"] is not None:
            before = s["s0"] * torch.exp(s["log_decay"])[:, None, None]
            state = state + (before if s["reset"] is None else torch.where((s["reset"][0] != 0)[:, None, None, None], 0.0, before))
        return ((q[..., None, :] @ state)[..., 0, :] * s["scale"]).to(s["q"].dtype)[None], state
    cut, live = _marks(s)
    y, last = _chunked(s["q"], s["k"], s["v"], s["log_decay"], cut, live, s["s0"], 0)
    return (y * s["scale"]).to(s["q"].dtype), last


def _plain_attend_backward(s):
    cut, live = _marks(s)
    g, dt = s["log_decay"], s["q"].dtype
    # dq reads the state that the tokens so far wrote, transposed; dk and dv read its gradient, which runs the other way
    dq, _ = _chunked(s["do"], s["v"], s["k"], g, cut, live, None if s["s0"] is None else s["s0"].transpose(-1, -2), 0)
    q, k, v, do, back = (x.flip(0) for x in (s["q"], s["k"], s["v"], s["do"], live))
    # in reverse a step begins after the one that a reset begins
    again = torch.cat([torch.zeros_like(cut[:1]), cut.flip(0)[:-1]])
    ds = None if s["ds_last"] is None else s["ds_last"] / s["scale"]
    dv, ds0 = _chunked(k, q, do, g, again, back, ds, 1)
    dk, _ = _chunked(v, do, q, g, again, back, None if ds is None else ds.transpose(-1, -2), 1)
    ds0 = torch.where(cut[0][:, None, None, None], 0.0, ds0 * s["scale"])
    return [x.to(dt) for x in (dq * s["scale"], dk.flip(0) * s["scale"], dv.flip(0) * s["scale"])] + [ds0]


def _angles(s):
    """cos and sin [T, N, 1, rotary / 2], of angles in 64 bits."""
    a = s["positions"].double()[..., None, None] * s["freqs"].double()
    return torch.cos(a).float(), torch.sin(a).float()


def _pairs(s, x):
    """The rotated pairs' first and second values, and what is not rotated."""
    R = s["rotary"]
    if s["interleaved"]:
        return x[..., 0:R:2], x[..., 1:R:2], x[..., R:]
    return x[..., :R // 2], x[..., R // 2:R], x[..., R:]


def _unpaired(s, a, b, rest):
    if s["interleaved"]:
        return torch.cat([torch.stack([a, b], -1).flatten(-2), rest], -1)
    return torch.cat([a, b, rest], -1)


def _plain_heads(s, x, weight, turn):
    xf = x.float()
    y = xf * (1.0 / torch.sqrt(xf.square().mean(-1, keepdim=True) + _EPS)) * weight
    if turn is not None:
        a, b, rest = _pairs(s, y)
        y = _unpaired(s, a * turn[0] - b * turn[1], b * turn[0] + a * turn[1], rest)
    return y.to(x.dtype)


def _plain_heads_backward(s, x, weight, dy, turn):
    d = dy.float()
    if turn is not None:
        a, b, rest = _pairs(s, d)
        d = _unpaired(s, a * turn[0] + b * turn[1], b * turn[0] - a * turn[1], rest)
    xf = x.float()
    r = 1.0 / torch.sqrt(xf.square().mean(-1, keepdim=True) + _EPS)
    xhat, g = xf * r, d * weight
    return (r * (g - xhat * (g * xhat).mean(-1, keepdim=True))).to(x.dtype), (d * xhat).sum((0, 1, 2))


# ------------------------------------------------------------------ one pass
@functools.cache
def _ops():
    import paper_2205_01435_gb300 as pkg

    return pkg.load_seq().SequenceOps()


def _run_attend(s):
    if not own:
        o, last = _plain_attend(s)
        if not s["train"]:
            return {"o": o, "s_last": last}
        dq, dk, dv, ds0 = _plain_attend_backward(s)
        return {"o": o, "s_last": last, "dproj": torch.cat([x.flatten(-2) for x in (dq, dk, dv)], -1), "ds0": ds0}
    ops, g, scale = _ops(), s["log_decay"], s["scale"]
    if s["T"] == 1 and not s["train"] and s["lengths"] is None:
        o, last = ops.decay_step(s["q"][0], s["k"][0], s["v"][0], g, s["s0"], scale=scale,
                                 reset=None if s["reset"] is None else s["reset"][0])
        return {"o": o[None], "s_last": last}
    out = None
    if s["batch_first"]:
        out = torch.empty((s["N"], s["T"], s["heads"], s["dv"]), dtype=s["q"].dtype, device="cuda").transpose(0, 1)
    o, last = ops.decay_attention(s["q"], s["k"], s["v"], g, scale=scale, s0=s["s0"], reset=s["reset"], lengths=s["lengths"], out=out)
    if not s["train"]:
        return {"o": o, "s_last": last}
    # the gradients side by side, as the projection's backward product takes them
    dproj = torch.empty_like(s["proj"])
    dq, dk, dv = s["split"](dproj)
    _, _, _, ds0 = ops.decay_attention_backward(s["q"], s["k"], s["v"], g, s["do"], scale=scale, ds_last=s["ds_last"], s0=s["s0"],
                                                reset=s["reset"], lengths=s["lengths"], dq=dq, dk=dk, dv=dv)
    return {"o": o, "s_last": last, "dproj": dproj.transpose(0, 1) if s["batch_first"] else dproj, "ds0": ds0}


def _run_heads(s):
    if not own:
        turn = _angles(s) if s["rotary"] else None
        q, k = _plain_heads(s, s["q"], s["q_weight"], turn), _plain_heads(s, s["k"], s["k_weight"], turn)
        if not s["train"]:
            return {"q": q, "k": k}
        dq, dqw = _plain_heads_backward(s, s["q"], s["q_weight"], s["dout"][0], turn)
        dk, dkw = _plain_heads_backward(s, s["k"], s["k_weight"], s["dout"][1], turn)
        return {"q": q, "k": k, "dproj": torch.cat([dq.flatten(-2), dk.flatten(-2)], -1), "dq_weight": dqw, "dk_weight": dkw}
    kw = dict(q_weight=s["q_weight"], k_weight=s["k_weight"], positions=s["positions"] if s["rotary"] else None, freqs=s["freqs"],
              eps=_EPS, interleaved=s["interleaved"])
    q, k = _ops().head_norm(s["q"], s["k"], **kw)
    if not s["train"]:
        return {"q": q, "k": k}
    dproj = torch.empty_like(s["proj"])
    dq, dk = s["split"](dproj)
    _, _, dqw, dkw = _ops().head_norm_backward(s["q"], s["dout"][0], s["k"], s["dout"][1], dq=dq, dk=dk, **kw)
    return {"q": q, "k": k, "dproj": dproj.transpose(0, 1) if s["batch_first"] else dproj, "dq_weight": dqw, "dk_weight": dkw}


def run(state):
    return _run_attend(state) if state["op"] == "attend" else _run_heads(state)


# ------------------------------------------------------------------ what a pass has to move and compute
def work(case):
    c = case
    b, tokens = {"fp32": 4, "bf16": 2}[c["dtype"]], c["T"] * c["N"]
    if c["op"] == "attend":
        H, dk, dv = c["heads"], c["dk"], c["dv"]
        state = c["N"] * H * dk * dv * 4
        # padded steps are not read but their outputs are written: about half of the steps count
        live = 0.5 if c["ragged"] and c["T"] > 1 else 1.0
        bytes_ = tokens * H * b * (live * (2 * dk + dv) + dv) + state * (2 if c["carried"] else 1) + 4 * H
        bytes_ += (tokens if c["resets"] > 0 else 0) + (4 * c["N"] if c["ragged"] else 0)
        flops = 5 * tokens * live * H * dk * dv  # the recurrence: decay, outer product, product with the query
        if c["train"]:
            bytes_ += tokens * H * b * (live * (2 * dk + 2 * dv) + 2 * dk + dv) + state * (3 if c["carried"] else 1)
            flops += 12 * tokens * live * H * dk * dv
        return {"bytes": bytes_, "flops": flops}
    n = tokens * (c["q_heads"] + c["k_heads"]) * c["d"]
    small = 4 * tokens + 8 * c["d"] + 2 * c["rotary"]
    if not c["train"]:
        return {"bytes": 2 * n * b + small, "flops": 8 * n}
    return {"bytes": 5 * n * b + 2 * small + 8 * c["d"], "flops": 24 * n}


# ------------------------------------------------------------------ the definitions, in 64 bits
def _exact_attend(s):
    """Token by token: S <- lambda S + k v, o = q S, and the gradients back through the same steps."""
    T, N, H, f64 = s["T"], s["N"], s["heads"], torch.float64
    lam = torch.exp(s["log_decay"].double())[None, :, None, None]
    dev = lam.device
    ends = torch.full((N,), T, device=dev) if s["lengths"] is None else s["lengths"].long()
    S = torch.zeros(N, H, s["dk"], s["dv"], dtype=f64, device=dev) if s["s0"] is None else s["s0"].double()
    o = torch.zeros(T, N, H, s["dv"], dtype=f64, device=dev)
    dq = torch.zeros(T, N, H, s["dk"], dtype=f64, device=dev) if s["train"] else None
    keep = [lam.expand(N, H, 1, 1)] * T
    if s["reset"] is not None or s["lengths"] is not None:
        starts = torch.zeros(T, N, dtype=torch.bool, device=dev) if s["reset"] is None else s["reset"] != 0
        on = torch.arange(T, device=dev)[:, None] < ends[None]
        on_ = on[..., None, None, None]
        keep = torch.where(on_, torch.where(starts[..., None, None, None], 0.0, lam), 1.0).unbind(0)
        on = on_.unbind(0)
    else:
        on = None
    rows = [x.double().unbind(0) for x in (s["q"], s["k"], s["v"])]
    do = None if s["do"] is None else s["do"].double().unbind(0)
    for t in range(T):
        q, k, v = (r[t] for r in rows)
        new = torch.addcmul(keep[t] * S, k[..., :, None], v[..., None, :])
        S = new if on is None else torch.where(on[t], new, S)
        here = None if on is None else on[t][..., 0]
        y = torch.matmul(q[..., None, :], S)[..., 0, :]
        o[t] = y if here is None else torch.where(here, y, 0.0)
        if dq is not None:
            y = torch.matmul(S, do[t][..., :, None])[..., 0]
            dq[t] = y if here is None else torch.where(here, y, 0.0)
    scale = s["scale"]
    out = {"o": o * scale, "s_last": S}
    if not s["train"]:
        return out
    G = torch.zeros_like(S) if s["ds_last"] is None else s["ds_last"].double()
    dk, dv = torch.zeros_like(dq), torch.zeros_like(o)
    for t in range(T - 1, -1, -1):
        q, k, v = (r[t] for r in rows)
        full = torch.addcmul(G, q[..., :, None], do[t][..., None, :], value=scale)
        a, b = torch.matmul(full, v[..., :, None])[..., 0], torch.matmul(k[..., None, :], full)[..., 0, :]
        if on is None:
            dk[t], dv[t], G = a, b, keep[t] * full
        else:
            here = on[t][..., 0]
            dk[t], dv[t] = torch.where(here, a, 0.0), torch.where(here, b, 0.0)
            G = torch.where(on[t], keep[t] * full, G)
    return dict(out, dproj=torch.cat([x.flatten(-2) for x in (dq * scale, dk, dv)], -1), ds0=G)


def _exact_heads(s):
    def turned(x, sign):  # as complex numbers
        if not s["rotary"]:
            return x
        z = torch.polar(torch.ones((), dtype=torch.float64, device=x.device),
                        sign * s["positions"].double()[..., None, None] * s["freqs"].double())
        R = s["rotary"]
        z = z * (torch.complex(x[..., 0:R:2], x[..., 1:R:2]) if s["interleaved"] else torch.complex(x[..., :R // 2], x[..., R // 2:R]))
        head = torch.view_as_real(z).flatten(-2) if s["interleaved"] else torch.cat([z.real, z.imag], -1)
        return torch.cat([head, x[..., R:]], -1)

    out, grads = {}, []
    for i, name in enumerate("qk"):
        x, w = s[name].double(), s[name + "_weight"].double()
        root = torch.sqrt((x * x).sum(-1, keepdim=True) / s["d"] + _EPS)
        out[name] = turned(x / root * w, 1.0)
        if s["train"]:
            dy = turned(s["dout"][i].double(), -1.0)
            out[f"d{name}_weight"] = torch.einsum("tnhd,tnhd->d", dy, x / root)
            gw = dy * w
            grads.append(((gw - x * (gw * x).sum(-1, keepdim=True) / (s["d"] * root * root)) / root).flatten(-2))
    if s["train"]:
        out["dproj"] = torch.cat(grads, -1)
    return {k: out[k] for k in ("q", "k", "dproj", "dq_weight", "dk_weight") if k in out}


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_attend(s) if s["op"] == "attend" else _exact_heads(s)
