"""The sequence operators' definitions in 64 bits on the CPU, with the error an fp32 evaluation may have.

Every function returns (value, bound) pairs: the bound follows the operations of an fp32 evaluation
(unit roundoff u = 2^-24) through the definition, from the published errors of the functions used
(expf: 1 ulp; the fast exponential: 2 + 1.173 |x| ulp; reciprocal and reciprocal root: 2 ulp).
``rounded`` adds the rounding of an output's type.
"""
import torch

U = 2.0 ** -24
F64 = torch.float64


def rounded(value, bound, dtype):
    """The bound of a value after rounding to its type (bf16: unit roundoff 2^-8)."""
    u = 2.0 ** -8 if dtype == torch.bfloat16 else U
    return bound + (value.abs() + bound) * u + 1e-37


def check(got, value, bound, what, dtype=None):
    got64 = got.detach().cpu().to(F64)
    tol = rounded(value, bound, dtype or got.dtype)
    assert got64.shape == value.shape, f"{what}: {got64.shape} for {value.shape}"
    off = (got64 - value).abs()
    bad = ~(off <= tol)
    assert not bad.any(), (f"{what}: {int(bad.sum())} of {bad.numel()} values off; worst {float((off / tol).nan_to_num(1e30).max()):.3g} "
                           f"times the bound, first at {bad.nonzero()[0].tolist()}")


# ------------------------------------------------------------------ gated scan
def _gate(p, fast):
    keep, write = torch.sigmoid(p), torch.sigmoid(-p)
    # e = exp(-|p|): 1 ulp, or 2 + 1.173 |p| ulp; then 1 + e, the reciprocal (2 ulp) and a product
    delta = (4 + 2.4 * p.abs() + 10) * U if fast else torch.full_like(p, 10 * U)
    return keep, write, delta


def scan(gate, x, h0=None, reset=None, lengths=None):
    """{h, h_last: (value, bound)}; the inputs as the kernel gets them (any type)."""
    fast = gate.dtype == torch.bfloat16
    gate, x = gate.cpu().to(F64), x.cpu().to(F64)
    T, N, H = gate.shape
    st = torch.zeros(N, H, dtype=F64) if h0 is None else h0.cpu().to(F64)
    err = torch.zeros(N, H, dtype=F64)
    h, hb = torch.zeros(T, N, H, dtype=F64), torch.zeros(T, N, H, dtype=F64)
    keep, write, delta = _gate(gate, fast)
    lens = torch.full((N,), T) if lengths is None else lengths.cpu().long()
    for t in range(T):
        live = (t < lens)[:, None]
        before, eb = st, err
        if reset is not None:
            cut = (reset[t].cpu() != 0)[:, None]
            before, eb = torch.where(cut, 0.0, before), torch.where(cut, 0.0, eb)
        new = keep[t] * before + write[t] * x[t]
        ne = keep[t] * eb + delta[t] * (keep[t] * before.abs() + write[t] * x[t].abs()) + 2 * U * new.abs()
        st, err = torch.where(live, new, st), torch.where(live, ne, err)
        h[t], hb[t] = torch.where(live, new, 0.0), torch.where(live, ne, 0.0)
    # joined spans take the same operations in another order: as much again
    return {"h": (h, 2 * hb), "h_last": (st, 2 * err)}


def scan_backward(gate, x, h, dh, dh_last=None, h0=None, reset=None, lengths=None):
    """{dgate, dx, dh0: (value, bound)}, from the forward's output h as it was rounded."""
    fast = gate.dtype == torch.bfloat16
    gate, x, h, dh = (v.cpu().to(F64) for v in (gate, x, h, dh))
    T, N, H = gate.shape
    keep, write, delta = _gate(gate, fast)
    c = torch.zeros(N, H, dtype=F64) if dh_last is None else dh_last.cpu().to(F64)
    ce = torch.zeros(N, H, dtype=F64)
    out = {k: (torch.zeros(T, N, H, dtype=F64), torch.zeros(T, N, H, dtype=F64)) for k in ("dgate", "dx")}
    lens = torch.full((N,), T) if lengths is None else lengths.cpu().long()
    start = torch.zeros(N, H, dtype=F64) if h0 is None else h0.cpu().to(F64)
    for t in range(T - 1, -1, -1):
        live = (t < lens)[:, None]
        before = h[t - 1] if t else start
        cut = torch.zeros(N, 1, dtype=torch.bool) if reset is None else (reset[t].cpu() != 0)[:, None]
        before = torch.where(cut, 0.0, before)
        L = dh[t] + c
        le = 2 * ce + U * (dh[t].abs() + c.abs())
        dx, dg = L * write[t], L * (before - x[t]) * keep[t] * write[t]
        for k, v, e in (("dx", dx, le * write[t] + (delta[t] + U) * dx.abs()),
                        ("dgate", dg, le * ((before - x[t]) * keep[t] * write[t]).abs() + (2 * delta[t] + 4 * U) * dg.abs())):
            out[k][0][t], out[k][1][t] = torch.where(live, v, 0.0), torch.where(live, e, 0.0)
        nc = torch.where(cut, 0.0, keep[t] * L)
        ne = torch.where(cut, 0.0, keep[t] * (ce + U * (dh[t].abs() + c.abs())) + (delta[t] + U) * nc.abs())
        c, ce = torch.where(live, nc, c), torch.where(live, ne, ce)
    out["dh0"] = (c, 2 * ce)
    return out


# ------------------------------------------------------------------ layer norm
# A sum of D values: at most 32 (or D / 512) one after the other in a thread, then a tree of up to 9
# levels and 16 warps: fewer than 80 roundings for the sizes tested (D <= 20000).
SUM = 80 * U


def norm(x, w, b, eps):
    x = x.cpu().to(F64)
    D = x.shape[-1]
    w = torch.ones(D, dtype=F64) if w is None else w.cpu().to(F64)
    b = torch.zeros(D, dtype=F64) if b is None else b.cpu().to(F64)
    mean = x.mean(-1, keepdim=True)
    me = SUM * x.abs().mean(-1, keepdim=True) + U * mean.abs()
    var = (x - mean).square().mean(-1, keepdim=True)
    # (x - mean): the mean's error, and a rounding; its square's sum
    dev = (x - mean).abs()
    ve = (2 * dev * (me + U * dev) + (me + U * dev) ** 2).mean(-1, keepdim=True) + (SUM + 3 * U) * var + U * (var + eps)
    rstd = 1 / torch.sqrt(var + eps)
    low = torch.clamp(var + eps - ve, min=1e-300)
    re = torch.maximum(1 / torch.sqrt(low) - rstd, rstd * ve / (2 * (var + eps))) + 6 * U * rstd
    y = (x - mean) * rstd * w + b
    ye = w.abs() * ((me + U * dev) * (rstd + re) + dev * re + 3 * U * dev * rstd) + U * (b.abs() + y.abs())
    return {"y": (y, ye), "mean": (mean[..., 0], me[..., 0]), "rstd": (rstd[..., 0], re[..., 0])}


def norm_backward(x, w, mean, rstd, dy):
    """From the statistics as the forward rounded them."""
    x, dy, mean, rstd = (v.cpu().to(F64) for v in (x, dy, mean, rstd))
    D = x.shape[-1]
    w = torch.ones(D, dtype=F64) if w is None else w.cpu().to(F64)
    xh = (x - mean[..., None]) * rstd[..., None]
    g = dy * w
    m1, m2 = g.mean(-1, keepdim=True), (g * xh).mean(-1, keepdim=True)
    e1, e2 = SUM * g.abs().mean(-1, keepdim=True), (SUM + 6 * U) * (g * xh).abs().mean(-1, keepdim=True)
    r = rstd[..., None]
    dx = r * (g - m1 - xh * m2)
    de = r * (e1 + xh.abs() * e2 + 8 * U * (g.abs() + m1.abs() + (xh * m2).abs()))
    lead = tuple(range(x.dim() - 1))
    # rows one after the other in a thread, then warps, slices and CTAs: fewer than 100 roundings
    # for up to 100,000 rows
    dwe = 106 * U * (dy * xh).abs().sum(lead)
    dbe = 100 * U * dy.abs().sum(lead)
    return {"dx": (dx, de), "dw": ((dy * xh).sum(lead), dwe), "db": (dy.sum(lead), dbe)}


# ------------------------------------------------------------------ embedding
def embed(table, tokens, scale):
    table, t = table.cpu().to(F64), tokens.cpu().long()
    ok = (t >= 0) & (t < table.shape[0])
    out = torch.where(ok[..., None], table[torch.where(ok, t, 0)] * scale, 0.0)
    return out, 2 * U * out.abs()


def embed_backward(tokens, dout, V, scale):
    t, d = tokens.cpu().long().reshape(-1), dout.cpu().to(F64).reshape(-1, dout.shape[-1])
    ok = (t >= 0) & (t < V)
    t, d = t[ok], d[ok]
    g = torch.zeros(V, d.shape[1], dtype=F64).index_add_(0, t, d) * scale
    mag = torch.zeros(V, d.shape[1], dtype=F64).index_add_(0, t, d.abs()) * abs(scale)
    count = torch.zeros(V, dtype=F64).index_add_(0, t, torch.ones(len(t), dtype=F64))
    # at most 32 terms in a block, then the blocks in 8 stretches
    adds = torch.minimum(count, 40 + count / 256) + 2
    return g, adds[:, None] * U * mag


# ------------------------------------------------------------------ clipping
def clip(grads, max_norm):
    norm = torch.sqrt(sum((g.cpu().to(F64).square().sum() for g in grads), torch.zeros((), dtype=F64)))
    f = min(1.0, max_norm / float(norm)) if float(norm) > 0 and torch.isfinite(norm) else 1.0
    # squares of 8 values in fp32, then fp64; the root and the factor rounded once
    return norm, 10 * U * norm, [(g.cpu().to(F64) * f, 14 * U * (g.cpu().to(F64) * f).abs()) for g in grads]
