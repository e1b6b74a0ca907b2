"""Decayed linear attention and the head norm by their definitions in 64 bits on the CPU, with the error that an evaluation
in fp32 (or bf16 factors with fp32 sums) may have.

Values are (value, bound): the bound follows the operations.  A rounding to bf16 is off by at most 2^-8 of the value, to fp32
by U = 2^-24.
"""
import torch

U = 2.0 ** -24
B = 2.0 ** -8
F64 = torch.float64


# ------------------------------------------------------------------ decayed attention
def _walk(a, b, c, g, keep, live, state, order, factors):
    """F_t = keep_t F + b_t c_t^T, y_t = F_t^T a_t over the steps in `order` ([T, N, H, .], keep [T, N, H], live [T, N]).
    Returns y, its bound, the last state and its bound.  `factors`: the products and the state were rounded to bf16 as factors."""
    T, N, H, da = a.shape
    dc = c.shape[-1]
    F = torch.zeros(N, H, da, dc, dtype=F64) if state is None else state.clone()
    M = F.abs()       # what the state's sums add up to without signs
    R = F.abs()       # the largest state that may have been rounded on the way, as this step sees it
    y, yb = torch.zeros(T, N, H, dc, dtype=F64), torch.zeros(T, N, H, dc, dtype=F64)
    # sums: da terms in a product, 128 in a chunk (two levels), da from the state; weights and their products; the carried
    # state is rounded twice a chunk, and its factor is off by |n g| U + 2 U, where n |g| lambda^n < 0.4
    n = 2 * da + 300 + 8 * (T // 64 + 1)
    order = list(order)
    if factors and order:
        # rounded products of a chunk's tokens, whatever the chunks are: of all tokens that a step sees
        kp = torch.where(live[..., None], keep, 1.0)[order].permute(1, 2, 0)
        fall, cut = torch.where(kp > 0, torch.log(kp), 0.0).cumsum(-1), (kp == 0).long().cumsum(-1)
        sees = torch.ones(len(order), len(order), dtype=torch.bool).tril() & (cut[..., :, None] == cut[..., None, :])
        w = torch.where(sees, torch.exp((fall[..., :, None] - fall[..., None, :]).clamp(max=0)), 0.0)
        pa, pb, pc = (x[order].permute(1, 2, 0, 3) for x in (a, b, c))
        prod = (((pa @ pb.transpose(-1, -2)).abs() * w) @ pc.abs()).permute(2, 0, 1, 3)
    for i, t in enumerate(order):
        on = live[t][:, None, None, None]
        k = keep[t][:, :, None, None]
        nf = torch.where(k == 0, 0.0, k * F) + b[t][..., :, None] * c[t][..., None, :]
        nm = torch.where(k == 0, 0.0, k * M) + b[t][..., :, None].abs() * c[t][..., None, :].abs()
        nr = torch.maximum(torch.where(k == 0, 0.0, k * R), nf.abs())
        F, M, R = torch.where(on, nf, F), torch.where(on, nm, M), torch.where(on, nr, R)
        at = a[t][..., :, None]
        y[t] = torch.where(on[..., 0], (F * at).sum(-2), 0.0)
        bound = n * U * (M * at.abs()).sum(-2)
        if factors:  # (or the rounded state)
            bound = bound + 1.01 * B * (prod[i] + (R * at.abs()).sum(-2))
        yb[t] = torch.where(on[..., 0], bound, 0.0)
    return y, yb, F, n * U * M


def _marks(T, N, H, g, reset, lengths):
    live = torch.ones(T, N, dtype=torch.bool) if lengths is None else torch.arange(T)[:, None] < lengths.cpu().long()[None]
    cut = torch.zeros(T, N, dtype=torch.bool) if reset is None else (reset.cpu() != 0) & live
    return live, cut, torch.exp(g.cpu().to(F64))


def _clean(x, live):
    return torch.where(live[..., None, None], x.cpu().to(F64), 0.0)


def attend(q, k, v, g, scale, s0=None, reset=None, lengths=None, factors=None):
    """{o, s_last: (value, bound)}; `factors`: rounded to bf16 as factors of products (by default in bf16)."""
    T, N, H, _ = q.shape
    factors = q.dtype == torch.bfloat16 if factors is None else factors
    live, cut, lam = _marks(T, N, H, g, reset, lengths)
    keep = torch.where(cut[..., None], 0.0, lam.expand(T, N, H))
    y, yb, F, fb = _walk(_clean(q, live) * scale, _clean(k, live), _clean(v, live), g, keep, live,
                         None if s0 is None else s0.cpu().to(F64), range(T), factors)
    return {"o": (y, yb), "s_last": (F, fb)}


def attend_backward(q, k, v, g, scale, do, ds_last=None, s0=None, reset=None, lengths=None, factors=None):
    """{dq, dk, dv, ds0: (value, bound)}."""
    T, N, H, _ = q.shape
    factors = q.dtype == torch.bfloat16 if factors is None else factors
    live, cut, lam = _marks(T, N, H, g, reset, lengths)
    q, k, v, do = (_clean(x, live) for x in (q, k, v, do))
    keep = torch.where(cut[..., None], 0.0, lam.expand(T, N, H))
    first = None if s0 is None else s0.cpu().to(F64).transpose(-1, -2)
    out = {"dq": _walk(do * scale, v, k, g, keep, live, first, range(T), factors)[:2]}
    # into a step from the one after it: not where that begins an episode; the gradient of the last state enters as it is
    back = torch.cat([keep[1:], torch.ones(1, N, H, dtype=F64)])
    last = torch.full((N,), T) if lengths is None else lengths.cpu().long()
    for n in range(N):
        if last[n] > 0:
            back[last[n] - 1, n] = 1.0
    ds = None if ds_last is None else ds_last.cpu().to(F64)
    dv = _walk(k, q * scale, do, g, back, live, ds, range(T - 1, -1, -1), factors)
    dk = _walk(v, do, q * scale, g, back, live, None if ds is None else ds.transpose(-1, -2), range(T - 1, -1, -1), factors)
    out["dv"], out["dk"] = dv[:2], dk[:2]
    k0 = torch.where((last == 0)[:, None], 1.0, keep[0] if T else torch.ones(N, H, dtype=F64))[..., None, None]
    out["ds0"] = (torch.where(k0 == 0, 0.0, k0 * dv[2]), k0 * (dv[3] + 4 * U * dv[2].abs()))
    return out


# ------------------------------------------------------------------ head norm
def _turn(x, e, rotary, interleaved, angle, sign):
    """x [T, N, heads, D] with errors e, turned by sign * angle [T, N, rotary / 2]; the angle's cosine and sine are off by 12 U
    (an angle in turns rounded to fp32, 4 U in half turns; 2 ulp of the functions) and what the frequency's 53 bits leave."""
    if rotary == 0:
        return x, e
    i = torch.arange(rotary // 2)
    ia, ib = (2 * i, 2 * i + 1) if interleaved else (i, i + rotary // 2)
    ang = angle[:, :, None, :]
    cs, sn, off = torch.cos(ang), sign * torch.sin(ang), 14 * U + ang.abs() * 2.0 ** -51
    y, ye = x.clone(), e.clone()
    a, b = x[..., ia], x[..., ib]
    y[..., ia], y[..., ib] = a * cs - b * sn, b * cs + a * sn
    mix = (off + 3 * U) * (a.abs() + b.abs()) + e[..., ia] + e[..., ib]
    ye[..., ia], ye[..., ib] = mix, mix
    return y, ye


def _norm(x, eps):
    D = x.shape[-1]
    r = 1 / torch.sqrt(x.square().mean(-1, keepdim=True) + eps)
    return r, (D + 12) * U * r  # D terms at most one after the other; the root and the quotient


def head_norm(x, w, eps, positions, freqs, interleaved):
    x = x.cpu().to(F64)
    w = torch.ones(x.shape[-1], dtype=F64) if w is None else w.cpu().to(F64)
    r, re = _norm(x, eps)
    y = x * r * w
    e = (x * w).abs() * re + 3 * U * y.abs()
    rotary = 0 if freqs is None else 2 * len(freqs)
    angle = None if freqs is None else positions.cpu().to(F64)[..., None] * freqs.cpu().to(F64)
    return _turn(y, e, rotary, interleaved, angle, 1.0)


def head_norm_backward(x, w, eps, positions, freqs, interleaved, dy):
    """{dx, dw: (value, bound)}."""
    x, dy = x.cpu().to(F64), dy.cpu().to(F64)
    D = x.shape[-1]
    w = torch.ones(D, dtype=F64) if w is None else w.cpu().to(F64)
    r, re = _norm(x, eps)
    rotary = 0 if freqs is None else 2 * len(freqs)
    angle = None if freqs is None else positions.cpu().to(F64)[..., None] * freqs.cpu().to(F64)
    d, de = _turn(dy, torch.zeros_like(dy), rotary, interleaved, angle, -1.0)
    g, ge = d * w, de * w.abs() + U * (d * w).abs()
    m = (g * x).mean(-1, keepdim=True)
    me = ((D + 4) * U * (g * x).abs() + ge * x.abs()).mean(-1, keepdim=True)
    dx = r * (g - x * r * r * m)
    dxe = r * (ge + (x * r * r).abs() * me + 4 * U * (g.abs() + (x * r * r * m).abs())) + 3 * re * (g.abs() + 3 * (x * r * r * m).abs())
    xh = x * r
    rows = x.numel() // D
    # a thread's rows one after the other, then up to 256 groups of a CTA, then the CTAs
    dwe = ((d * xh).abs() * (min(rows, 2000) + 400) * U + de * xh.abs() + (d * x).abs() * re).sum((0, 1, 2))
    return {"dx": (dx, dxe), "dw": ((d * xh).sum((0, 1, 2)), dwe)}
