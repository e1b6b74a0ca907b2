"""Thin Python binding of the sequence operators in include/wm_seq.h (ctypes, argument
marshalling only).

``SequenceOps`` owns one handle on one CUDA device.  Its methods take CUDA tensors, allocate
their outputs unless given, and run on the current stream (or ``stream=``) without
synchronising.  There is no CPU fallback.

    ops = SequenceOps()
    e = ops.embed(table, actions, scale=32.0)
    y, mean, rstd = ops.layer_norm(e, weight, bias, want_stats=True)
    h, state = ops.gated_scan(gate, x, h0=state, reset=starts, lengths=lengths)
    dgate, dx, dh0 = ops.gated_scan_backward(gate, x, h, dh, h0=state)
    norm = ops.clip_grads(grads, max_norm=1.0)
    ops.sync()                               # raises WMError on a device-side error
"""
from __future__ import annotations

import ctypes as C

import torch

from . import wm as _wm
from .wm import WM_BF16, WM_FP32, WMError

_lib = _wm._lib
_raw_stream = torch._C._cuda_getCurrentRawStream
_DTYPE = {torch.float32: WM_FP32, torch.bfloat16: WM_BF16}


class wm_seq_view(C.Structure):
    _fields_ = [("data", C.c_void_p), ("stride_t", C.c_longlong), ("stride_n", C.c_longlong)]


class wm_seq_grad(C.Structure):
    _fields_ = [("src", C.c_void_p), ("dst", C.c_void_p), ("n", C.c_longlong), ("dtype", C.c_int)]


def _declare():
    P, I, L, F, V = C.c_void_p, C.c_int, C.c_longlong, C.c_float, C.c_void_p  # V: a view's address
    sig = {
        "wm_seq_create": [C.POINTER(P)],
        "wm_seq_sync": [P],
        "wm_seq_inject_wait_timeout": [P, C.c_uint],
        "wm_seq_embed": [P, I, L, I, I, P, P, F, P, P],
        "wm_seq_embed_backward": [P, I, L, I, I, P, P, F, P, P],
        "wm_seq_layer_norm": [P, I, L, I, P, L, P, P, F, P, L, P, P, P],
        "wm_seq_layer_norm_backward": [P, I, L, I, P, L, P, P, P, P, L, P, L, P, P, P],
        "wm_seq_gated_scan": [P, I, L, I, I, V, V, P, P, P, V, P, P],
        "wm_seq_gated_scan_backward": [P, I, L, I, I, V, V, P, P, P, V, V, P, V, V, P, P],
        "wm_seq_clip": [P, I, P, F, P, P],
    }
    for name, args in sig.items():
        f = getattr(_lib, name)
        f.argtypes, f.restype = args, C.c_int
    _lib.wm_seq_last_error.argtypes, _lib.wm_seq_last_error.restype = [P], C.c_char_p
    _lib.wm_seq_last_launches.argtypes, _lib.wm_seq_last_launches.restype = [P], C.c_int
    _lib.wm_seq_destroy.argtypes, _lib.wm_seq_destroy.restype = [P], None


_declare()


def _need(ok, why):
    if not ok:
        raise ValueError(why)


class SequenceOps:
    """Owns one wm_seq handle on one CUDA device."""

    def __init__(self, device: int | torch.device | None = None):
        if device is None:
            index = torch.cuda.current_device()
        else:
            index = device if isinstance(device, int) else torch.device(device).index
            index = torch.cuda.current_device() if index is None else index
        self.device = torch.device("cuda", index)
        h = C.c_void_p()
        with torch.cuda.device(self.device):
            st = _lib.wm_seq_create(C.byref(h))
        if st:
            raise WMError(st, "wm_seq_create failed")
        self.h = h.value
        # the views of a call, filled anew by each
        self._views = [wm_seq_view() for _ in range(6)]
        self._at = [C.addressof(v) for v in self._views]

    def close(self):
        if getattr(self, "h", None):
            _lib.wm_seq_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # ------------------------------------------------------------- helpers
    def _check(self, st: int, what: str):
        if st:
            raise WMError(st, _lib.wm_seq_last_error(self.h).decode() or what)

    def _stream(self) -> int:
        # the stream's address without a Stream object: 0.1 us against 2 us, of a call of 10
        return _raw_stream(self.device.index)

    def _elsewhere(self, stream, method, args, kwargs):
        """The call on another stream: its outputs are allocated there, and its inputs' memory is
        not used again before it is done."""
        s = stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(int(stream), device=self.device)
        with torch.cuda.stream(s):
            out = method(*args, **kwargs)

        def mark(v):
            if isinstance(v, torch.Tensor) and v.is_cuda:
                v.record_stream(s)
            elif isinstance(v, (list, tuple)):
                for x in v:
                    mark(x)

        mark(args)
        mark(list(kwargs.values()))
        return out

    def _dtype(self, t: torch.Tensor) -> int:
        d = _DTYPE.get(t.dtype)
        _need(d is not None, f"float32 or bfloat16 tensors are needed, got {t.dtype}")
        return d

    def _flat(self, t, dtype, shape, what):
        """The address of a dense tensor of this type and shape (None: 0)."""
        if t is None:
            return None
        if t.dtype != dtype or t.device != self.device or tuple(t.shape) != shape or not t.is_contiguous():
            raise ValueError(f"{what}: a contiguous {dtype} tensor of shape {shape} on {self.device} is needed, "
                             f"got {t.dtype} {tuple(t.shape)} on {t.device}")
        return t.data_ptr()

    def _view(self, i, t, dtype, shape, what):
        """View i of the call: a [T, N, H] tensor whose last axis is dense."""
        if t.dtype != dtype or t.device != self.device or t.shape != shape or (t.stride(2) != 1 and shape[2] > 1):
            raise ValueError(f"{what}: a {dtype} tensor of shape {tuple(shape)} on {self.device} with a dense last axis is "
                             f"needed, got {t.dtype} {tuple(t.shape)} on {t.device}")
        v = self._views[i]
        v.data = t.data_ptr()
        v.stride_t, v.stride_n = t.stride(0), t.stride(1)
        return self._at[i]

    def _rows(self, t, what):
        """(rows, D, row stride) of a tensor whose leading axes are one run of rows."""
        _need(t.device == self.device, f"{what} must be on {self.device}")
        _need(t.dim() >= 1, f"{what} needs at least one axis")
        D = t.shape[-1]
        _need(D <= 1 or t.stride(-1) == 1, f"{what}: its last axis must be dense")
        if t.is_contiguous():
            return t.numel() // D if D else 0, D, D
        r = t.unsqueeze(0) if t.dim() == 1 else t.flatten(0, -2) if t.dim() > 2 else t
        _need(r.data_ptr() == t.data_ptr(), f"{what}: its leading axes must be one run of rows with a fixed stride")
        return r.shape[0], D, r.stride(0)

    # ------------------------------------------------------------- embedding
    def embed(self, table, tokens, scale: float = 1.0, out=None, stream=None):
        """wm_seq_embed: scale * table[tokens] (0 where a token is negative); tokens int32 of any shape."""
        if stream is not None:
            return self._elsewhere(stream, self.embed, (table, tokens, scale, out), {})
        _need(table.dim() == 2, "table [V, D] is needed")
        dt = self._dtype(table)
        V, D = table.shape
        shape = tuple(tokens.shape)
        if out is None:
            out = torch.empty(shape + (D,), dtype=table.dtype, device=self.device)
        self._check(_lib.wm_seq_embed(self.h, dt, tokens.numel(), V, D, self._flat(table, table.dtype, (V, D), "table"),
                                      self._flat(tokens, torch.int32, shape, "tokens"), scale,
                                      self._flat(out, table.dtype, shape + (D,), "out"), self._stream()), "wm_seq_embed")
        return out

    def embed_backward(self, tokens, dout, vocab: int, scale: float = 1.0, out=None, stream=None):
        """wm_seq_embed_backward: the gradient [vocab, D] of embed's table."""
        if stream is not None:
            return self._elsewhere(stream, self.embed_backward, (tokens, dout, vocab, scale, out), {})
        dt = self._dtype(dout)
        shape, D = tuple(tokens.shape), dout.shape[-1]
        if out is None:
            out = torch.empty((vocab, D), dtype=dout.dtype, device=self.device)
        self._check(_lib.wm_seq_embed_backward(self.h, dt, tokens.numel(), vocab, D,
                                               self._flat(tokens, torch.int32, shape, "tokens"),
                                               self._flat(dout, dout.dtype, shape + (D,), "dout"), scale,
                                               self._flat(out, dout.dtype, (vocab, D), "out"), self._stream()),
                    "wm_seq_embed_backward")
        return out

    # ------------------------------------------------------------- layer norm
    def layer_norm(self, x, weight=None, bias=None, eps: float = 1e-5, want_stats: bool = False, out=None, stream=None):
        """wm_seq_layer_norm over the last axis; (y, mean, rstd) with want_stats.  out may be x."""
        if stream is not None:
            return self._elsewhere(stream, self.layer_norm, (x, weight, bias, eps, want_stats, out), {})
        dt = self._dtype(x)
        rows, D, ldx = self._rows(x, "x")
        if out is None:
            out = torch.empty(x.shape, dtype=x.dtype, device=self.device)
            ldy = D
        else:
            _need(out.shape == x.shape and out.dtype == x.dtype, "out must have x's shape and type")
            _, _, ldy = self._rows(out, "out")
        mean = rstd = None
        if want_stats:
            mean, rstd = torch.empty((2,) + tuple(x.shape[:-1]), device=self.device).unbind(0)
        self._check(_lib.wm_seq_layer_norm(self.h, dt, rows, D, x.data_ptr(), ldx,
                                           self._flat(weight, torch.float32, (D,), "weight"),
                                           self._flat(bias, torch.float32, (D,), "bias"), eps, out.data_ptr(), ldy,
                                           mean.data_ptr() if want_stats else None, rstd.data_ptr() if want_stats else None,
                                           self._stream()), "wm_seq_layer_norm")
        return (out, mean, rstd) if want_stats else out

    def layer_norm_backward(self, x, weight, mean, rstd, dy, dx=None, want_params: bool = True, stream=None):
        """wm_seq_layer_norm_backward: (dx, dweight, dbias), the last two None without want_params.  dx may be dy."""
        if stream is not None:
            return self._elsewhere(stream, self.layer_norm_backward, (x, weight, mean, rstd, dy, dx, want_params), {})
        dt = self._dtype(x)
        rows, D, ldx = self._rows(x, "x")
        _need(dy.shape == x.shape and dy.dtype == x.dtype, "dy must have x's shape and type")
        _, _, lddy = self._rows(dy, "dy")
        if dx is None:
            dx = torch.empty(x.shape, dtype=x.dtype, device=self.device)
            lddx = D
        else:
            _need(dx.shape == x.shape and dx.dtype == x.dtype, "dx must have x's shape and type")
            _, _, lddx = self._rows(dx, "dx")
        dw = db = None
        if want_params:
            dw, db = torch.empty((2, D), device=self.device).unbind(0)
        lead = tuple(x.shape[:-1])
        self._check(_lib.wm_seq_layer_norm_backward(self.h, dt, rows, D, x.data_ptr(), ldx,
                                                    self._flat(weight, torch.float32, (D,), "weight"),
                                                    self._flat(mean, torch.float32, lead, "mean"),
                                                    self._flat(rstd, torch.float32, lead, "rstd"), dy.data_ptr(), lddy,
                                                    dx.data_ptr(), lddx, dw.data_ptr() if want_params else None,
                                                    db.data_ptr() if want_params else None, self._stream()),
                    "wm_seq_layer_norm_backward")
        return dx, dw, db

    # ------------------------------------------------------------- gated scan
    def gated_scan(self, gate, x, h0=None, reset=None, lengths=None, out=None, want_last: bool = True, h_last=None,
                   stream=None):
        """wm_seq_gated_scan over [T, N, H]; (h, h_last).  gate, x and out may be strided over T and N
        (columns of a wider array, a transposed batch-major array); h_last may be h0."""
        if stream is not None:
            return self._elsewhere(stream, self.gated_scan, (gate, x, h0, reset, lengths, out, want_last, h_last), {})
        dt = self._dtype(gate)
        _need(gate.dim() == 3, "gate [T, N, H] is needed")
        shape, dtype = gate.shape, gate.dtype
        T, N, H = shape
        if out is None:
            out = torch.empty(shape, dtype=dtype, device=self.device)
        if h_last is None and want_last:
            h_last = torch.empty((N, H), device=self.device)
        self._check(_lib.wm_seq_gated_scan(self.h, dt, T, N, H, self._view(0, gate, dtype, shape, "gate"),
                                           self._view(1, x, dtype, shape, "x"),
                                           self._flat(h0, torch.float32, (N, H), "h0"),
                                           self._flat(reset, torch.uint8, (T, N), "reset"),
                                           self._flat(lengths, torch.int32, (N,), "lengths"),
                                           self._view(2, out, dtype, shape, "out"),
                                           self._flat(h_last, torch.float32, (N, H), "h_last"), self._stream()),
                    "wm_seq_gated_scan")
        return out, h_last

    def gated_step(self, gate, x, state, reset=None, out=None, out_state=None, stream=None):
        """One step of N sequences: gate, x [N, H] and the state [N, H] fp32 (or None) give (h, state').
        out_state may be the state itself."""
        if stream is not None:
            return self._elsewhere(stream, self.gated_step, (gate, x, state, reset, out, out_state), {})
        h, state = self.gated_scan(gate.unsqueeze(0), x.unsqueeze(0), state, None if reset is None else reset.unsqueeze(0),
                                   None, None if out is None else out.unsqueeze(0), True, out_state)
        return (h.squeeze(0) if out is None else out), state

    def gated_scan_backward(self, gate, x, h, dh, dh_last=None, h0=None, reset=None, lengths=None, dgate=None, dx=None,
                            want_dh0: bool = True, stream=None):
        """wm_seq_gated_scan_backward: (dgate, dx, dh0); dgate and dx may be given, strided as in gated_scan."""
        if stream is not None:
            return self._elsewhere(stream, self.gated_scan_backward,
                                   (gate, x, h, dh, dh_last, h0, reset, lengths, dgate, dx, want_dh0), {})
        dt = self._dtype(gate)
        _need(gate.dim() == 3, "gate [T, N, H] is needed")
        shape, dtype = gate.shape, gate.dtype
        T, N, H = shape
        if dgate is None:
            dgate = torch.empty(shape, dtype=dtype, device=self.device)
        if dx is None:
            dx = torch.empty(shape, dtype=dtype, device=self.device)
        dh0 = torch.empty((N, H), device=self.device) if want_dh0 else None
        self._check(_lib.wm_seq_gated_scan_backward(
            self.h, dt, T, N, H, self._view(0, gate, dtype, shape, "gate"), self._view(1, x, dtype, shape, "x"),
            self._flat(h0, torch.float32, (N, H), "h0"), self._flat(reset, torch.uint8, (T, N), "reset"),
            self._flat(lengths, torch.int32, (N,), "lengths"), self._view(2, h, dtype, shape, "h"),
            self._view(3, dh, dtype, shape, "dh"), self._flat(dh_last, torch.float32, (N, H), "dh_last"),
            self._view(4, dgate, dtype, shape, "dgate"), self._view(5, dx, dtype, shape, "dx"),
            None if dh0 is None else dh0.data_ptr(), self._stream()), "wm_seq_gated_scan_backward")
        return dgate, dx, dh0

    # ------------------------------------------------------------- clipping
    def clip_grads(self, grads, max_norm: float, out=None, stream=None):
        """wm_seq_clip: the global norm [] of the gradients, which are scaled to it in place (or into `out`,
        tensors of the same sizes and types).  max_norm = inf only measures."""
        if stream is not None:
            return self._elsewhere(stream, self.clip_grads, (grads, max_norm, out), {})
        n = len(grads)
        _need(out is None or len(out) == n, "out needs a tensor for each gradient")
        table = (wm_seq_grad * n)()
        for i, g in enumerate(grads):
            o = g if out is None else out[i]
            if g.device != self.device or not g.is_contiguous() or not (
                    o is g or (o.dtype == g.dtype and o.shape == g.shape and o.is_contiguous() and o.device == self.device)):
                raise ValueError(f"gradient {i}: contiguous tensors on {self.device}, out of the same shape and type, are needed")
            table[i] = (g.data_ptr(), o.data_ptr(), g.numel(), self._dtype(g))
        norm = torch.empty((), device=self.device)
        self._check(_lib.wm_seq_clip(self.h, n, table, max_norm, norm.data_ptr(), self._stream()), "wm_seq_clip")
        return norm

    # ------------------------------------------------------------- status
    def sync(self):
        """Waits for the device; raises WMError on a device-side error since the last call."""
        self._check(_lib.wm_seq_sync(self.h), "wm_seq_sync")

    def inject_wait_timeout(self, polls: int):
        """wm_seq_inject_wait_timeout: a wait of the next long scan gives up (tests of the timeout path)."""
        self._check(_lib.wm_seq_inject_wait_timeout(self.h, int(polls)), "wm_seq_inject_wait_timeout")

    @property
    def last_launches(self) -> int:
        return int(_lib.wm_seq_last_launches(self.h))
