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
import sys
from array import array

import torch

from . import wm as _wm
from .wm import WM_BF16, WM_FP32, WMError

_lib = _wm._lib
# the current stream's address without a Stream object: 0.1 us against 2 us, of a call of 10
_raw_stream = torch._C._cuda_getCurrentRawStream
_DTYPE = {torch.float32: WM_FP32, torch.bfloat16: WM_BF16}


class wm_seq_view(C.Structure):
    _fields_ = [("data", C.c_void_p), ("stride_t", C.c_longlong), ("stride_n", C.c_longlong)]


class wm_seq_grad(C.Structure):
    _fields_ = [("src", C.c_void_p), ("dst", C.c_void_p), ("n", C.c_longlong), ("dtype", C.c_int)]


assert C.sizeof(wm_seq_grad) == 32 and wm_seq_grad.dtype.offset == 24 and sys.byteorder == "little"


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
        self._index = index
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

    # Checks of types, shapes and strides; that an array is memory of the handle's device, and aligned,
    # the library checks itself.
    def _dtype(self, t: torch.Tensor) -> int:
        d = _DTYPE.get(t.dtype)
        if d is None:
            raise ValueError(f"float32 or bfloat16 tensors are needed, got {t.dtype}")
        return d

    def _flat(self, t, dtype, shape, what):
        """The address of a dense tensor of this type and shape (None: 0)."""
        if t is None:
            return None
        if t.dtype is not dtype or t.shape != shape or not t.is_contiguous():
            raise ValueError(f"{what}: a contiguous {dtype} tensor of shape {tuple(shape)} is needed, got {t.dtype} {tuple(t.shape)}")
        return t.data_ptr()

    def _view(self, i, t, dtype, shape, what):
        """View i of the call: a [T, N, H] tensor whose last axis is dense."""
        st, sn, sh = t.stride() if t.dim() == 3 else (0, 0, 0)
        if t.dtype is not dtype or t.shape != shape or (sh != 1 and shape[2] > 1):
            raise ValueError(f"{what}: a {dtype} tensor of shape {tuple(shape)} with a dense last axis is needed, "
                             f"got {t.dtype} {tuple(t.shape)}")
        v = self._views[i]
        v.data = t.data_ptr()
        v.stride_t = st
        v.stride_n = sn
        return self._at[i]

    def _row(self, i, t, dtype, shape, what):
        """View i of a one-step call: a [N, H] tensor whose last axis is dense."""
        sn, sh = t.stride() if t.dim() == 2 else (0, 0)
        if t.dtype is not dtype or t.shape != shape or (sh != 1 and shape[1] > 1):
            raise ValueError(f"{what}: a {dtype} tensor of shape {tuple(shape)} with a dense last axis is needed, "
                             f"got {t.dtype} {tuple(t.shape)}")
        v = self._views[i]
        v.data = t.data_ptr()
        v.stride_t = 0
        v.stride_n = sn
        return self._at[i]

    def _rows(self, t, what):
        """The row stride of a tensor whose leading axes are one run of rows."""
        n = t.dim()
        if n and t.is_contiguous():
            return t.shape[-1]
        _need(n >= 1 and (t.shape[-1] <= 1 or t.stride(-1) == 1), f"{what}: its last axis must be dense")
        if n == 2:
            return t.stride(0)
        if n == 1:
            return t.shape[0]
        r = t.flatten(0, -2)
        _need(r.data_ptr() == t.data_ptr(), f"{what}: its leading axes must be one run of rows with a fixed stride")
        return r.stride(0)

    # ------------------------------------------------------------- embedding
    def embed(self, table, tokens, scale: float = 1.0, out=None, stream=None):
        """wm_seq_embed: scale * table[tokens] (0 where a token is negative); tokens int32 of any shape."""
        if stream is not None:
            return self._elsewhere(stream, self.embed, (table, tokens, scale, out), {})
        _need(table.dim() == 2, "table [V, D] is needed")
        dtype, shape = table.dtype, tokens.shape
        V, D = table.shape
        full = (*shape, D)
        if out is None:
            out = torch.empty(full, dtype=dtype, device=self.device)
        st = _lib.wm_seq_embed(self.h, self._dtype(table), tokens.numel(), V, D, self._flat(table, dtype, (V, D), "table"),
                               self._flat(tokens, torch.int32, shape, "tokens"), scale, self._flat(out, dtype, full, "out"),
                               _raw_stream(self._index))
        if st:
            self._check(st, "wm_seq_embed")
        return out

    def embed_backward(self, tokens, dout, vocab: int, scale: float = 1.0, out=None, stream=None):
        """wm_seq_embed_backward: the gradient [vocab, D] of embed's table."""
        if stream is not None:
            return self._elsewhere(stream, self.embed_backward, (tokens, dout, vocab, scale, out), {})
        dtype, shape, D = dout.dtype, tokens.shape, dout.shape[-1]
        if out is None:
            out = torch.empty((vocab, D), dtype=dtype, device=self.device)
        st = _lib.wm_seq_embed_backward(self.h, self._dtype(dout), tokens.numel(), vocab, D,
                                        self._flat(tokens, torch.int32, shape, "tokens"),
                                        self._flat(dout, dtype, (*shape, D), "dout"), scale,
                                        self._flat(out, dtype, (vocab, D), "out"), _raw_stream(self._index))
        if st:
            self._check(st, "wm_seq_embed_backward")
        return out

    # ------------------------------------------------------------- layer norm
    def layer_norm(self, x, weight=None, bias=None, eps: float = 1e-5, want_stats: bool = False, out=None, stream=None):
        """wm_seq_layer_norm over the last axis; (y, mean, rstd) with want_stats.  out may be x."""
        if stream is not None:
            return self._elsewhere(stream, self.layer_norm, (x, weight, bias, eps, want_stats, out), {})
        dtype, shape = x.dtype, x.shape
        ldx = ldy = self._rows(x, "x")
        D = shape[-1]
        if out is None:
            out = torch.empty(shape, dtype=dtype, device=self.device)
            ldy = D
        elif out is not x:
            _need(out.shape == shape and out.dtype is dtype, "out must have x's shape and type")
            ldy = self._rows(out, "out")
        mean = rstd = pm = pr = None
        if want_stats:
            mean = torch.empty(shape[:-1], device=self.device)
            rstd = torch.empty(shape[:-1], device=self.device)
            pm, pr = mean.data_ptr(), rstd.data_ptr()
        par = (D,)
        st = _lib.wm_seq_layer_norm(self.h, self._dtype(x), x.numel() // D if D else 0, D, x.data_ptr(), ldx,
                                    self._flat(weight, torch.float32, par, "weight"),
                                    self._flat(bias, torch.float32, par, "bias"), eps, out.data_ptr(), ldy, pm, pr,
                                    _raw_stream(self._index))
        if st:
            self._check(st, "wm_seq_layer_norm")
        return (out, mean, rstd) if want_stats else out

    def layer_norm_backward(self, x, weight, mean, rstd, dy, dx=None, want_params: bool = True, stream=None):
        """wm_seq_layer_norm_backward: (dx, dweight, dbias), the last two None without want_params.  dx may be dy."""
        if stream is not None:
            return self._elsewhere(stream, self.layer_norm_backward, (x, weight, mean, rstd, dy, dx, want_params), {})
        dtype, shape = x.dtype, x.shape
        ldx = self._rows(x, "x")
        D = shape[-1]
        _need(dy.shape == shape and dy.dtype is dtype, "dy must have x's shape and type")
        lddy = lddx = self._rows(dy, "dy")
        if dx is None:
            dx = torch.empty(shape, dtype=dtype, device=self.device)
            lddx = D
        elif dx is not dy:
            _need(dx.shape == shape and dx.dtype is dtype, "dx must have x's shape and type")
            lddx = self._rows(dx, "dx")
        dw = db = pw = pb = None
        par, lead = (D,), shape[:-1]
        if want_params:
            dw = torch.empty(par, device=self.device)
            db = torch.empty(par, device=self.device)
            pw, pb = dw.data_ptr(), db.data_ptr()
        st = _lib.wm_seq_layer_norm_backward(self.h, self._dtype(x), x.numel() // D if D else 0, D, x.data_ptr(), ldx,
                                             self._flat(weight, torch.float32, par, "weight"),
                                             self._flat(mean, torch.float32, lead, "mean"),
                                             self._flat(rstd, torch.float32, lead, "rstd"), dy.data_ptr(), lddy,
                                             dx.data_ptr(), lddx, pw, pb, _raw_stream(self._index))
        if st:
            self._check(st, "wm_seq_layer_norm_backward")
        return dx, dw, db

    # ------------------------------------------------------------- gated scan
    def gated_scan(self, gate, x, h0=None, reset=None, lengths=None, out=None, want_last: bool = True, h_last=None,
                   stream=None):
        """wm_seq_gated_scan over [T, N, H]; (h, h_last).  gate, x and out may be strided over T and N
        (columns of a wider array, a transposed batch-major array); h_last may be h0."""
        if stream is not None:
            return self._elsewhere(stream, self.gated_scan, (gate, x, h0, reset, lengths, out, want_last, h_last), {})
        dtype, shape = gate.dtype, gate.shape
        _need(len(shape) == 3, "gate [T, N, H] is needed")
        T, N, H = shape
        if out is None:
            out = torch.empty(shape, dtype=dtype, device=self.device)
        nh = (N, H)
        if h_last is None and want_last:
            h_last = torch.empty(nh, device=self.device)
        st = _lib.wm_seq_gated_scan(self.h, self._dtype(gate), T, N, H, self._view(0, gate, dtype, shape, "gate"),
                                    self._view(1, x, dtype, shape, "x"), self._flat(h0, torch.float32, nh, "h0"),
                                    self._flat(reset, torch.uint8, (T, N), "reset"),
                                    self._flat(lengths, torch.int32, (N,), "lengths"),
                                    self._view(2, out, dtype, shape, "out"),
                                    self._flat(h_last, torch.float32, nh, "h_last"), _raw_stream(self._index))
        if st:
            self._check(st, "wm_seq_gated_scan")
        return out, h_last

    def gated_step(self, gate, x, state, reset=None, out=None, out_state=None, stream=None):
        """One step of N sequences: gate, x [N, H] and the state [N, H] fp32 (or None) give (h, state').
        out_state may be the state itself."""
        if stream is not None:
            return self._elsewhere(stream, self.gated_step, (gate, x, state, reset, out, out_state), {})
        dtype, shape = gate.dtype, gate.shape
        _need(len(shape) == 2, "gate [N, H] is needed")
        N, H = shape
        if out is None:
            out = torch.empty(shape, dtype=dtype, device=self.device)
        if out_state is None:
            out_state = torch.empty(shape, device=self.device)
        st = _lib.wm_seq_gated_scan(self.h, self._dtype(gate), 1, N, H, self._row(0, gate, dtype, shape, "gate"),
                                    self._row(1, x, dtype, shape, "x"), self._flat(state, torch.float32, shape, "state"),
                                    self._flat(reset, torch.uint8, (N,), "reset"), None,
                                    self._row(2, out, dtype, shape, "out"),
                                    self._flat(out_state, torch.float32, shape, "out_state"), _raw_stream(self._index))
        if st:
            self._check(st, "wm_seq_gated_scan")
        return out, out_state

    def gated_scan_backward(self, gate, x, h, dh, dh_last=None, h0=None, reset=None, lengths=None, dgate=None, dx=None,
                            want_dh0: bool = True, stream=None):
        """wm_seq_gated_scan_backward: (dgate, dx, dh0); dgate and dx may be given, strided as in gated_scan."""
        if stream is not None:
            return self._elsewhere(stream, self.gated_scan_backward,
                                   (gate, x, h, dh, dh_last, h0, reset, lengths, dgate, dx, want_dh0), {})
        dtype, shape = gate.dtype, gate.shape
        _need(len(shape) == 3, "gate [T, N, H] is needed")
        T, N, H = shape
        if dgate is None:
            dgate = torch.empty(shape, dtype=dtype, device=self.device)
        if dx is None:
            dx = torch.empty(shape, dtype=dtype, device=self.device)
        dh0 = torch.empty((N, H), device=self.device) if want_dh0 else None
        nh = (N, H)
        st = _lib.wm_seq_gated_scan_backward(
            self.h, self._dtype(gate), T, N, H, self._view(0, gate, dtype, shape, "gate"), self._view(1, x, dtype, shape, "x"),
            self._flat(h0, torch.float32, nh, "h0"), self._flat(reset, torch.uint8, (T, N), "reset"),
            self._flat(lengths, torch.int32, (N,), "lengths"), self._view(2, h, dtype, shape, "h"),
            self._view(3, dh, dtype, shape, "dh"), self._flat(dh_last, torch.float32, nh, "dh_last"),
            self._view(4, dgate, dtype, shape, "dgate"), self._view(5, dx, dtype, shape, "dx"),
            None if dh0 is None else dh0.data_ptr(), _raw_stream(self._index))
        if st:
            self._check(st, "wm_seq_gated_scan_backward")
        return dgate, dx, dh0

    # ------------------------------------------------------------- clipping
    def clip_grads(self, grads, max_norm: float, out=None, stream=None):
        """wm_seq_clip: the global norm [] of the gradients, which are scaled to it in place (or into `out`,
        tensors of the same sizes and types).  max_norm = inf only measures."""
        if stream is not None:
            return self._elsewhere(stream, self.clip_grads, (grads, max_norm, out), {})
        n = len(grads)
        _need(out is None or len(out) == n, "out needs a tensor for each gradient")
        to = grads if out is None else out
        # the gradients as arrays of words, which is how wm_seq_grad is laid out
        words = []
        for g, o in zip(grads, to):
            d = _DTYPE.get(g.dtype)
            if d is None or not g.is_contiguous() or not (
                    o is g or (o.dtype is g.dtype and o.shape == g.shape and o.is_contiguous())):
                raise ValueError("contiguous float32 or bfloat16 gradients, and out of the same shapes and types, are needed")
            words += (g.data_ptr(), o.data_ptr(), g.numel(), d)
        table = array("Q", words)
        norm = torch.empty((), device=self.device)
        st = _lib.wm_seq_clip(self.h, n, table.buffer_info()[0], max_norm, norm.data_ptr(), _raw_stream(self._index))
        if st:
            self._check(st, "wm_seq_clip")
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
