"""Thin Python binding of the sequence operators in include/wm_seq.h (argument marshalling only,
in the compiled module ``_seq_ext``).

``SequenceOps`` owns one handle on one CUDA device.  Its methods take CUDA tensors, allocate
their outputs unless given, and run on the current stream (or ``stream=``) without
synchronising.  There is no CPU fallback.

All calls of one object share its workspace: calls on several streams have to be ordered among
them (``wait_stream``, events), or go through an object for each stream.  ``stream=`` makes that
stream wait for nothing: what the inputs' own stream still has to do comes first by the caller's
order.  Nothing is recorded for autograd: a tensor that requires a gradient is taken for its values,
and the ``_backward`` methods are called by hand.

    ops = SequenceOps()
    e = ops.embed(table, actions, scale=32.0)
    y, mean, rstd = ops.layer_norm(e, weight, bias, want_stats=True)
    h, state = ops.gated_scan(gate, x, h0=state, reset=starts, lengths=lengths)
    dgate, dx, dh0 = ops.gated_scan_backward(gate, x, h, dh, h0=state)
    q, k = ops.head_norm(q, k, q_weight, k_weight, positions=positions, freqs=freqs)
    o, state = ops.decay_attention(q, k, v, log_decay, scale=0.125, s0=state, reset=starts)
    dq, dk, dv, ds0 = ops.decay_attention_backward(q, k, v, log_decay, do, scale=0.125, s0=state)
    norm = ops.clip_grads(grads, max_norm=1.0)
    ops.sync()                               # raises WMError on a device-side error
"""
from __future__ import annotations

import ctypes as C
import os

import torch

from . import wm as _wm
from .wm import WMError

if not os.path.exists(os.path.join(os.path.dirname(os.path.abspath(__file__)), "_seq_ext.so")):
    raise ImportError("_seq_ext.so is missing: build it with `python -c 'import __graft_entry__ as g; g.build()'` (no CPU fallback)")
from . import _seq_ext as _ext  # noqa: E402

_ext.set_error(WMError)
_lib = _wm._lib


def _declare():
    """The C names, for ctypes."""
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
        "wm_seq_head_norm": [P, I, L, I, I, I, I, I, V, P, I, V, P, F, P, P, V, V, P],
        "wm_seq_head_norm_backward": [P, I, L, I, I, I, I, I, V, P, V, I, V, P, V, F, P, P, V, V, P, P, P],
        "wm_seq_decay_attention": [P, I, L, I, I, I, I, V, V, V, P, F, P, P, P, V, P, P],
        "wm_seq_decay_attention_backward": [P, I, L, I, I, I, I, V, V, V, P, F, P, P, P, V, P, V, V, V, P, P],
        "wm_seq_clip": [P, I, P, F, P, P],
    }
    for name, args in sig.items():
        f = getattr(_lib, name)
        f.argtypes, f.restype = args, C.c_int
    _lib.wm_seq_last_error.argtypes, _lib.wm_seq_last_error.restype = [P], C.c_char_p
    _lib.wm_seq_last_launches.argtypes, _lib.wm_seq_last_launches.restype = [P], C.c_int
    _lib.wm_seq_destroy.argtypes, _lib.wm_seq_destroy.restype = [P], None


_declare()


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

    def close(self):
        if getattr(self, "h", None):
            _lib.wm_seq_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, st: int, what: str):
        if st:
            raise WMError(st, _lib.wm_seq_last_error(self.h).decode() or what)

    def _elsewhere(self, stream, method, *args):
        """The call on another stream: its outputs are allocated there, and its inputs' memory is
        not used again before it is done."""
        s = stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(int(stream), device=self.device)
        if s.device != self.device:  # (it would be current on its own device, and the call go to this one's current stream)
            raise ValueError(f"a stream of {self.device} is needed, got one of {s.device}")
        with torch.cuda.stream(s):
            out = method(*args)

        def mark(v):
            if isinstance(v, torch.Tensor) and v.is_cuda:
                v.record_stream(s)
            elif isinstance(v, (list, tuple)):
                for x in v:
                    mark(x)

        mark(args)
        return out

    # ------------------------------------------------------------- embedding
    def embed(self, table, tokens, scale: float = 1.0, out=None, stream=None):
        """wm_seq_embed: scale * table[tokens] (0 where a token is negative); tokens int32 of any shape."""
        if stream is not None:
            return self._elsewhere(stream, self.embed, table, tokens, scale, out)
        return _ext.embed(self.h, self._index, table, tokens, scale, out)

    def embed_backward(self, tokens, dout, vocab: int, scale: float = 1.0, out=None, stream=None):
        """wm_seq_embed_backward: the gradient [vocab, D] of embed's table."""
        if stream is not None:
            return self._elsewhere(stream, self.embed_backward, tokens, dout, vocab, scale, out)
        return _ext.embed_backward(self.h, self._index, tokens, dout, vocab, scale, out)

    # ------------------------------------------------------------- layer norm
    def layer_norm(self, x, weight=None, bias=None, eps: float = 1e-5, want_stats: bool = False, out=None, stream=None):
        """wm_seq_layer_norm over the last axis; (y, mean, rstd) with want_stats.  out may be x."""
        if stream is not None:
            return self._elsewhere(stream, self.layer_norm, x, weight, bias, eps, want_stats, out)
        return _ext.layer_norm(self.h, self._index, x, weight, bias, eps, want_stats, out)

    def layer_norm_backward(self, x, weight, mean, rstd, dy, dx=None, want_params: bool = True, stream=None):
        """wm_seq_layer_norm_backward: (dx, dweight, dbias), the last two None without want_params.  dx may be dy."""
        if stream is not None:
            return self._elsewhere(stream, self.layer_norm_backward, x, weight, mean, rstd, dy, dx, want_params)
        return _ext.layer_norm_backward(self.h, self._index, x, weight, mean, rstd, dy, dx, want_params)

    # ------------------------------------------------------------- gated scan
    def gated_scan(self, gate, x, h0=None, reset=None, lengths=None, out=None, want_last: bool = True, h_last=None,
                   stream=None):
        """wm_seq_gated_scan over [T, N, H]; (h, h_last).  gate, x and out may be strided over T and N
        (columns of a wider array, a transposed batch-major array); h_last may be h0."""
        if stream is not None:
            return self._elsewhere(stream, self.gated_scan, gate, x, h0, reset, lengths, out, want_last, h_last)
        return _ext.gated_scan(self.h, self._index, gate, x, h0, reset, lengths, out, want_last, h_last)

    def gated_step(self, gate, x, state, reset=None, out=None, out_state=None, stream=None):
        """One step of N sequences: gate, x [N, H] and the state [N, H] fp32 (or None) give (h, state').
        out_state may be the state itself."""
        if stream is not None:
            return self._elsewhere(stream, self.gated_step, gate, x, state, reset, out, out_state)
        return _ext.gated_step(self.h, self._index, gate, x, state, reset, None, out, True, out_state)

    def gated_scan_backward(self, gate, x, h, dh, dh_last=None, h0=None, reset=None, lengths=None, dgate=None, dx=None,
                            want_dh0: bool = True, stream=None, dh0=None):
        """wm_seq_gated_scan_backward: (dgate, dx, dh0); dgate and dx may be given, strided as in gated_scan, and dh0,
        which may be dh_last."""
        if stream is not None:
            return self._elsewhere(stream, self.gated_scan_backward, gate, x, h, dh, dh_last, h0, reset, lengths, dgate, dx,
                                   want_dh0, None, dh0)
        return _ext.gated_scan_backward(self.h, self._index, gate, x, h, dh, dh_last, h0, reset, lengths, dgate, dx, want_dh0, dh0)

    # ------------------------------------------------------------- head norm
    def head_norm(self, q, k=None, q_weight=None, k_weight=None, positions=None, freqs=None, eps: float = 1e-6,
                  interleaved: bool = False, q_out=None, k_out=None, stream=None):
        """wm_seq_head_norm of queries [T, N, heads, D] (or [N, heads, D], one step) and keys, which may have another number
        of heads: (q', k'), or q' without keys.  Without positions and freqs nothing is rotated; len(freqs) is half of the
        rotated values.  q_out may be q, and k_out k."""
        if stream is not None:
            return self._elsewhere(stream, self.head_norm, q, k, q_weight, k_weight, positions, freqs, eps, interleaved, q_out, k_out)
        return _ext.head_norm(self.h, self._index, q, k, q_weight, k_weight, positions, freqs, eps, interleaved, q_out, k_out)

    def head_norm_backward(self, q, dq_out, k=None, dk_out=None, q_weight=None, k_weight=None, positions=None, freqs=None,
                           eps: float = 1e-6, interleaved: bool = False, dq=None, dk=None, want_params: bool = True, stream=None):
        """wm_seq_head_norm_backward: (dq, dk, dq_weight, dk_weight), those of the keys None without keys, the weights' None
        without want_params.  dq may be dq_out, and dk dk_out."""
        if stream is not None:
            return self._elsewhere(stream, self.head_norm_backward, q, dq_out, k, dk_out, q_weight, k_weight, positions, freqs, eps,
                                   interleaved, dq, dk, want_params)
        return _ext.head_norm_backward(self.h, self._index, q, k, q_weight, k_weight, positions, freqs, eps, interleaved, dq, dk,
                                       dq_out, dk_out, want_params)

    # ------------------------------------------------------------- decayed attention
    def decay_attention(self, q, k, v, log_decay, scale: float = 1.0, s0=None, reset=None, lengths=None, out=None,
                        want_last: bool = True, s_last=None, stream=None):
        """wm_seq_decay_attention over q, k [T, N, heads, Dk] and v [T, N, heads, Dv]: (o, s_last).  The arrays may be strided over
        T, N and heads; s_last may be s0."""
        if stream is not None:
            return self._elsewhere(stream, self.decay_attention, q, k, v, log_decay, scale, s0, reset, lengths, out, want_last, s_last)
        return _ext.decay_attention(self.h, self._index, q, k, v, log_decay, scale, s0, reset, lengths, out, want_last, s_last)

    def decay_step(self, q, k, v, log_decay, state, scale: float = 1.0, reset=None, out=None, out_state=None, stream=None):
        """One token of N sequences: q, k [N, heads, Dk], v [N, heads, Dv] and the state [N, heads, Dk, Dv] fp32 (or None) give
        (o, state').  out_state may be the state itself."""
        if stream is not None:
            return self._elsewhere(stream, self.decay_step, q, k, v, log_decay, state, scale, reset, out, out_state)
        return _ext.decay_step(self.h, self._index, q, k, v, log_decay, scale, state, reset, None, out, True, out_state)

    def decay_attention_backward(self, q, k, v, log_decay, dout, scale: float = 1.0, ds_last=None, s0=None, reset=None, lengths=None,
                                 dq=None, dk=None, dv=None, want_ds0: bool = True, ds0=None, stream=None):
        """wm_seq_decay_attention_backward: (dq, dk, dv, ds0); each may be given, ds0 may be ds_last."""
        if stream is not None:
            return self._elsewhere(stream, self.decay_attention_backward, q, k, v, log_decay, dout, scale, ds_last, s0, reset, lengths,
                                   dq, dk, dv, want_ds0, ds0)
        return _ext.decay_attention_backward(self.h, self._index, q, k, v, log_decay, scale, s0, reset, lengths, dout, ds_last, dq, dk,
                                             dv, want_ds0, ds0)

    # ------------------------------------------------------------- clipping
    def clip_grads(self, grads, max_norm: float, out=None, stream=None):
        """wm_seq_clip: the global norm [] of the gradients, which are scaled to it in place (or into `out`,
        tensors of the same sizes and types).  max_norm = inf only measures."""
        if stream is not None:  # (lists: what a view or a generator gives is to be kept until the call is done)
            return self._elsewhere(stream, self.clip_grads, list(grads), max_norm, None if out is None else list(out))
        return _ext.clip_grads(self.h, self._index, grads, max_norm, out)

    # ------------------------------------------------------------- status
    def sync(self):
        """Waits for the device; raises WMError on a device-side error since the last call."""
        self._check(_lib.wm_seq_sync(self.h), "wm_seq_sync")

    def inject_wait_timeout(self, polls: int):
        """wm_seq_inject_wait_timeout: a wait of the next long scan, small clipping or decayed attention on the
        tensor cores gives up (tests of the timeout path)."""
        self._check(_lib.wm_seq_inject_wait_timeout(self.h, int(polls)), "wm_seq_inject_wait_timeout")

    @property
    def last_launches(self) -> int:
        return int(_lib.wm_seq_last_launches(self.h))
