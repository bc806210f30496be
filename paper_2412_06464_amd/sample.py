"""ctypes binding of the choice of the next token (include/gdn_sample.h).

As ``gdn``: argument marshalling only, no fallback, PyTorch for device memory and the current
stream."""
from __future__ import annotations

import ctypes

import torch

from . import gdn
from .gdn import _DTYPES, _check, _on, _stream

EXPORTS = ("gdn_sample",)


class Sampling(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int32), ("vocab", ctypes.c_int32), ("dtype", ctypes.c_int),
                ("logits", ctypes.c_void_p), ("row_stride", ctypes.c_int64),
                ("temperature", ctypes.c_void_p), ("top_k", ctypes.c_void_p),
                ("top_p", ctypes.c_void_p), ("min_p", ctypes.c_void_p), ("u", ctypes.c_void_p)]


_lib = None


def load_library():
    """The library of ``gdn``, with this header's entry point declared."""
    global _lib
    if _lib is None:
        lib = gdn.load_library()
        P = ctypes.c_void_p
        lib.gdn_sample.argtypes = [ctypes.POINTER(Sampling), P, P, P]
        lib.gdn_sample.restype = ctypes.c_int
        _lib = lib
    return _lib


def _per_row(name, x, rows, dtype, device):
    if x is None:
        return None
    if not isinstance(x, torch.Tensor):
        raise TypeError("%s must be a tensor" % name)
    if x.dtype is not dtype or x.device != device or x.shape != (rows,) or not x.is_contiguous():
        raise ValueError("%s must be contiguous %s [%d] on the logits' device"
                         % (name, str(dtype)[6:], rows))
    return x.data_ptr()


def gdn_sample(logits, u, temperature=None, top_k=None, top_p=None, min_p=None, tokens=None,
               logprob=None, output_logprob=True):
    """Draws a token for each row of logits [rows, vocab] (fp32 or bf16, contiguous rows, any row
    stride) with the random numbers u (fp32 [rows], in [0, 1)); returns (tokens, logprob).

    ``temperature`` (<= 0: the likeliest token), ``top_p`` and ``min_p`` fp32 [rows], ``top_k``
    int32 [rows], or None: 1, off, off, off.  ``tokens`` int32 [rows] (-1: nothing to draw),
    ``logprob`` fp32 [rows]: the drawn token's under what was kept; ``output_logprob`` False: none."""
    lib = load_library()
    if not isinstance(logits, torch.Tensor):
        raise TypeError("logits must be a tensor")
    dt = _DTYPES.get(logits.dtype)
    if dt is None:
        raise TypeError("logits must be float32 or bfloat16")
    if logits.dim() != 2 or logits.get_device() < 0:
        raise ValueError("logits must be [rows, vocab] on the GPU")
    rows, vocab = logits.shape
    if vocab > 1 and logits.stride(1) != 1:
        raise ValueError("logits must be contiguous in a row")
    if rows > 0x7fffffff or vocab > 0x7fffffff:
        raise ValueError("the logits are too large")
    dev, f32, i32 = logits.device, torch.float32, torch.int32
    if tokens is None:
        tokens = torch.empty(rows, dtype=i32, device=dev)
    if logprob is None and output_logprob:
        logprob = torch.empty(rows, dtype=f32, device=dev)
    a = Sampling(rows, vocab, dt, logits.data_ptr(), logits.stride(0),
                 _per_row("temperature", temperature, rows, f32, dev),
                 _per_row("top_k", top_k, rows, i32, dev), _per_row("top_p", top_p, rows, f32, dev),
                 _per_row("min_p", min_p, rows, f32, dev), _per_row("u", u, rows, f32, dev))
    t = _per_row("tokens", tokens, rows, i32, dev)
    lp = _per_row("logprob", logprob, rows, f32, dev)
    with _on(dev):
        _check(lib.gdn_sample(ctypes.byref(a), t, lp, _stream(dev)))
    return tokens, logprob
