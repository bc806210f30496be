"""ctypes binding of linear attention with a decay for each head (include/gdn_linear.h): the
other recurrent layer of a hybrid model, in the forms that serve it.

As ``gdn``: argument marshalling only, no fallback, PyTorch for device memory and the current
stream."""
from __future__ import annotations

import ctypes

import torch

from . import gdn
from .gdn import _check, _check_tensors, _nstate, _on, _ptr, _stream, make_problem

EXPORTS = ("gdn_linear_chunk_fwd_workspace_size", "gdn_linear_chunk_fwd",
           "gdn_linear_recurrent_fwd")

_lib = None


def load_library():
    """The library of ``gdn``, with this header's entry points declared."""
    global _lib
    if _lib is None:
        lib = gdn.load_library()
        P, S, I = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int32
        pp = ctypes.POINTER(gdn.Problem)
        lib.gdn_linear_chunk_fwd_workspace_size.argtypes = [pp]
        lib.gdn_linear_chunk_fwd_workspace_size.restype = S
        lib.gdn_linear_chunk_fwd.argtypes = [pp, P, P, P, P, I, P, P, P, P, S, P]
        lib.gdn_linear_chunk_fwd.restype = ctypes.c_int
        lib.gdn_linear_recurrent_fwd.argtypes = [pp, P, P, P, P, I, P, P, P, P]
        lib.gdn_linear_recurrent_fwd.restype = ctypes.c_int
        _lib = lib
    return _lib


def _arguments(q, k, v, log_alpha, h0, cu_seqlens, cu_seqlens_host, output_final_state, o, ht):
    """(problem, what it refers to, per_head, o, ht), checked."""
    p, keep = make_problem(q, v, cu_seqlens, cu_seqlens_host)
    H, n = q.shape[2], _nstate(q, cu_seqlens)
    if o is None:
        o = torch.empty_like(v, memory_format=torch.contiguous_format)
    if ht is None and output_final_state:
        ht = torch.empty((n, H, q.shape[3], v.shape[3]), dtype=torch.float32, device=q.device)
    per_head = isinstance(log_alpha, torch.Tensor) and log_alpha.dim() == 1
    if per_head:
        if (log_alpha.dtype != torch.float32 or log_alpha.device != q.device
                or log_alpha.shape[0] != H or not log_alpha.is_contiguous()):
            raise ValueError("log_alpha must be contiguous float32 [B,T,H] or [H] on q's device")
    _check_tensors(q, rows=(("k", k), ("v", v), ("o", o)),
                   gates=() if per_head else (("log_alpha", log_alpha),),
                   states=(("h0", h0, v.shape[3]), ("ht", ht, v.shape[3])), nstate=n)
    if q.get_device() < 0:
        raise ValueError("q must be on the GPU")
    if k.shape != q.shape or o.shape != v.shape:
        raise ValueError("k must match q, and o must match v")
    return p, keep, int(per_head), o, ht


def gdn_linear_chunk_fwd_workspace_size(q, v, cu_seqlens=None, cu_seqlens_host=None) -> int:
    """Workspace bytes of gdn_linear_chunk_fwd for these tensors (0: none is needed)."""
    p, keep = make_problem(q, v, cu_seqlens, cu_seqlens_host)
    return int(load_library().gdn_linear_chunk_fwd_workspace_size(ctypes.byref(p)))


def gdn_linear_chunk_fwd(q, k, v, log_alpha, h0=None, cu_seqlens=None, cu_seqlens_host=None,
                         output_final_state=True, o=None, ht=None, workspace=None):
    """S_t = exp(log_alpha_t) S_{t-1} + k_t v_t^T, o_t = S_t^T q_t over all tokens, in chunks.

    q, k [B,T,H,dk] and v [B,T,H,dv] (fp32 or bf16, one dtype; dk of 64, 128, 256, dv of 64, 128,
    256, 512); log_alpha fp32 [B,T,H], or [H] (the same for every token of a head), or None (no
    decay); h0 [Nseq,H,dk,dv] fp32 or None.  Packed input passes cu_seqlens (int32 [N+1]) with
    B == 1.  Returns (o, ht); ``ht=h0`` updates the states in place."""
    lib = load_library()
    p, keep, per_head, o, ht = _arguments(q, k, v, log_alpha, h0, cu_seqlens, cu_seqlens_host,
                                          output_final_state, o, ht)
    need = lib.gdn_linear_chunk_fwd_workspace_size(ctypes.byref(p))
    size = 0
    if need:
        if workspace is None or workspace.numel() < need:
            workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
        elif (workspace.dtype != torch.uint8 or workspace.device != q.device
              or not workspace.is_contiguous()):
            raise ValueError("workspace must be a contiguous uint8 tensor on q's device")
        size = workspace.numel()
    with _on(q.device):
        _check(lib.gdn_linear_chunk_fwd(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(v),
                                        _ptr(log_alpha), per_head, _ptr(h0), _ptr(o), _ptr(ht),
                                        _ptr(workspace) if size else None, size,
                                        _stream(q.device)))
    del keep
    return o, ht


def gdn_linear_recurrent_fwd(q, k, v, log_alpha, h0=None, cu_seqlens=None, cu_seqlens_host=None,
                             output_final_state=True, o=None, ht=None):
    """gdn_linear_chunk_fwd token by token, for few tokens a sequence (T = 1: a decode step)."""
    lib = load_library()
    p, keep, per_head, o, ht = _arguments(q, k, v, log_alpha, h0, cu_seqlens, cu_seqlens_host,
                                          output_final_state, o, ht)
    with _on(q.device):
        _check(lib.gdn_linear_recurrent_fwd(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(v),
                                            _ptr(log_alpha), per_head, _ptr(h0), _ptr(o), _ptr(ht),
                                            _stream(q.device)))
    del keep
    return o, ht
