"""Thin ctypes binding of libgdn's attention layer (include/gdn_paged.h).

Rotary positions, a cache of keys and values in pages, attention of new tokens
over it and the management of its pages: what a model needs that alternates the
gated delta rule with attention.  As ``gdn``: argument marshalling only, every
step runs in the HIP kernels of ``libgdn.so`` on the current stream, and there
is no fallback.

Row tensors are [B, T, heads, d] (packed input: B == 1 with ``cu_seqlens``),
float32 or bfloat16, the last dim contiguous; the strides of heads and tokens
are free, so q, k and v may be slices of one projection.  A cache's k and v are
[num_pages, Hk, page_size, d] each, last dim contiguous, alike in strides; one
allocation [layers, 2, num_pages, Hk, page_size, d] serves all layers and is
the ``pool`` of the page calls after ``flatten(0, 1)``.
"""
from __future__ import annotations

import ctypes
import importlib.util
import os
import struct
from typing import NamedTuple

import torch

from .gdn import _check, _cu_pair, _ptr, _stream, load_library as _load

EXPORTS = ("gdn_rotary_turns", "gdn_rotary_fwd", "gdn_rotary_bwd", "gdn_cache_append",
           "gdn_cache_attn", "gdn_cache_attn_workspace_size", "gdn_pages_workspace_size",
           "gdn_pages_extend", "gdn_pages_select", "gdn_pages_compact", "gdn_pages_copy")

LAYOUTS = {"halves": 0, "interleaved": 1}
SCALINGS = {"none": 0, "linear": 1, "base": 2, "parts": 3}


class Tokens(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("T", ctypes.c_int32), ("Hq", ctypes.c_int32),
                ("Hk", ctypes.c_int32), ("d", ctypes.c_int32), ("num_seqs", ctypes.c_int32),
                ("cu_seqlens", ctypes.c_void_p), ("cu_seqlens_host", ctypes.c_void_p),
                ("dtype", ctypes.c_int)]


class Rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("token_stride", ctypes.c_int64),
                ("head_stride", ctypes.c_int64)]


class Cache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("page_stride", ctypes.c_int64),
                ("head_stride", ctypes.c_int64), ("token_stride", ctypes.c_int64),
                ("num_pages", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("max_blocks", ctypes.c_int32), ("table", ctypes.c_void_p),
                ("kv_lens", ctypes.c_void_p), ("skip", ctypes.c_void_p)]


class RotaryStruct(ctypes.Structure):
    _fields_ = [("rot", ctypes.c_int32), ("layout", ctypes.c_int32), ("scale", ctypes.c_float),
                ("turns", ctypes.c_void_p)]


class Attn(ctypes.Structure):
    _fields_ = [("scale", ctypes.c_float), ("causal", ctypes.c_int32), ("window", ctypes.c_int32),
                ("max_kv", ctypes.c_int32)]


class Book(ctypes.Structure):
    _fields_ = [("S", ctypes.c_int32), ("max_blocks", ctypes.c_int32),
                ("num_pages", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("table", ctypes.c_void_p), ("lens", ctypes.c_void_p), ("refs", ctypes.c_void_p),
                ("table_out", ctypes.c_void_p), ("lens_out", ctypes.c_void_p),
                ("refs_out", ctypes.c_void_p)]


class Pool(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("parts", ctypes.c_int32),
                ("num_pages", ctypes.c_int32), ("part_stride", ctypes.c_int64),
                ("page_stride", ctypes.c_int64), ("page_bytes", ctypes.c_int64)]


class Rotary(NamedTuple):
    """A rotation: its frequencies (float64 [rot / 2] turns a position, on the
    device), pair layout and the factor of cos and sin."""
    turns: torch.Tensor
    layout: str
    scale: float


_lib = None


def load_library():
    """libgdn.so with this module's entry points declared; raises if absent."""
    global _lib
    if _lib is None:
        lib = _load()
        P, I, D, S = ctypes.c_void_p, ctypes.c_int32, ctypes.c_double, ctypes.c_size_t
        # structures go in as their bytes (c_void_p), see below
        for name, args in (
                ("gdn_rotary_turns", [I, D, I, D, D, D, D, P, P]),
                ("gdn_rotary_fwd", [P] * 8),
                ("gdn_rotary_bwd", [P] * 8),
                ("gdn_cache_append", [P] * 8),
                ("gdn_cache_attn", [P] * 7 + [S, P]),
                ("gdn_cache_attn_workspace_size", [P] * 3),
                ("gdn_pages_workspace_size", [P]),
                ("gdn_pages_extend", [P] * 4 + [S, P]),
                ("gdn_pages_select", [P] * 5 + [S, P]),
                ("gdn_pages_compact", [P] * 4 + [S, P]),
                ("gdn_pages_copy", [P, P, P, I, P])):
            f = getattr(lib, name)
            f.argtypes = args
            f.restype = S if name.endswith("_size") else ctypes.c_int
        _lib = lib
    return _lib


# A call of a few microseconds on the GPU must not spend longer here: the
# tensors are checked and the structures of the C ABI filled in by a native
# helper (csrc/paged_binding.cpp); structures go in as their bytes.  Host time
# of a call, with all of it in Python and so: storing a token for each of 256
# sequences 19.4 and 6.9 us, attention of one token for each of 4 15.1 and 8.7.
_ATTN = struct.Struct("@fiii")
_BOOK = struct.Struct("@iiiiPPPPPP")
_Tensor = torch.Tensor


def _native():
    """The native helper; raises if it is not built."""
    path = os.path.join(os.path.dirname(os.path.abspath(__file__)), "_paged_binding.so")
    if not os.path.exists(path):
        raise RuntimeError("_paged_binding.so is not built (%s); run "
                           "`python -m paper_2412_06464_amd.build`" % path)
    spec = importlib.util.spec_from_file_location("_paged_binding", path)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


class _Helper:
    """The helper's functions, loaded at their first use."""

    def __getattr__(self, name):
        mod = _native()
        for f in ("first", "rows", "like", "ints", "tokens", "cache", "rotary", "pool", "book"):
            setattr(self, f, getattr(mod, f))
        return getattr(self, name)


_n = _Helper()


def _tokens(first, Hq, Hk, cu_seqlens, cu_seqlens_host, device, keep):
    """gdn_tokens; boundaries that are not as the library takes them are converted."""
    if cu_seqlens is None and cu_seqlens_host is not None:
        raise ValueError("cu_seqlens_host without cu_seqlens")
    t = _n.tokens(first, Hq, Hk, cu_seqlens, cu_seqlens_host)
    if t is None:
        pair = _cu_pair(cu_seqlens, cu_seqlens_host, device, keep)
        keep.append(pair)
        t = _n.tokens(first, Hq, Hk, *pair)
    return t


# ------------------------------------------------------------------ rotary positions


def gdn_rotary_turns(rot, base=10000.0, scaling="none", factor=1.0, original=0, slow=1.0,
                     fast=32.0):
    """Turns a position of each pair (float64 [rot / 2], CPU) and the factor of cos and sin.

    ``scaling`` for a context ``factor`` times the ``original`` one: "linear" (positions
    interpolated), "base" (a larger base), "parts" (pairs that turn less than ``slow`` times over
    the original context interpolated, those over ``fast`` kept, in between blended)."""
    if scaling not in SCALINGS:
        raise ValueError("scaling must be one of %s" % sorted(SCALINGS))
    turns = torch.zeros(max(int(rot) // 2, 1), dtype=torch.float64)
    scale = ctypes.c_float()
    _check(load_library().gdn_rotary_turns(int(rot), base, SCALINGS[scaling], factor, original,
                                           slow, fast, turns.data_ptr(), ctypes.addressof(scale)))
    return turns, scale.value


def gdn_rotary(rot, base=10000.0, layout="halves", scaling="none", factor=1.0, original=0,
               slow=1.0, fast=32.0, device="cuda"):
    """A Rotary: made once by a model, passed to the calls.  ``layout`` "halves": channel i pairs
    with i + rot / 2; "interleaved": 2 i with 2 i + 1."""
    if layout not in LAYOUTS:
        raise ValueError("layout must be one of %s" % sorted(LAYOUTS))
    turns, scale = gdn_rotary_turns(rot, base, scaling, factor, original, slow, fast)
    return Rotary(turns.to(device), layout, scale)


def _rotary(r, first):
    if not isinstance(r, Rotary):
        raise TypeError("rotary must be a Rotary (see gdn_rotary)")
    if r.layout not in LAYOUTS:
        raise ValueError("layout must be one of %s" % sorted(LAYOUTS))
    return _n.rotary(r.turns, LAYOUTS[r.layout], r.scale, first)


def _rotate(f, q, k, rotary, positions, cu_seqlens, cu_seqlens_host, q_out, k_out):
    keep = []
    rq = _n.first("q", q)
    B, T, Hq, _ = q.shape
    rk, ko, Hk = None, None, 1
    if q_out is None:
        q_out, ro = _n.like(q)
    else:
        ro = _n.rows("q_out", q_out, "q", q, Hq)
    if k is not None:
        rk, Hk = _n.rows("k", k, "q", q, -1), k.shape[2]
        if k_out is None:
            k_out, ko = _n.like(k)
        else:
            ko = _n.rows("k_out", k_out, "q", q, Hk)
    dev = q.device
    t = _tokens(q, Hq, Hk, cu_seqlens, cu_seqlens_host, dev, keep)
    p = None if positions is None else _n.ints("positions", positions, q, B, T)
    _check(f(t, _rotary(rotary, q), rq, rk, p, ro, ko, _stream(dev)))
    return q_out, k_out


def gdn_rotary_fwd(q, k, rotary, positions=None, cu_seqlens=None, cu_seqlens_host=None, q_out=None,
                   k_out=None):
    """Rotary positions of q [B, T, Hq, d] and k [B, T, Hk, d] (or None): (q_out, k_out).

    ``positions`` int32 [B, T]; None: a token's place in its row, or in its packed sequence.
    ``q_out=q`` and ``k_out=k`` rotate in place."""
    return _rotate(load_library().gdn_rotary_fwd, q, k, rotary, positions, cu_seqlens,
                   cu_seqlens_host, q_out, k_out)


def gdn_rotary_bwd(dq_out, dk_out, rotary, positions=None, cu_seqlens=None, cu_seqlens_host=None,
                   dq=None, dk=None):
    """Gradients of gdn_rotary_fwd's inputs from those of its outputs: (dq, dk)."""
    return _rotate(load_library().gdn_rotary_bwd, dq_out, dk_out, rotary, positions, cu_seqlens,
                   cu_seqlens_host, dq, dk)


# ------------------------------------------------------------------ the cache


def gdn_cache_append(q, k, v, k_pages, v_pages, table, kv_lens, rotary=None, cu_seqlens=None,
                     cu_seqlens_host=None, q_out=None, skip=None):
    """Stores the new tokens' k (rotated) and v in their sequences' pages; returns q, rotated.

    q [B, T, Hq, d] or None, k and v [B, T, Hk, d]; table int32 [sequences, blocks], kv_lens int32
    [sequences]: the tokens of each sequence with the new ones, which are its last.  ``rotary``
    None: nothing is rotated.  Tokens whose page is a hole are not stored.  ``skip`` int32
    [sequences]: the ``short`` of the gdn_pages_extend before; nothing is stored for a sequence with
    a non-zero entry.  Without it, a sequence that was refused room must not be in the call: its
    new tokens would go over its last ones, in pages that others may share."""
    lib = load_library()
    keep = []
    rk = _n.first("k", k)
    B, _, Hk, _ = k.shape
    dev, Hq, rq, ro = k.device, Hk, None, None
    if q is not None:
        rq, Hq = _n.rows("q", q, "k", k, -1), q.shape[2]
        if q_out is None:
            q_out, ro = _n.like(q)
        else:
            ro = _n.rows("q_out", q_out, "k", k, Hq)
    n = B if cu_seqlens is None else cu_seqlens.shape[0] - 1
    c = _n.cache("k", k, k_pages, v_pages, table, kv_lens, n, skip)
    if k_pages.shape[1] != Hk:
        raise ValueError("k_pages must have k's heads")
    t = _tokens(k, Hq, Hk, cu_seqlens, cu_seqlens_host, dev, keep)
    _check(lib.gdn_cache_append(t, None if rotary is None else _rotary(rotary, k), rq, rk,
                                _n.rows("v", v, "k", k, Hk), c, ro, _stream(dev)))
    return q_out


def _attn(scale, d, causal, window, max_kv):
    return _ATTN.pack(d ** -0.5 if scale is None else scale, 1 if causal else 0, window or 0,
                      max_kv or 0)


def gdn_cache_attn_workspace_size(q, k_pages, table, scale=None, causal=True, window=0, max_kv=0,
                                  cu_seqlens=None, cu_seqlens_host=None) -> int:
    """Workspace bytes of gdn_cache_attn with these arguments (0: none is needed)."""
    keep = []
    _n.first("q", q)
    B, _, Hq, d = q.shape
    n = B if cu_seqlens is None else cu_seqlens.shape[0] - 1
    c = _n.cache("q", q, k_pages, k_pages, table, None, n, None)
    t = _tokens(q, Hq, k_pages.shape[1], cu_seqlens, cu_seqlens_host, q.device, keep)
    return int(load_library().gdn_cache_attn_workspace_size(t, c, _attn(scale, d, causal, window,
                                                                        max_kv)))


def gdn_cache_attn(q, k_pages, v_pages, table, kv_lens, scale=None, causal=True, window=0,
                   max_kv=0, cu_seqlens=None, cu_seqlens_host=None, o=None, lse=None,
                   workspace=None, skip=None):
    """Attention of the new tokens q [B, T, Hq, d] over their sequences' cached keys; returns o.

    The new tokens are the last of the kv_lens[n] that sequence n holds (gdn_cache_append has
    stored them).  ``scale`` None: 1 / sqrt(d); ``window`` > 0: a token sees itself and the window - 1
    before it; ``max_kv``: how long a sequence may be at most (0: what the table has room for),
    which the launches are sized by.  ``lse`` float32 [B, T, Hq] receives the log of each softmax's
    sum.  A token that sees no key gets 0 (lse -inf), and so do those of a sequence with a non-zero
    entry in ``skip`` (as in gdn_cache_append)."""
    lib = load_library()
    keep = []
    rq = _n.first("q", q)
    B, T, Hq, d = q.shape
    dev = q.device
    n = B if cu_seqlens is None else cu_seqlens.shape[0] - 1
    c = _n.cache("q", q, k_pages, v_pages, table, kv_lens, n, skip)
    t = _tokens(q, Hq, k_pages.shape[1], cu_seqlens, cu_seqlens_host, dev, keep)
    if o is None:
        o, ro = _n.like(q)
    else:
        ro = _n.rows("o", o, "q", q, Hq)
    if lse is not None and (lse.dtype is not torch.float32 or lse.device != dev
                            or not lse.is_contiguous() or lse.shape != q.shape[:3]):
        raise ValueError("lse must be contiguous float32 [B, T, Hq] on q's device")
    a = _attn(scale, d, causal, window, max_kv)
    need = lib.gdn_cache_attn_workspace_size(t, c, a)
    ws, size = None, 0
    if need:
        if workspace is None or workspace.numel() < need:
            workspace = torch.empty(need, dtype=torch.uint8, device=dev)
        elif (workspace.device != dev or workspace.dtype is not torch.uint8
              or not workspace.is_contiguous()):
            raise ValueError("workspace must be a contiguous uint8 tensor on q's device")
        ws, size = workspace.data_ptr(), workspace.numel()
    _check(lib.gdn_cache_attn(t, a, rq, c, ro, _ptr(lse), ws, size, _stream(dev)))
    return o


# ------------------------------------------------------------------ pages


def _pool(pool, table):
    return None if pool is None else _n.pool(pool, table)


def _work(lib, b, workspace, device):
    """(the workspace, its pointer, its size)."""
    need = lib.gdn_pages_workspace_size(b)
    if workspace is None or workspace.numel() < need:
        workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=device)
    elif workspace.device != device or workspace.dtype is not torch.uint8 \
            or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous uint8 tensor on %s" % device)
    return workspace, workspace.data_ptr(), workspace.numel()


def gdn_pages_workspace_size(table, refs) -> int:
    """Workspace bytes of the page calls for a table and reference counts of these shapes."""
    b = _BOOK.pack(table.shape[0], table.shape[1], refs.numel(), 1, 0, 0, 0, 0, 0, 0)
    return int(load_library().gdn_pages_workspace_size(b))


def gdn_pages_extend(table, lens, refs, add, page_size, out=None, workspace=None):
    """Room for add[s] more tokens in each sequence: dict table, lens, refs, short.

    table int32 [S, blocks], lens and add int32 [S], refs int32 [pages] (holders of each page; 0:
    free).  short[s] > 0: there was no room for the pages it needs, and sequence s is as it was: pass
    ``short`` on as ``skip`` of the calls on the cache, or leave such sequences out of them.
    ``out``: dict of tensors to write; the inputs themselves update in place."""
    lib = load_library()
    b, got, short = _n.book(table, lens, refs, page_size, out, True, "short")
    device = table.device
    ws, p, n = _work(lib, b, workspace, device)
    _check(lib.gdn_pages_extend(b, _n.ints("add", add, table, lens.shape[0]), short, p, n,
                                _stream(device)))
    return got


def gdn_pages_select(table, lens, refs, parents, page_size, pool=None, out=None, workspace=None):
    """Row i goes on from old row parents[i] (out of range: it ends): dict table, lens, refs, short.

    Frees, forks and reorders sequences in one call: full pages are shared, a partly filled last
    page is copied for every row but the lowest of its parent, in ``pool`` [parts, pages, ...].
    short[i] == 1: no page was left and row i is empty."""
    lib = load_library()
    b, got, short = _n.book(table, lens, refs, page_size, out, True, "short")
    device = table.device
    ws, p, n = _work(lib, b, workspace, device)
    _check(lib.gdn_pages_select(b, _n.ints("parents", parents, table, lens.shape[0]),
                                _pool(pool, table), short, p, n, _stream(device)))
    return got


def gdn_pages_compact(table, lens, refs, page_size, pool=None, out=None, workspace=None):
    """Moves the pages in use into the lowest indexes: dict table, refs, map (new index of each
    page, -1 if it was free).  The data moves in ``pool`` [parts, pages, ...]."""
    lib = load_library()
    b, got, to = _n.book(table, lens, refs, page_size, out, False, "map")
    device = table.device
    ws, p, n = _work(lib, b, workspace, device)
    _check(lib.gdn_pages_compact(b, _pool(pool, table), to, p, n, _stream(device)))
    return got


def gdn_pages_copy(pool, src, dst):
    """Copies pages src[i] to dst[i] (int32) in every part of ``pool`` [parts, pages, ...], a cache
    or a pool of recurrent states; pairs out of range are skipped."""
    if not isinstance(pool, _Tensor):
        raise TypeError("pool must be a tensor")
    p = _n.pool(pool, pool)
    if not isinstance(src, _Tensor) or src.dim() != 1:
        raise ValueError("src must be int32 [pairs]")
    n = src.shape[0]
    _check(load_library().gdn_pages_copy(p, _n.ints("src", src, pool),
                                         _n.ints("dst", dst, pool, n), n, _stream(pool.device)))
