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
from typing import NamedTuple

import torch

from .gdn import GDN_BF16, GDN_F32, _check, _cu_pair, _ptr, _stream, load_library as _load

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
                ("kv_lens", ctypes.c_void_p)]


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
        tok, rot, rows, cache, attn, book, pool = (ctypes.POINTER(x) for x in (
            Tokens, RotaryStruct, Rows, Cache, Attn, Book, Pool))
        for name, args in (
                ("gdn_rotary_turns", [I, D, I, D, D, D, D, P, P]),
                ("gdn_rotary_fwd", [tok, rot, rows, rows, P, rows, rows, P]),
                ("gdn_rotary_bwd", [tok, rot, rows, rows, P, rows, rows, P]),
                ("gdn_cache_append", [tok, rot, rows, rows, rows, cache, rows, P]),
                ("gdn_cache_attn", [tok, attn, rows, cache, rows, P, P, S, P]),
                ("gdn_cache_attn_workspace_size", [tok, cache, attn]),
                ("gdn_pages_workspace_size", [book]),
                ("gdn_pages_extend", [book, P, P, P, S, P]),
                ("gdn_pages_select", [book, P, pool, P, P, S, P]),
                ("gdn_pages_compact", [book, pool, P, P, S, P]),
                ("gdn_pages_copy", [pool, P, P, I, P])):
            f = getattr(lib, name)
            f.argtypes = args
            f.restype = S if name.endswith("_size") else ctypes.c_int
        _lib = lib
    return _lib


_DTYPES = {torch.float32: GDN_F32, torch.bfloat16: GDN_BF16}


def _rows(name, x, like=None):
    """gdn_rows of a [B, T, heads, d] tensor; ``like``: (name, tensor) whose B,
    T, d, dtype and device it has to share."""
    if not isinstance(x, torch.Tensor):
        raise TypeError("%s must be a tensor" % name)
    if x.dim() != 4:
        raise ValueError("%s must be [B, T, heads, d]" % name)
    B, T, H, d = x.shape
    sb, st, sh, sd = x.stride()
    if x.dtype not in _DTYPES:
        raise TypeError("%s must be float32 or bfloat16" % name)
    if x.get_device() < 0:
        raise ValueError("%s must be on the GPU" % name)
    if like is not None:
        other, y = like
        if x.dtype is not y.dtype or x.get_device() != y.get_device():
            raise ValueError("%s must have %s's dtype and device" % (name, other))
        if y.shape[0] != B or y.shape[1] != T or y.shape[3] != d:
            raise ValueError("%s must have %s's B, T and d" % (name, other))
    if sd != 1 and d != 1:
        raise ValueError("%s must be contiguous in its last dim" % name)
    if B > 1 and T == 1:
        st = sb  # a token a row: the rows' own stride
    elif B > 1 and sb != T * st:
        raise ValueError("%s: the rows of B must follow each other (stride %d, not T tokens of %d)"
                         % (name, sb, st))
    return Rows(x.data_ptr(), st, sh)


def _ints(name, x, device, shape=None):
    """Pointer of a contiguous int32 tensor on ``device``."""
    if not isinstance(x, torch.Tensor):
        raise TypeError("%s must be a tensor" % name)
    if x.dtype is not torch.int32 or x.device != device or not x.is_contiguous():
        raise ValueError("%s must be contiguous int32 on %s" % (name, device))
    if shape is not None and tuple(x.shape) != tuple(shape):
        raise ValueError("%s must be %s" % (name, list(shape)))
    return x.data_ptr()


def _tokens(q, Hk, cu_seqlens, cu_seqlens_host, keep):
    B, T, Hq, d = q.shape
    t = Tokens(B, T, Hq, Hk, d, 0, None, None, _DTYPES[q.dtype])
    if cu_seqlens is None:
        if cu_seqlens_host is not None:
            raise ValueError("cu_seqlens_host without cu_seqlens")
        return t, B
    dev, host = _cu_pair(cu_seqlens, cu_seqlens_host, q.device, keep)
    t.num_seqs = host.numel() - 1
    t.cu_seqlens, t.cu_seqlens_host = dev.data_ptr(), host.data_ptr()
    return t, t.num_seqs


def _cache(q, k_pages, v_pages, table, kv_lens, num_seqs):
    if not (isinstance(k_pages, torch.Tensor) and isinstance(v_pages, torch.Tensor)):
        raise TypeError("k_pages and v_pages must be tensors")
    if k_pages.dim() != 4 or k_pages.shape != v_pages.shape or k_pages.stride() != v_pages.stride():
        raise ValueError("k_pages and v_pages must be [num_pages, Hk, page_size, d], alike in "
                         "shape and strides")
    for x in (k_pages, v_pages):
        if x.dtype is not q.dtype or x.get_device() != q.get_device():
            raise ValueError("k_pages and v_pages must have q's dtype and device")
    num, Hk, page, d = k_pages.shape
    if d != q.shape[3] or k_pages.stride(3) != 1:
        raise ValueError("k_pages and v_pages must have q's d, contiguous")
    if not isinstance(table, torch.Tensor) or table.dim() != 2:
        raise ValueError("table must be int32 [sequences, blocks]")
    sp, sh, st, _ = k_pages.stride()
    return Cache(k_pages.data_ptr(), v_pages.data_ptr(), sp, sh, st, num, page, table.shape[1],
                 _ints("table", table, q.device, (num_seqs, table.shape[1])),
                 None if kv_lens is None else _ints("kv_lens", kv_lens, q.device, (num_seqs,)))


def _ref(x):
    return None if x is None else ctypes.byref(x)


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


def _rotary(r, device):
    if r is None:
        return None
    if not isinstance(r, Rotary):
        raise TypeError("rotary must be a Rotary (see gdn_rotary)")
    if r.turns.device != device or r.turns.dtype is not torch.float64 \
            or not r.turns.is_contiguous() or r.turns.dim() != 1:
        raise ValueError("rotary.turns must be contiguous float64 [rot / 2] on %s" % device)
    if r.layout not in LAYOUTS:
        raise ValueError("layout must be one of %s" % sorted(LAYOUTS))
    return RotaryStruct(2 * r.turns.numel(), LAYOUTS[r.layout], r.scale, r.turns.data_ptr())


def _rotate(f, q, k, rotary, positions, cu_seqlens, cu_seqlens_host, q_out, k_out):
    keep = []
    rq = _rows("q", q)
    rk = None if k is None else _rows("k", k, ("q", q))
    t, _ = _tokens(q, q.shape[2] if k is None else k.shape[2], cu_seqlens, cu_seqlens_host, keep)
    r = _rotary(rotary, q.device)
    if r is None:
        raise TypeError("rotary must be a Rotary (see gdn_rotary)")
    p = None if positions is None else _ints("positions", positions, q.device, q.shape[:2])
    if q_out is None:
        q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    if k is not None and k_out is None:
        k_out = torch.empty(k.shape, dtype=k.dtype, device=k.device)
    if q_out.shape != q.shape or (k is not None and k_out.shape != k.shape):
        raise ValueError("the outputs must be shaped as the inputs")
    ro = _rows("q_out", q_out, ("q", q))
    ko = None if k is None else _rows("k_out", k_out, ("q", q))
    _check(f(ctypes.byref(t), ctypes.byref(r), ctypes.byref(rq), _ref(rk), p, ctypes.byref(ro),
             _ref(ko), _stream(q.device)))
    del keep
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
                     cu_seqlens_host=None, q_out=None):
    """Stores the new tokens' k (rotated) and v in their sequences' pages; returns q, rotated.

    q [B, T, Hq, d] or None, k and v [B, T, Hk, d]; table int32 [sequences, blocks], kv_lens int32
    [sequences]: the tokens of each sequence with the new ones, which are its last.  ``rotary``
    None: nothing is rotated.  Tokens whose page is a hole are not stored."""
    lib = load_library()
    keep = []
    rk = _rows("k", k)
    rv = _rows("v", v, ("k", k))
    if v.shape != k.shape:
        raise ValueError("v must be shaped as k")
    rq = ro = None
    if q is not None:
        rq = _rows("q", q, ("k", k))
        if q_out is None:
            q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        if q_out.shape != q.shape:
            raise ValueError("q_out must be shaped as q")
        ro = _rows("q_out", q_out, ("k", k))
    t, n = _tokens(k if q is None else q, k.shape[2], cu_seqlens, cu_seqlens_host, keep)
    c = _cache(k, k_pages, v_pages, table, kv_lens, n)
    if k_pages.shape[1] != k.shape[2]:
        raise ValueError("k_pages must have k's heads")
    r = _rotary(rotary, k.device)
    _check(lib.gdn_cache_append(ctypes.byref(t), _ref(r), _ref(rq), ctypes.byref(rk),
                                ctypes.byref(rv), ctypes.byref(c), _ref(ro), _stream(k.device)))
    del keep
    return q_out


def _attn(scale, d, causal, window, max_kv):
    return Attn(d ** -0.5 if scale is None else scale, int(bool(causal)), int(window or 0),
                int(max_kv or 0))


def gdn_cache_attn_workspace_size(q, k_pages, table, scale=None, causal=True, window=0, max_kv=0,
                                  cu_seqlens=None, cu_seqlens_host=None) -> int:
    """Workspace bytes of gdn_cache_attn with these arguments (0: none is needed)."""
    keep = []
    t, n = _tokens(q, k_pages.shape[1], cu_seqlens, cu_seqlens_host, keep)
    c = _cache(q, k_pages, k_pages, table, None, n)
    a = _attn(scale, q.shape[3], causal, window, max_kv)
    size = int(load_library().gdn_cache_attn_workspace_size(ctypes.byref(t), ctypes.byref(c),
                                                            ctypes.byref(a)))
    del keep
    return size


def gdn_cache_attn(q, k_pages, v_pages, table, kv_lens, scale=None, causal=True, window=0,
                   max_kv=0, cu_seqlens=None, cu_seqlens_host=None, o=None, lse=None,
                   workspace=None):
    """Attention of the new tokens q [B, T, Hq, d] over their sequences' cached keys; returns o.

    The new tokens are the last of the kv_lens[n] that sequence n holds (gdn_cache_append has
    stored them).  ``scale`` None: 1 / sqrt(d); ``window`` > 0: a token sees itself and the window - 1
    before it; ``max_kv``: how long a sequence may be at most (0: what the table has room for),
    which the launches are sized by.  ``lse`` float32 [B, T, Hq] receives the log of each softmax's
    sum.  A token that sees no key gets 0 (lse -inf)."""
    lib = load_library()
    keep = []
    rq = _rows("q", q)
    t, n = _tokens(q, k_pages.shape[1] if isinstance(k_pages, torch.Tensor) else 0, cu_seqlens,
                   cu_seqlens_host, keep)
    c = _cache(q, k_pages, v_pages, table, kv_lens, n)
    if o is None:
        o = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    if o.shape != q.shape:
        raise ValueError("o must be shaped as q")
    ro = _rows("o", o, ("q", q))
    if lse is not None and (lse.dtype is not torch.float32 or lse.device != q.device
                            or not lse.is_contiguous() or lse.shape != q.shape[:3]):
        raise ValueError("lse must be contiguous float32 [B, T, Hq] on q's device")
    a = _attn(scale, q.shape[3], causal, window, max_kv)
    need = lib.gdn_cache_attn_workspace_size(ctypes.byref(t), ctypes.byref(c), ctypes.byref(a))
    if need and (workspace is None or workspace.numel() < need):
        workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
    if workspace is not None and (workspace.device != q.device or workspace.dtype is not torch.uint8
                                  or not workspace.is_contiguous()):
        raise ValueError("workspace must be a contiguous uint8 tensor on q's device")
    _check(lib.gdn_cache_attn(ctypes.byref(t), ctypes.byref(a), ctypes.byref(rq), ctypes.byref(c),
                              ctypes.byref(ro), _ptr(lse), _ptr(workspace),
                              0 if workspace is None else workspace.numel(), _stream(q.device)))
    del keep
    return o


# ------------------------------------------------------------------ pages


def _book(table, lens, refs, page_size, out, with_lens):
    """gdn_book of tensors, and the output tensors (``out``: the caller's, where given)."""
    if not isinstance(table, torch.Tensor) or table.dim() != 2:
        raise ValueError("table must be int32 [sequences, blocks]")
    if not isinstance(refs, torch.Tensor) or refs.dim() != 1:
        raise ValueError("refs must be int32 [pages]")
    dev, S = table.device, table.shape[0]
    if table.get_device() < 0:
        raise ValueError("table must be on the GPU")
    got = dict(out or {})
    for name, x in (("table", table), ("refs", refs)) + ((("lens", lens),) if with_lens else ()):
        if got.get(name) is None:
            got[name] = torch.empty_like(x)
    b = Book(S, table.shape[1], refs.numel(), page_size,
             _ints("table", table, dev, table.shape), _ints("lens", lens, dev, (S,)),
             _ints("refs", refs, dev), _ints("out table", got["table"], dev, table.shape),
             _ints("out lens", got["lens"], dev, (S,)) if with_lens else None,
             _ints("out refs", got["refs"], dev, refs.shape))
    return b, got


def _extra(got, name, shape, device):
    if got.get(name) is None:
        got[name] = torch.empty(shape, dtype=torch.int32, device=device)
    return _ints("out " + name, got[name], device, shape)


def _pool(pool, device):
    """gdn_pool of a [parts, num_pages, ...] tensor whose pages are contiguous."""
    if pool is None:
        return None
    if not isinstance(pool, torch.Tensor) or pool.dim() < 3 or pool.device != device:
        raise ValueError("pool must be a [parts, pages, ...] tensor on %s" % device)
    inner = 1
    for n, s in zip(reversed(pool.shape[2:]), reversed(pool.stride()[2:])):
        if n != 1 and s != inner:
            raise ValueError("pool must be contiguous within a page")
        inner *= n
    e = pool.element_size()
    return Pool(pool.data_ptr(), pool.shape[0], pool.shape[1], pool.stride(0) * e,
                pool.stride(1) * e, inner * e)


def _work(b, workspace, device):
    need = load_library().gdn_pages_workspace_size(ctypes.byref(b))
    if workspace is None or workspace.numel() < need:
        workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=device)
    if workspace.device != device or workspace.dtype is not torch.uint8 \
            or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous uint8 tensor on %s" % device)
    return workspace


def gdn_pages_workspace_size(table, refs) -> int:
    """Workspace bytes of the page calls for a table and reference counts of these shapes."""
    b = Book(table.shape[0], table.shape[1], refs.numel(), 1)
    return int(load_library().gdn_pages_workspace_size(ctypes.byref(b)))


def gdn_pages_extend(table, lens, refs, add, page_size, out=None, workspace=None):
    """Room for add[s] more tokens in each sequence: dict table, lens, refs, short.

    table int32 [S, blocks], lens and add int32 [S], refs int32 [pages] (holders of each page; 0:
    free).  short[s] > 0: there was no room for the pages it needs, and sequence s is as it was.  ``out``: dict of
    tensors to write; the inputs themselves update in place."""
    b, got = _book(table, lens, refs, page_size, out, True)
    short = _extra(got, "short", lens.shape, table.device)
    ws = _work(b, workspace, table.device)
    _check(load_library().gdn_pages_extend(
        ctypes.byref(b), _ints("add", add, table.device, lens.shape), short, ws.data_ptr(),
        ws.numel(), _stream(table.device)))
    return got


def gdn_pages_select(table, lens, refs, parents, page_size, pool=None, out=None, workspace=None):
    """Row i goes on from old row parents[i] (out of range: it ends): dict table, lens, refs, short.

    Frees, forks and reorders sequences in one call: full pages are shared, a partly filled last
    page is copied for every row but the lowest of its parent, in ``pool`` [parts, pages, ...].
    short[i] == 1: no page was left and row i is empty."""
    b, got = _book(table, lens, refs, page_size, out, True)
    short = _extra(got, "short", lens.shape, table.device)
    p = _pool(pool, table.device)
    ws = _work(b, workspace, table.device)
    _check(load_library().gdn_pages_select(
        ctypes.byref(b), _ints("parents", parents, table.device, lens.shape), _ref(p), short,
        ws.data_ptr(), ws.numel(), _stream(table.device)))
    return got


def gdn_pages_compact(table, lens, refs, page_size, pool=None, out=None, workspace=None):
    """Moves the pages in use into the lowest indexes: dict table, refs, map (new index of each
    page, -1 if it was free).  The data moves in ``pool`` [parts, pages, ...]."""
    b, got = _book(table, lens, refs, page_size, out, False)
    to = _extra(got, "map", refs.shape, table.device)
    p = _pool(pool, table.device)
    ws = _work(b, workspace, table.device)
    _check(load_library().gdn_pages_compact(ctypes.byref(b), _ref(p), to, ws.data_ptr(),
                                            ws.numel(), _stream(table.device)))
    return got


def gdn_pages_copy(pool, src, dst):
    """Copies pages src[i] to dst[i] (int32) in every part of ``pool`` [parts, pages, ...], a cache
    or a pool of recurrent states; pairs out of range are skipped."""
    if not isinstance(pool, torch.Tensor):
        raise TypeError("pool must be a tensor")
    p = _pool(pool, pool.device)
    if not isinstance(src, torch.Tensor) or src.dim() != 1:
        raise ValueError("src must be int32 [pairs]")
    _check(load_library().gdn_pages_copy(
        ctypes.byref(p), _ints("src", src, pool.device), _ints("dst", dst, pool.device, src.shape),
        src.numel(), _stream(pool.device)))
