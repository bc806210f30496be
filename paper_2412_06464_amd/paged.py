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
import struct
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


# A call of a few microseconds on the GPU must not spend longer here.  The
# structures are packed as bytes, in the layout of the ctypes classes above
# (0.2 us each instead of 0.5 to 1), and what every call checks of a tensor is
# read once (host time of a call: storing a token for each of 256 sequences
# 19.4 -> 10.0 us, attention of one token for each of 4 15.1 -> 10.3 us).
_ROWS = struct.Struct("@Pqq")
_TOKENS = struct.Struct("@iiiiiiPPi0P")
_CACHE = struct.Struct("@PPqqqiiiPP")
_ROTARY = struct.Struct("@iifP")
_ATTN = struct.Struct("@fiii")
_BOOK = struct.Struct("@iiiiPPPPPP")
_POOL = struct.Struct("@Piiqqq")
_DTYPES = {torch.float32: GDN_F32, torch.bfloat16: GDN_BF16}
_Tensor = torch.Tensor
_I32 = torch.int32


class _Like(NamedTuple):
    """What the tensors of a call share, read off its first."""
    name: str
    B: int
    T: int
    d: int
    dtype: torch.dtype
    dev: int


def _first(name, x):
    """(_Like, heads) of a call's first [B, T, heads, d] tensor."""
    if not isinstance(x, _Tensor):
        raise TypeError("%s must be a tensor" % name)
    if x.dim() != 4:
        raise ValueError("%s must be [B, T, heads, d]" % name)
    B, T, H, d = x.shape
    dev = x.get_device()
    if x.dtype not in _DTYPES:
        raise TypeError("%s must be float32 or bfloat16" % name)
    if dev < 0:
        raise ValueError("%s must be on the GPU" % name)
    return _Like(name, B, T, d, x.dtype, dev), H


def _rows(name, x, like, heads=None):
    """gdn_rows of a [B, T, heads, d] tensor alike to the call's first."""
    if not isinstance(x, _Tensor):
        raise TypeError("%s must be a tensor" % name)
    if x.dim() != 4:
        raise ValueError("%s must be [B, T, heads, d]" % name)
    B, T, H, d = x.shape
    sb, st, sh, sd = x.stride()
    if x.dtype is not like.dtype or x.get_device() != like.dev:
        raise ValueError("%s must have %s's dtype and device" % (name, like.name))
    if B != like.B or T != like.T or d != like.d:
        raise ValueError("%s must have %s's B, T and d" % (name, like.name))
    if heads is not None and H != heads:
        raise ValueError("%s must have %d heads" % (name, heads))
    if sd != 1 and d != 1:
        raise ValueError("%s must be contiguous in its last dim" % name)
    if B > 1 and sb != T * st:
        if T != 1:
            raise ValueError("%s: the rows of B must follow each other (stride %d, not T tokens of "
                             "%d)" % (name, sb, st))
        st = sb  # a token a row: the rows' own stride
    return _ROWS.pack(x.data_ptr(), st, sh)


def _ints(name, x, dev, shape=None):
    """Pointer of a contiguous int32 tensor on device ``dev``."""
    if not isinstance(x, _Tensor):
        raise TypeError("%s must be a tensor" % name)
    if x.dtype is not _I32 or x.get_device() != dev or not x.is_contiguous():
        raise ValueError("%s must be contiguous int32 on the call's device" % name)
    if shape is not None and x.shape != shape:
        raise ValueError("%s must be %s" % (name, list(shape)))
    return x.data_ptr()


def _tokens(like, Hq, Hk, cu_seqlens, cu_seqlens_host, device, keep):
    """gdn_tokens, and the number of sequences."""
    if cu_seqlens is None:
        if cu_seqlens_host is not None:
            raise ValueError("cu_seqlens_host without cu_seqlens")
        return _TOKENS.pack(like.B, like.T, Hq, Hk, like.d, 0, 0, 0, _DTYPES[like.dtype]), like.B
    dev, host = _cu_pair(cu_seqlens, cu_seqlens_host, device, keep)
    keep.append(dev)
    n = host.numel() - 1
    return _TOKENS.pack(like.B, like.T, Hq, Hk, like.d, n, dev.data_ptr(), host.data_ptr(),
                        _DTYPES[like.dtype]), n


def _cache(like, k_pages, v_pages, table, kv_lens, num_seqs):
    """gdn_cache, and the cache's heads."""
    if not (isinstance(k_pages, _Tensor) and isinstance(v_pages, _Tensor)):
        raise TypeError("k_pages and v_pages must be tensors")
    shape, stride = k_pages.shape, k_pages.stride()
    if len(shape) != 4 or shape != v_pages.shape or stride != v_pages.stride():
        raise ValueError("k_pages and v_pages must be [num_pages, Hk, page_size, d], alike in "
                         "shape and strides")
    if (k_pages.dtype is not like.dtype or v_pages.dtype is not like.dtype
            or k_pages.get_device() != like.dev or v_pages.get_device() != like.dev):
        raise ValueError("k_pages and v_pages must have %s's dtype and device" % like.name)
    num, Hk, page, d = shape
    if d != like.d or stride[3] != 1:
        raise ValueError("k_pages and v_pages must have %s's d, contiguous" % like.name)
    if not isinstance(table, _Tensor) or table.dim() != 2 or table.shape[0] != num_seqs:
        raise ValueError("table must be int32 [%d sequences, blocks]" % num_seqs)
    return _CACHE.pack(k_pages.data_ptr(), v_pages.data_ptr(), stride[0], stride[1], stride[2], num,
                       page, table.shape[1], _ints("table", table, like.dev),
                       0 if kv_lens is None
                       else _ints("kv_lens", kv_lens, like.dev, (num_seqs,))), Hk


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


def _rotary(r, dev):
    if not isinstance(r, Rotary):
        raise TypeError("rotary must be a Rotary (see gdn_rotary)")
    t = r.turns
    if t.get_device() != dev or t.dtype is not torch.float64 or t.dim() != 1 \
            or not t.is_contiguous():
        raise ValueError("rotary.turns must be contiguous float64 [rot / 2] on the call's device")
    if r.layout not in LAYOUTS:
        raise ValueError("layout must be one of %s" % sorted(LAYOUTS))
    return _ROTARY.pack(2 * t.numel(), LAYOUTS[r.layout], r.scale, t.data_ptr())


def _rotate(f, q, k, rotary, positions, cu_seqlens, cu_seqlens_host, q_out, k_out):
    keep = []
    like, Hq = _first("q", q)
    rq, rk, ko, Hk = _rows("q", q, like), None, None, 1
    if q_out is None:
        q_out = torch.empty_like(q)
    if k is not None:
        rk, Hk = _rows("k", k, like), k.shape[2]
        if k_out is None:
            k_out = torch.empty_like(k)
        ko = _rows("k_out", k_out, like, Hk)
    dev = q.device
    t, _ = _tokens(like, Hq, Hk, cu_seqlens, cu_seqlens_host, dev, keep)
    p = None if positions is None else _ints("positions", positions, like.dev, q.shape[:2])
    _check(f(t, _rotary(rotary, like.dev), rq, rk, p, _rows("q_out", q_out, like, Hq), ko,
             _stream(dev)))
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
    like, Hk = _first("k", k)
    dev, Hq, rq, ro = k.device, Hk, None, None
    if q is not None:
        rq, Hq = _rows("q", q, like), q.shape[2]
        if q_out is None:
            q_out = torch.empty_like(q)
        ro = _rows("q_out", q_out, like, Hq)
    t, n = _tokens(like, Hq, Hk, cu_seqlens, cu_seqlens_host, dev, keep)
    c, heads = _cache(like, k_pages, v_pages, table, kv_lens, n)
    if heads != Hk:
        raise ValueError("k_pages must have k's heads")
    _check(lib.gdn_cache_append(t, None if rotary is None else _rotary(rotary, like.dev), rq,
                                _rows("k", k, like), _rows("v", v, like, Hk), c, ro,
                                _stream(dev)))
    return q_out


def _attn(scale, d, causal, window, max_kv):
    return _ATTN.pack(d ** -0.5 if scale is None else scale, 1 if causal else 0, window or 0,
                      max_kv or 0)


def gdn_cache_attn_workspace_size(q, k_pages, table, scale=None, causal=True, window=0, max_kv=0,
                                  cu_seqlens=None, cu_seqlens_host=None) -> int:
    """Workspace bytes of gdn_cache_attn with these arguments (0: none is needed)."""
    keep = []
    like, Hq = _first("q", q)
    n = like.B if cu_seqlens is None else cu_seqlens.numel() - 1
    c, Hk = _cache(like, k_pages, k_pages, table, None, n)
    t, _ = _tokens(like, Hq, Hk, cu_seqlens, cu_seqlens_host, q.device, keep)
    return int(load_library().gdn_cache_attn_workspace_size(t, c, _attn(scale, like.d, causal,
                                                                        window, max_kv)))


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
    like, Hq = _first("q", q)
    dev = q.device
    n = like.B if cu_seqlens is None else cu_seqlens.numel() - 1
    c, Hk = _cache(like, k_pages, v_pages, table, kv_lens, n)
    t, _ = _tokens(like, Hq, Hk, cu_seqlens, cu_seqlens_host, dev, keep)
    if o is None:
        o = torch.empty_like(q)
    if lse is not None and (lse.dtype is not torch.float32 or lse.get_device() != like.dev
                            or not lse.is_contiguous() or lse.shape != q.shape[:3]):
        raise ValueError("lse must be contiguous float32 [B, T, Hq] on q's device")
    a = _attn(scale, like.d, causal, window, max_kv)
    need = lib.gdn_cache_attn_workspace_size(t, c, a)
    ws, size = None, 0
    if need:
        if workspace is None or workspace.numel() < need:
            workspace = torch.empty(need, dtype=torch.uint8, device=dev)
        elif (workspace.get_device() != like.dev or workspace.dtype is not torch.uint8
              or not workspace.is_contiguous()):
            raise ValueError("workspace must be a contiguous uint8 tensor on q's device")
        ws, size = workspace.data_ptr(), workspace.numel()
    _check(lib.gdn_cache_attn(t, a, _rows("q", q, like), c, _rows("o", o, like, Hq), _ptr(lse), ws,
                              size, _stream(dev)))
    return o


# ------------------------------------------------------------------ pages


def _book(table, lens, refs, page_size, out, with_lens, extra, extra_shape):
    """gdn_book of tensors, the output tensors (``out``: the caller's, where given), the pointer of
    the one named ``extra``, the device."""
    if not isinstance(table, _Tensor) or table.dim() != 2:
        raise ValueError("table must be int32 [sequences, blocks]")
    if not isinstance(refs, _Tensor) or refs.dim() != 1:
        raise ValueError("refs must be int32 [pages]")
    dev, shape = table.get_device(), table.shape
    if dev < 0:
        raise ValueError("table must be on the GPU")
    S = shape[:1]
    pt, pl, pr = _ints("table", table, dev), _ints("lens", lens, dev, S), _ints("refs", refs, dev)
    if out is None:
        got = {"table": torch.empty_like(table)}
        if with_lens:
            got["lens"] = torch.empty_like(lens)
        got["refs"] = torch.empty_like(refs)
        got[extra] = torch.empty_like(refs if extra == "map" else lens)
    else:
        got = dict(out)
        for name, x in (("table", table), ("refs", refs), ("lens", lens if with_lens else None),
                        (extra, refs if extra == "map" else lens)):
            if x is not None and got.get(name) is None:
                got[name] = torch.empty_like(x)
    b = _BOOK.pack(S[0], shape[1], refs.numel(), page_size, pt, pl, pr,
                   _ints("out table", got["table"], dev, shape),
                   _ints("out lens", got["lens"], dev, S) if with_lens else 0,
                   _ints("out refs", got["refs"], dev, refs.shape))
    return b, got, _ints("out " + extra, got[extra], dev, extra_shape), dev


def _pool(pool, dev):
    """gdn_pool of a [parts, num_pages, ...] tensor whose pages are contiguous."""
    if pool is None:
        return None
    if not isinstance(pool, _Tensor) or pool.dim() < 3 or pool.get_device() != dev or dev < 0:
        raise ValueError("pool must be a [parts, pages, ...] tensor on the GPU of the call")
    shape, stride, inner = pool.shape, pool.stride(), 1
    for i in range(len(shape) - 1, 1, -1):
        if shape[i] != 1 and stride[i] != inner:
            raise ValueError("pool must be contiguous within a page")
        inner *= shape[i]
    e = pool.element_size()
    return _POOL.pack(pool.data_ptr(), shape[0], shape[1], stride[0] * e, stride[1] * e, inner * e)


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
    free).  short[s] > 0: there was no room for the pages it needs, and sequence s is as it was.
    ``out``: dict of tensors to write; the inputs themselves update in place."""
    lib = load_library()
    b, got, short, dev = _book(table, lens, refs, page_size, out, True, "short", lens.shape)
    device = table.device
    ws, p, n = _work(lib, b, workspace, device)
    _check(lib.gdn_pages_extend(b, _ints("add", add, dev, lens.shape), short, p, n,
                                _stream(device)))
    return got


def gdn_pages_select(table, lens, refs, parents, page_size, pool=None, out=None, workspace=None):
    """Row i goes on from old row parents[i] (out of range: it ends): dict table, lens, refs, short.

    Frees, forks and reorders sequences in one call: full pages are shared, a partly filled last
    page is copied for every row but the lowest of its parent, in ``pool`` [parts, pages, ...].
    short[i] == 1: no page was left and row i is empty."""
    lib = load_library()
    b, got, short, dev = _book(table, lens, refs, page_size, out, True, "short", lens.shape)
    device = table.device
    ws, p, n = _work(lib, b, workspace, device)
    _check(lib.gdn_pages_select(b, _ints("parents", parents, dev, lens.shape), _pool(pool, dev),
                                short, p, n, _stream(device)))
    return got


def gdn_pages_compact(table, lens, refs, page_size, pool=None, out=None, workspace=None):
    """Moves the pages in use into the lowest indexes: dict table, refs, map (new index of each
    page, -1 if it was free).  The data moves in ``pool`` [parts, pages, ...]."""
    lib = load_library()
    b, got, to, dev = _book(table, lens, refs, page_size, out, False, "map", refs.shape)
    device = table.device
    ws, p, n = _work(lib, b, workspace, device)
    _check(lib.gdn_pages_compact(b, _pool(pool, dev), to, p, n, _stream(device)))
    return got


def gdn_pages_copy(pool, src, dst):
    """Copies pages src[i] to dst[i] (int32) in every part of ``pool`` [parts, pages, ...], a cache
    or a pool of recurrent states; pairs out of range are skipped."""
    if not isinstance(pool, _Tensor):
        raise TypeError("pool must be a tensor")
    dev = pool.get_device()
    p = _pool(pool, dev)
    if not isinstance(src, _Tensor) or src.dim() != 1:
        raise ValueError("src must be int32 [pairs]")
    _check(load_library().gdn_pages_copy(p, _ints("src", src, dev), _ints("dst", dst, dev, src.shape),
                                         src.numel(), _stream(pool.device)))
