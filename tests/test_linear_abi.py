"""C-ABI and binding checks of linear attention with a decay that need no GPU: the exported
symbols, and every refusal, made on the host before any launch."""
import ctypes
import os
import re

import pytest
import torch

from paper_2412_06464_amd import gdn, linear

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "gdn_linear.h")
FAKE, ODD = 0x10000, 0x10008  # device addresses are never dereferenced on the host
OK, NULL, SHAPE, UNSUP, CU, WS, ALIGN = 0, 1, 2, 3, 4, 5, 7


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(gdn.LIB_PATH):
        from paper_2412_06464_amd import build
        build.build()
    return linear.load_library()


def problem(**kw):
    return gdn.Problem(**dict(dict(B=2, T=100, H=4, dk=128, dv=256, num_seqs=0, cu_seqlens=None,
                                   cu_seqlens_host=None, dtype=gdn.GDN_BF16), **kw))


def calls(lib, p, q=FAKE, k=FAKE, v=FAKE, la=FAKE, h0=FAKE, o=FAKE, ht=FAKE, ws=FAKE,
          size=1 << 45):
    p = None if p is None else ctypes.byref(p)
    return [lib.gdn_linear_chunk_fwd(p, q, k, v, la, 0, h0, o, ht, ws, size, None),
            lib.gdn_linear_recurrent_fwd(p, q, k, v, la, 0, h0, o, ht, None)]


def test_header_and_library_agree(lib):
    text = open(HEADER).read()
    names = set(re.findall(r"^\s*(?:gdn_status|size_t)\s+(gdn_[a-z_0-9]+)\s*\(", text, re.M))
    assert sorted(names) == sorted(linear.EXPORTS)
    for name in names:
        assert hasattr(lib, name)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=7), UNSUP), (dict(dk=32), UNSUP), (dict(dk=192), UNSUP), (dict(dk=512), UNSUP),
    (dict(dv=32), UNSUP), (dict(dv=384), UNSUP), (dict(B=0), SHAPE), (dict(T=0), SHAPE),
    (dict(H=0), SHAPE), (dict(B=-1), SHAPE), (dict(B=2, T=1 << 30), SHAPE),
    (dict(B=1, T=(1 << 31) - 256), SHAPE), (dict(B=1 << 20, T=1), SHAPE),
    (dict(B=2, cu_seqlens=FAKE, num_seqs=1), SHAPE)])
def test_bad_problems(lib, kw, code):
    p = problem(**kw)
    assert calls(lib, p) == [code] * 2
    assert lib.gdn_linear_chunk_fwd_workspace_size(ctypes.byref(p)) == 0


@pytest.mark.parametrize("cu", [[1, 100], [0, 60, 50, 100], [0, 50, 99], [0, 50, 101]])
def test_bad_boundaries(lib, cu):
    host = (ctypes.c_int32 * len(cu))(*cu)
    p = problem(B=1, num_seqs=len(cu) - 1, cu_seqlens=FAKE, cu_seqlens_host=ctypes.addressof(host))
    assert calls(lib, p) == [CU] * 2
    assert lib.gdn_linear_chunk_fwd_workspace_size(ctypes.byref(p)) == 0
    for more in (dict(cu_seqlens_host=None), dict(cu_seqlens=None), dict(num_seqs=0)):
        q = problem(B=1, num_seqs=len(cu) - 1, cu_seqlens=FAKE,
                    cu_seqlens_host=ctypes.addressof(host))
        for f, x in more.items():
            setattr(q, f, x)
        assert calls(lib, q) == [CU] * 2


def test_pointers(lib):
    assert calls(lib, None) == [NULL] * 2
    assert lib.gdn_linear_chunk_fwd_workspace_size(None) == 0
    p = problem()
    for name in ("q", "k", "v", "o"):
        assert calls(lib, p, **{name: None}) == [NULL] * 2, name
    for name in ("q", "k", "v", "la", "h0", "o", "ht"):
        assert calls(lib, p, **{name: ODD}) == [ALIGN] * 2, name


def test_workspace(lib):
    """One long sequence of few heads is cut, and its segments' states need room; sequences that
    fill the GPU need none."""
    p = problem(B=1, T=16384)
    need = lib.gdn_linear_chunk_fwd_workspace_size(ctypes.byref(p))
    assert need >= 2 * 4 * 128 * 256 * 4
    assert calls(lib, p, ws=None)[0] == WS
    assert calls(lib, p, size=need - 1)[0] == WS
    assert calls(lib, p, ws=ODD)[0] == ALIGN
    assert lib.gdn_linear_chunk_fwd_workspace_size(ctypes.byref(problem(B=64, T=512, H=8))) == 0
    assert lib.gdn_linear_chunk_fwd_workspace_size(ctypes.byref(problem(B=1, T=64, H=1))) == 0
    # packed: any boundaries of these sequences fit what their lengths ask for
    cu = [0, 0, 9000, 9001, 16384]
    host = (ctypes.c_int32 * len(cu))(*cu)
    p = problem(B=1, T=16384, num_seqs=4, cu_seqlens=FAKE, cu_seqlens_host=ctypes.addressof(host))
    assert lib.gdn_linear_chunk_fwd_workspace_size(ctypes.byref(p)) >= 4 * 4 * 128 * 256 * 4


def test_binding_refuses_cpu_tensors_and_mismatches():
    q, v = torch.zeros(1, 4, 2, 64), torch.zeros(1, 4, 2, 128)
    for call in (linear.gdn_linear_chunk_fwd, linear.gdn_linear_recurrent_fwd):
        with pytest.raises(ValueError):
            call(q, q, v, None)
        with pytest.raises(TypeError):
            call(q.double(), q.double(), v.double(), None)
        with pytest.raises(ValueError):
            call(q[0], q[0], v[0], None)
        with pytest.raises(ValueError):
            call(q, q, v[:, :, :1], None)
        with pytest.raises(ValueError, match="log_alpha"):
            call(q, q, v, torch.zeros(3))
