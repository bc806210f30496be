"""C-ABI and binding checks of the attention layer that need no GPU: the exported symbols, the
frequencies, and every refusal, made on the host before any launch."""
import ctypes
import math
import os
import re

import pytest
import torch

from paper_2412_06464_amd import gdn, paged

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "gdn_paged.h")
FAKE, ODD = 0x10000, 0x10008  # device addresses are never dereferenced on the host
NULL, SHAPE, UNSUP, CU, WS, ALIGN, VALUE = 1, 2, 3, 4, 5, 7, 9


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(gdn.LIB_PATH):
        from paper_2412_06464_amd import build
        build.build()
    return paged.load_library()


def test_header_and_library_agree(lib):
    text = open(HEADER).read()
    names = set(re.findall(r"^\s*(?:gdn_status|size_t)\s+(gdn_[a-z_0-9]+)\s*\(", text, re.M))
    assert sorted(names) == sorted(paged.EXPORTS)
    for name in names:
        assert hasattr(lib, name)


def test_structs_match_the_header():
    """Sizes of the structures as a C compiler lays them out."""
    import shutil
    import subprocess
    import tempfile
    if shutil.which("gcc") is None:
        pytest.skip("needs gcc")
    names = dict(gdn_tokens=paged.Tokens, gdn_rows=paged.Rows, gdn_cache=paged.Cache,
                 gdn_rotary=paged.RotaryStruct, gdn_attn=paged.Attn, gdn_book=paged.Book,
                 gdn_pool=paged.Pool)
    with tempfile.TemporaryDirectory() as d:
        src = "#include <stdio.h>\n#include \"%s\"\nint main(void) {\n%s  return 0;\n}\n" % (
            HEADER, "".join('  printf("%s %%zu\\n", sizeof(%s));\n' % (n, n) for n in names))
        open(os.path.join(d, "s.c"), "w").write(src)
        subprocess.run(["gcc", "s.c", "-o", "s"], cwd=d, check=True)
        out = subprocess.run([os.path.join(d, "s")], capture_output=True, text=True, check=True)
    packed = dict(gdn_attn=paged._ATTN, gdn_book=paged._BOOK)
    for line in out.stdout.split("\n"):
        if line:
            name, size = line.split()
            assert ctypes.sizeof(names[name]) == int(size), name
            if name not in packed:
                continue
            # what the binding packs has the same fields at the same places
            values = range(1, 1 + len(names[name]._fields_))
            got = names[name].from_buffer_copy(packed[name].pack(*values).ljust(int(size), b"\0"))
            assert [getattr(got, f) for f, _ in names[name]._fields_] == list(values), name


# ------------------------------------------------------------------ frequencies


@pytest.mark.parametrize("rot", [2, 6, 64, 256])
def test_turns(rot):
    i = torch.arange(rot // 2, dtype=torch.float64)
    th = 10000.0 ** (-2 * i / rot)
    turns, scale = paged.gdn_rotary_turns(rot)
    assert scale == 1 and torch.allclose(turns, th / (2 * math.pi), rtol=1e-15, atol=0)
    turns, scale = paged.gdn_rotary_turns(rot, 5000.0, "linear", 4.0)
    assert torch.allclose(turns, 5000.0 ** (-2 * i / rot) / 4 / (2 * math.pi), rtol=1e-15, atol=0)
    turns, scale = paged.gdn_rotary_turns(rot, scaling="base", factor=8.0)
    b = 10000.0 * 8.0 ** (rot / (rot - 2)) if rot > 2 else 10000.0
    assert scale == 1 and torch.allclose(turns, b ** (-2 * i / rot) / (2 * math.pi), rtol=1e-14,
                                         atol=0)
    if rot > 2:  # the slowest pair is slowed by the whole factor
        assert turns[-1] / (th[-1] / (2 * math.pi)) == pytest.approx(1 / 8.0, rel=1e-12)
    turns, scale = paged.gdn_rotary_turns(rot, scaling="parts", factor=16.0, original=4096)
    g = ((4096 * th / (2 * math.pi) - 1) / 31).clamp(0, 1)
    want = ((1 - g) * th / 16 + g * th) / (2 * math.pi)
    assert torch.allclose(turns, want, rtol=1e-14, atol=0)
    assert scale == pytest.approx(0.1 * math.log(16) + 1, rel=1e-7)


@pytest.mark.parametrize("kw", [
    dict(rot=0), dict(rot=3), dict(rot=-2), dict(rot=8, base=1.0), dict(rot=8, base=math.nan),
    dict(rot=8, scaling="linear", factor=0.5), dict(rot=8, scaling="base", factor=math.inf),
    dict(rot=8, scaling="parts", factor=2.0), dict(rot=8, scaling="parts", factor=2.0, original=9,
                                                   slow=4.0, fast=4.0)])
def test_turns_refused(kw):
    with pytest.raises(gdn.GdnError) as e:
        paged.gdn_rotary_turns(**kw)
    assert e.value.code == VALUE


def test_turns_of_an_unknown_kind():
    with pytest.raises(ValueError):
        paged.gdn_rotary_turns(8, scaling="other")
    with pytest.raises(ValueError):
        paged.gdn_rotary(8, layout="other", device="cpu")


# ------------------------------------------------------------------ C entry points


def tokens(**kw):
    return paged.Tokens(**dict(dict(B=2, T=10, Hq=4, Hk=2, d=128, dtype=gdn.GDN_BF16), **kw))


def rows(p=FAKE, ts=512, hs=128):
    return paged.Rows(p, ts, hs)


def cache(**kw):
    return paged.Cache(**dict(dict(k=FAKE, v=FAKE, page_stride=16384, head_stride=8192,
                                   token_stride=128, num_pages=9, page_size=64, max_blocks=4,
                                   table=FAKE, kv_lens=FAKE), **kw))


def rotary(**kw):
    return paged.RotaryStruct(**dict(dict(rot=64, layout=0, scale=1.0, turns=FAKE), **kw))


def attn(**kw):
    return paged.Attn(**dict(dict(scale=0.1, causal=1, window=0, max_kv=0), **kw))


def ref(x):
    return None if x is None else ctypes.byref(x)


def call_rotary(lib, t=None, r=None, q=None, k=None, pos=None, qo=None, ko=None, **none):
    t, r = t or tokens(), r or rotary()
    q, qo = q or rows(), qo or rows()
    return lib.gdn_rotary_fwd(ref(t), ref(r), None if "q" in none else ref(q), ref(k), pos, ref(qo),
                              ref(ko), None)


BAD_TOKENS = [(dict(d=96), UNSUP), (dict(dtype=5), UNSUP), (dict(B=0), SHAPE), (dict(T=0), SHAPE),
              (dict(Hk=0), SHAPE), (dict(Hq=0), SHAPE),
              (dict(T=1 << 30), SHAPE)]


@pytest.mark.parametrize("kw,code", BAD_TOKENS)
def test_bad_tokens(lib, kw, code):
    t = tokens(**kw)
    r, c, a = rows(), cache(), attn()
    assert call_rotary(lib, t=t) == code
    assert lib.gdn_cache_append(ref(t), None, ref(r), ref(r), ref(r), ref(c), ref(r), None) == code
    assert lib.gdn_cache_attn(ref(t), ref(a), ref(r), ref(c), ref(r), None, None, 0, None) == code
    assert lib.gdn_cache_attn_workspace_size(ref(t), ref(c), ref(a)) == 0


def test_boundaries(lib):
    r = rows()
    for cu, kw in (([0, 6, 5, 10], {}), ([0, 4, 9], {}), ([1, 10], {}), ([0, 10], dict(B=2))):
        arr = (ctypes.c_int32 * len(cu))(*cu)
        t = tokens(**dict(dict(B=1, T=10, num_seqs=len(cu) - 1, cu_seqlens=FAKE,
                               cu_seqlens_host=ctypes.addressof(arr)), **kw))
        assert call_rotary(lib, t=t) == (SHAPE if kw else CU)
    assert call_rotary(lib, t=tokens(B=1, cu_seqlens=FAKE, num_seqs=1)) == CU
    assert call_rotary(lib, t=tokens(B=1, cu_seqlens_host=FAKE)) == CU
    assert lib.gdn_rotary_fwd(None, ref(rotary()), ref(r), None, None, ref(r), None, None) == NULL


def test_rotary_refusals(lib):
    r = rows()
    for kw in (dict(rot=0), dict(rot=7), dict(rot=130), dict(layout=2), dict(scale=math.inf)):
        assert call_rotary(lib, r=rotary(**kw)) == VALUE, kw
    assert call_rotary(lib, r=rotary(turns=None)) == NULL
    assert call_rotary(lib, r=rotary(turns=FAKE + 4)) == ALIGN
    t, h = tokens(), rotary()
    assert lib.gdn_rotary_bwd(ref(t), None, ref(r), None, None, ref(r), None, None) == NULL
    assert lib.gdn_rotary_bwd(ref(t), ref(h), None, None, None, ref(r), None, None) == NULL
    assert lib.gdn_rotary_bwd(ref(t), ref(h), ref(r), ref(r), None, ref(r), None, None) == NULL
    assert call_rotary(lib, q=rows(ODD)) == ALIGN
    assert call_rotary(lib, q=rows(ts=514)) == ALIGN
    assert call_rotary(lib, qo=rows(hs=132)) == ALIGN
    assert call_rotary(lib, pos=FAKE + 2) == ALIGN


@pytest.mark.parametrize("kw,code", [
    (dict(num_pages=0), SHAPE), (dict(max_blocks=0), SHAPE), (dict(page_size=8), SHAPE),
    (dict(page_size=48), SHAPE), (dict(page_size=2048), SHAPE), (dict(max_blocks=1 << 26), SHAPE),
    (dict(k=None), NULL), (dict(table=None), NULL), (dict(kv_lens=None), NULL),
    (dict(v=ODD), ALIGN), (dict(table=FAKE + 2), ALIGN), (dict(page_stride=12), ALIGN),
    (dict(token_stride=-128), SHAPE), (dict(token_stride=1 << 27), SHAPE)])
def test_bad_cache(lib, kw, code):
    t, r, c, a = tokens(), rows(), cache(**kw), attn()
    assert lib.gdn_cache_append(ref(t), None, ref(r), ref(r), ref(r), ref(c), ref(r), None) == code
    assert lib.gdn_cache_attn(ref(t), ref(a), ref(r), ref(c), ref(r), None, None, 0, None) == code


def test_append_and_attn_refusals(lib):
    t, r, c, a = tokens(), rows(), cache(), attn()
    ap = lib.gdn_cache_append
    assert ap(ref(t), None, ref(r), None, ref(r), ref(c), ref(r), None) == NULL
    assert ap(ref(t), None, ref(r), ref(r), None, ref(c), ref(r), None) == NULL
    assert ap(ref(t), None, ref(r), ref(r), ref(r), None, ref(r), None) == NULL
    assert ap(ref(t), None, ref(r), ref(r), ref(r), ref(c), None, None) == NULL
    assert ap(ref(t), ref(rotary(rot=256)), ref(r), ref(r), ref(r), ref(c), ref(r), None) == VALUE
    at = lib.gdn_cache_attn
    for kw in (dict(scale=0.0), dict(scale=-1.0), dict(scale=math.nan), dict(window=-1),
               dict(max_kv=-1), dict(window=4, causal=0)):
        assert at(ref(t), ref(attn(**kw)), ref(r), ref(c), ref(r), None, None, 0, None) == VALUE
    assert at(ref(tokens(Hk=3)), ref(a), ref(r), ref(c), ref(r), None, None, 0, None) == SHAPE
    assert at(ref(t), None, ref(r), ref(c), ref(r), None, None, 0, None) == NULL
    assert at(ref(t), ref(a), None, ref(c), ref(r), None, None, 0, None) == NULL
    assert at(ref(t), ref(a), ref(r), ref(c), None, None, None, 0, None) == NULL
    assert at(ref(t), ref(a), ref(r), ref(c), ref(r), FAKE + 2, None, 0, None) == ALIGN
    # a long cache for few rows is split: the workspace is required
    long = cache(max_blocks=4096)
    need = lib.gdn_cache_attn_workspace_size(ref(t), ref(long), ref(a))
    assert need >= 2 * 2 * 10 * 4 * (128 + 2) * 4  # at least two splits of the call's rows
    assert at(ref(t), ref(a), ref(r), ref(long), ref(r), None, None, 0, None) == WS
    assert at(ref(t), ref(a), ref(r), ref(long), ref(r), None, FAKE, need - 1, None) == WS
    assert at(ref(t), ref(a), ref(r), ref(long), ref(r), None, ODD, need, None) == ALIGN
    # many rows are not
    big = tokens(B=8, T=4096, Hq=16, Hk=4)
    assert lib.gdn_cache_attn_workspace_size(ref(big), ref(long), ref(a)) == 0


def book(**kw):
    return paged.Book(**dict(dict(S=4, max_blocks=8, num_pages=50, page_size=16, table=FAKE,
                                  lens=FAKE, refs=FAKE, table_out=FAKE, lens_out=FAKE,
                                  refs_out=FAKE), **kw))


def pool(**kw):
    return paged.Pool(**dict(dict(data=FAKE, parts=2, num_pages=50, part_stride=1 << 20,
                                  page_stride=4096, page_bytes=4096), **kw))


def page_calls(lib, b, p=None, ws=FAKE, n=1 << 40, x=FAKE, y=FAKE):
    return [lib.gdn_pages_extend(ref(b), x, y, ws, n, None),
            lib.gdn_pages_select(ref(b), x, ref(p), y, ws, n, None),
            lib.gdn_pages_compact(ref(b), ref(p), y, ws, n, None)]


@pytest.mark.parametrize("kw,code", [
    (dict(S=0), SHAPE), (dict(max_blocks=0), SHAPE), (dict(num_pages=0), SHAPE),
    (dict(num_pages=(1 << 20) + 1), SHAPE), (dict(page_size=0), SHAPE),
    (dict(page_size=1 << 28), SHAPE), (dict(table=None), NULL), (dict(refs=None), NULL),
    (dict(table_out=None), NULL), (dict(refs_out=None), NULL), (dict(table=FAKE + 1), ALIGN)])
def test_bad_book(lib, kw, code):
    assert page_calls(lib, book(**kw)) == [code] * 3


def test_page_refusals(lib):
    assert page_calls(lib, None) == [NULL] * 3
    assert page_calls(lib, book(lens_out=None))[:2] == [NULL] * 2
    need = lib.gdn_pages_workspace_size(ref(book()))
    assert need >= 4 * (2 * 50 + 3 * 4 + 4 * 8)
    assert page_calls(lib, book(), ws=None) == [WS] * 3
    assert page_calls(lib, book(), n=need - 1) == [WS] * 3
    assert page_calls(lib, book(), ws=ODD) == [ALIGN] * 3
    assert page_calls(lib, book(), y=None) == [NULL] * 3
    assert page_calls(lib, book(), x=None)[:2] == [NULL] * 2
    assert page_calls(lib, book(), y=FAKE + 2) == [ALIGN] * 3
    for kw, code in ((dict(data=None), NULL), (dict(parts=0), SHAPE), (dict(num_pages=49), SHAPE),
                     (dict(page_bytes=0), SHAPE), (dict(page_bytes=24), ALIGN),
                     (dict(page_stride=8), ALIGN), (dict(data=ODD), ALIGN)):
        assert page_calls(lib, book(), pool(**kw))[1:] == [code] * 2, kw
        if "num_pages" not in kw:
            assert lib.gdn_pages_copy(ref(pool(**kw)), FAKE, FAKE, 3, None) == code
    assert lib.gdn_pages_copy(None, FAKE, FAKE, 3, None) == NULL
    assert lib.gdn_pages_copy(ref(pool()), None, FAKE, 3, None) == NULL
    assert lib.gdn_pages_copy(ref(pool()), FAKE, FAKE + 2, 3, None) == ALIGN
    assert lib.gdn_pages_copy(ref(pool()), FAKE, FAKE, -1, None) == SHAPE
    assert lib.gdn_pages_copy(ref(pool()), FAKE, FAKE, 0, None) == 0


# ------------------------------------------------------------------ binding


def test_binding_refuses_cpu_tensors_and_mismatches():
    q, k = torch.zeros(1, 4, 2, 64), torch.zeros(1, 4, 1, 64)
    r = paged.gdn_rotary(64, device="cpu")
    with pytest.raises(ValueError, match="GPU"):
        paged.gdn_rotary_fwd(q, k, r)
    with pytest.raises(TypeError):
        paged.gdn_rotary_fwd([1], k, r)
    with pytest.raises(ValueError, match="heads, d"):
        paged.gdn_rotary_fwd(q[0], k, r)
    with pytest.raises(TypeError):
        paged.gdn_rotary_fwd(q.double(), k, r)
    with pytest.raises(ValueError):
        paged.gdn_pages_copy(torch.zeros(3, 4), None, None)
    with pytest.raises(ValueError, match="GPU"):
        paged.gdn_pages_extend(*[torch.zeros(s, dtype=torch.int32) for s in ((2, 3), (2,), (5,))],
                               add=None, page_size=16)


def test_longest_cache(lib):
    """Key positions stay clear of 32 bits: 2^31 - 2^18 tokens of room are the most."""
    t, a = tokens(), attn(max_kv=1000)
    most = (2 ** 31 - 2 ** 18) // 16
    for blocks, code in ((most, ALIGN), (most + 1, SHAPE), (2 ** 27 - 1, SHAPE)):
        c = cache(page_size=16, max_blocks=blocks)
        q = rows(ODD)  # what is checked next
        assert lib.gdn_cache_attn(ref(t), ref(a), ref(q), ref(c), ref(q), None, None, 0,
                                  None) == code
