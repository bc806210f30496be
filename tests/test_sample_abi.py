"""C-ABI and binding checks of the choice of the next token that need no GPU: the exported symbol,
the structure, and every refusal, made on the host before any launch."""
import ctypes
import os
import re
import shutil
import subprocess

import pytest
import torch

from paper_2412_06464_amd import gdn, sample

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "gdn_sample.h")
FAKE = 0x10000  # device addresses are never dereferenced on the host
NULL, SHAPE, UNSUP, ALIGN = 1, 2, 3, 7


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(gdn.LIB_PATH):
        from paper_2412_06464_amd import build
        build.build()
    return sample.load_library()


def call(lib, tokens=FAKE, logprob=FAKE, **kw):
    s = sample.Sampling(**dict(dict(rows=4, vocab=100, dtype=gdn.GDN_BF16, logits=FAKE,
                                    row_stride=100, temperature=FAKE, top_k=FAKE, top_p=FAKE,
                                    min_p=FAKE, u=FAKE), **kw))
    return lib.gdn_sample(ctypes.byref(s), tokens, logprob, None)


def test_header_and_library_agree(lib, tmp_path):
    text = open(HEADER).read()
    names = set(re.findall(r"^\s*(?:gdn_status|size_t)\s+(gdn_[a-z_0-9]+)\s*\(", text, re.M))
    assert sorted(names) == sorted(sample.EXPORTS)
    for name in names:
        assert hasattr(lib, name)
    if shutil.which("gcc") is None:
        pytest.skip("needs gcc")
    fields = [f for f, _ in sample.Sampling._fields_]
    (tmp_path / "s.c").write_text(
        "#include <stddef.h>\n#include <stdio.h>\n#include \"%s\"\nint main(void) {\n%s"
        "  printf(\"%%zu\\n\", sizeof(gdn_sampling));\n  return 0;\n}\n"
        % (HEADER, "".join('  printf("%%zu\\n", offsetof(gdn_sampling, %s));\n' % f
                           for f in fields)))
    subprocess.run(["gcc", "s.c", "-o", "s"], cwd=tmp_path, check=True)
    out = subprocess.run([str(tmp_path / "s")], capture_output=True, text=True, check=True)
    want = [getattr(sample.Sampling, f).offset for f in fields] + [ctypes.sizeof(sample.Sampling)]
    assert [int(x) for x in out.stdout.split()] == want


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=9), UNSUP), (dict(rows=0), SHAPE), (dict(rows=-1), SHAPE),
    (dict(rows=1 << 22), SHAPE), (dict(vocab=0), SHAPE), (dict(vocab=(1 << 20) + 1), SHAPE),
    (dict(row_stride=(1 << 40) + 1), SHAPE), (dict(row_stride=-(1 << 40) - 1), SHAPE),
    (dict(logits=None), NULL), (dict(tokens=None), NULL), (dict(u=None, temperature=None), NULL),
    (dict(logits=FAKE + 1), ALIGN), (dict(logits=FAKE + 2, dtype=gdn.GDN_F32), ALIGN),
    (dict(temperature=FAKE + 2), ALIGN), (dict(top_k=FAKE + 2), ALIGN),
    (dict(top_p=FAKE + 1), ALIGN), (dict(min_p=FAKE + 2), ALIGN), (dict(u=FAKE + 2), ALIGN),
    (dict(tokens=FAKE + 2), ALIGN), (dict(logprob=FAKE + 2), ALIGN)])
def test_refusals(lib, kw, code):
    assert call(lib, **kw) == code


def test_no_description(lib):
    assert lib.gdn_sample(None, FAKE, FAKE, None) == NULL


def test_binding_refuses_cpu_tensors_and_mismatches():
    u = torch.zeros(4)
    with pytest.raises(TypeError):
        sample.gdn_sample([1.0], u)
    with pytest.raises(TypeError):
        sample.gdn_sample(torch.zeros(4, 10, dtype=torch.float64), u)
    with pytest.raises(ValueError, match="GPU"):
        sample.gdn_sample(torch.zeros(4, 10), u)
    with pytest.raises(ValueError, match="rows, vocab"):
        sample.gdn_sample(torch.zeros(4, 10, 2), u)
