"""Wait states around the direct-to-LDS copies (global_load_lds), on the built gfx950 code objects.

The copies are issued from inline assembly, which the compiler's own hazard handling does not
look into, so what it would do for a copy of its own has to stand in the statement.  gfx950 does
not check for these by itself (the "manually inserted wait states" of the CDNA3 instruction set
manual, and what this compiler inserts around its builtin for the copy):

  * m0, the LDS address of a copy, written by a scalar instruction: one wait state before the copy;
  * a scalar register written by a vector instruction: five before a copy that reads it.

The compiler reserves m0 and does not honour it as a clobber, so the kernels also rely on its
never keeping a value of its own there: m0 is only ever written, by s_mov_b32, and only for the
copy that follows, and nothing that reads m0 implicitly appears."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2412_06464_amd import gdn

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
IMPLICIT_M0 = re.compile(r"^(s_movrel|v_movrel|s_sendmsg|ds_gws|v_interp|lds_param|ds_.*addtid)")
SGPRS = re.compile(r"\bs(?:(\d+)|\[(\d+):(\d+)\])")


def sgprs(text):
    """Scalar registers named in operands."""
    out = set()
    for one, lo, hi in SGPRS.findall(text):
        out |= {int(one)} if one else set(range(int(lo), int(hi) + 1))
    return out


def states(ins):
    """Wait states that an instruction takes."""
    return int(ins.split()[1], 0) + 1 if ins.startswith("s_nop") else 1


def faults(ins):
    """What is wrong in a list of instructions, in program order."""
    bad = []
    for i, x in enumerate(ins):
        op = x.split()[0]
        if IMPLICIT_M0.match(op):
            bad.append((i, "reads m0", x))
        if re.search(r"\bm0\b", x):
            # a write for the copy behind its wait state
            if op != "s_mov_b32" or x.split()[1].rstrip(",") != "m0":
                bad.append((i, "uses m0", x))
            elif not (ins[i + 1:i + 2] and ins[i + 1].startswith("s_nop")
                      and ins[i + 2:i + 3] and ins[i + 2].startswith("global_load_lds")):
                bad.append((i, "no copy behind a wait state", x))
        if not op.startswith("global_load_lds"):
            continue
        if i < 2 or not (ins[i - 1].startswith("s_nop") and ins[i - 2].startswith("s_mov_b32 m0")):
            bad.append((i, "no wait state behind its m0", x))
        read, passed = sgprs(x.split(None, 1)[1]), 0
        for y in reversed(ins[:i]):
            if passed >= 5:
                break
            parts = y.split(None, 1)
            # a vector instruction's first operand (and a carry's second) is what it writes
            if parts[0].startswith("v_") and len(parts) > 1:
                if sgprs(",".join(parts[1].split(",")[:2])) & read and not (
                        parts[1].startswith("v") and "co_" not in parts[0]):
                    bad.append((i, "reads a scalar register too soon behind " + y, x))
            passed += states(y)
    return bad


def code(lib, tmp):
    """Instructions of every gfx950 code object of a library."""
    copy = os.path.join(tmp, "lib.so")
    shutil.copy(lib, copy)
    subprocess.run([OBJDUMP, "--offloading", copy], cwd=tmp, check=True, capture_output=True)
    out = []
    for f in sorted(os.listdir(tmp)):
        if f.endswith("gfx950"):
            text = subprocess.run([OBJDUMP, "-d", "--mcpu=gfx950", os.path.join(tmp, f)],
                                  check=True, capture_output=True, text=True).stdout
            lines = [ln.split("//")[0].strip() for ln in text.splitlines()]
            out.append([x for x in lines
                        if x and re.match(r"^[a-z_0-9]+", x) and not x.endswith(">:")])
    return out


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="llvm-objdump not available")
def test_every_copy_waits_for_its_registers(tmp_path):
    if not os.path.exists(gdn.LIB_PATH):
        from paper_2412_06464_amd import build
        build.build()
    objs = code(gdn.LIB_PATH, str(tmp_path))
    assert objs, "no gfx950 code object in libgdn.so"
    assert sum(x.startswith("global_load_lds") for ins in objs for x in ins) > 0
    for ins in objs:
        bad = faults(ins)
        assert not bad, (len(bad), bad[:5])


@pytest.mark.parametrize("ins,what", [
    (["s_mov_b32 m0, s4", "global_load_lds_dword v1, off"], "no copy behind a wait state"),
    (["s_mov_b32 m0, s4", "s_nop 0", "s_mov_b32 s1, m0"], "uses m0"),
    (["s_add_i32 m0, s4, s5", "s_nop 0", "global_load_lds_dword v1, off"], "uses m0"),
    (["v_readfirstlane_b32 s2, v1", "s_mov_b32 m0, s4", "s_nop 0",
      "global_load_lds_dword v1, s[2:3]"], "reads a scalar register too soon"),
    (["s_sendmsg sendmsg(1)"], "reads m0")])
def test_checker_flags_planted_faults(ins, what):
    assert any(b[1].startswith(what) for b in faults(ins))


def test_checker_passes_what_waits():
    assert faults(["v_readfirstlane_b32 s2, v1", "s_nop 2", "s_mov_b32 m0, s4", "s_nop 0",
                   "global_load_lds_dword v1, s[2:3]", "v_cmp_lt_u32_e64 s[8:9], v1, s4",
                   "s_mov_b32 m0, s5", "s_nop 0", "global_load_lds_dwordx4 v[2:3], off"]) == []
