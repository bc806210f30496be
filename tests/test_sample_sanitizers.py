"""Host side of the choice of tokens under AddressSanitizer and UndefinedBehaviorSanitizer (CPU): all
of gdn_sample.hip built with them on its host side, where its entry point is, and
tests/sanitize/sample_driver.c linked to it; none of its calls reaches a HIP call."""
import os
import subprocess

import pytest

from tests.test_sanitizers import CSRC, ENV, HOST_SAN, SAN, run


@pytest.mark.skipif(not os.path.exists("/opt/rocm/bin/hipcc"), reason="needs hipcc")
def test_host_side_under_asan_ubsan(tmp_path):
    from paper_2412_06464_amd import build
    api, drv, exe = (str(tmp_path / n) for n in ("api.o", "driver.o", "driver"))
    flags = [f for f in build.FLAGS if f != "-O3"] + ["-O1", "-g"]
    run([build.HIPCC, *flags, *HOST_SAN, "-c", os.path.join(CSRC, "gdn_sample.hip"), "-o", api])
    names = subprocess.run(["nm", api], capture_output=True, text=True, check=True).stdout
    assert "__ubsan_handle" in names and "__asan" in names  # the entry point is instrumented
    clang = "/opt/rocm/llvm/bin/clang"
    san = ["-fsanitize=address,undefined"]
    run([clang, "-O1", "-g", *san, "-fno-sanitize-recover=undefined", "-c",
         os.path.join(SAN, "sample_driver.c"), "-o", drv])
    run([clang + "++", *san, drv, api, "-L/opt/rocm/lib", "-lamdhip64",
         "-Wl,-rpath,/opt/rocm/lib", "-o", exe])
    assert "sample driver: ok" in run([exe], env=ENV, timeout=300).stdout
