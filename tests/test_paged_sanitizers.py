"""Host side of the attention layer under AddressSanitizer and UndefinedBehaviorSanitizer (CPU):
gdn_paged_api.hip built with them on its host side, tests/sanitize/paged_driver.c linked to it and
to the kernel objects of the regular build; none of its calls reaches a HIP call."""
import os

import pytest

from tests.test_sanitizers import CSRC, ENV, HOST_SAN, KBUILD, SAN, run


@pytest.mark.skipif(not os.path.exists("/opt/rocm/bin/hipcc"), reason="needs hipcc")
def test_host_side_under_asan_ubsan(tmp_path):
    from paper_2412_06464_amd import build
    kernels = [os.path.join(KBUILD, n + ".o") for n in ("gdn_attn", "gdn_paged")]
    if not all(os.path.exists(o) for o in kernels):
        build.build()
    api, drv, exe = (str(tmp_path / n) for n in ("api.o", "driver.o", "driver"))
    flags = [f for f in build.FLAGS if f != "-O3"] + ["-O1", "-g"]
    run([build.HIPCC, *flags, *HOST_SAN, "-c", os.path.join(CSRC, "gdn_paged_api.hip"), "-o", api])
    clang = "/opt/rocm/llvm/bin/clang"
    san = ["-fsanitize=address,undefined"]
    run([clang, "-O1", "-g", *san, "-fno-sanitize-recover=undefined", "-c",
         os.path.join(SAN, "paged_driver.c"), "-o", drv])
    run([clang + "++", *san, drv, api, *kernels, "-L/opt/rocm/lib", "-lamdhip64",
         "-Wl,-rpath,/opt/rocm/lib", "-o", exe])
    assert "paged driver: ok" in run([exe], env=ENV, timeout=300).stdout
