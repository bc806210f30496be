"""Host side of linear attention, of attention over a shared prefix and of the choice of tokens
under AddressSanitizer and UndefinedBehaviorSanitizer (CPU): gdn_linear_api.hip and
gdn_paged_api.hip built with them on the host side, tests/sanitize/answers_driver.c linked to them
and to the kernel objects of the regular build; none of its calls reaches a HIP call."""
import os

import pytest

from tests.test_sanitizers import CSRC, ENV, HOST_SAN, KBUILD, SAN, run


@pytest.mark.skipif(not os.path.exists("/opt/rocm/bin/hipcc"), reason="needs hipcc")
def test_host_side_under_asan_ubsan(tmp_path):
    from paper_2412_06464_amd import build
    kernels = [os.path.join(KBUILD, n + ".o")
               for n in ("gdn_attn", "gdn_paged", "gdn_linear", "gdn_sample")]
    if not all(os.path.exists(o) for o in kernels):
        build.build()
    drv, exe = (str(tmp_path / n) for n in ("driver.o", "driver"))
    flags = [f for f in build.FLAGS if f != "-O3"] + ["-O1", "-g"]
    apis = []
    for n in ("gdn_linear_api", "gdn_paged_api"):
        apis.append(str(tmp_path / (n + ".o")))
        run([build.HIPCC, *flags, *HOST_SAN, "-c", os.path.join(CSRC, n + ".hip"), "-o", apis[-1]])
    clang = "/opt/rocm/llvm/bin/clang"
    san = ["-fsanitize=address,undefined"]
    run([clang, "-O1", "-g", *san, "-fno-sanitize-recover=undefined", "-c",
         os.path.join(SAN, "answers_driver.c"), "-o", drv])
    run([clang + "++", *san, drv, *apis, *kernels, "-L/opt/rocm/lib", "-lamdhip64",
         "-Wl,-rpath,/opt/rocm/lib", "-o", exe])
    assert "answers driver: ok" in run([exe], env=ENV, timeout=300).stdout
