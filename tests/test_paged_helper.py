"""The binding's native helper holds what paged.py calls, and nothing else."""
import inspect
import os
import re

from paper_2412_06464_amd import paged


def test_every_function_of_the_helper_is_called():
    here = os.path.dirname(os.path.abspath(paged.__file__))
    if not os.path.exists(os.path.join(here, "_paged_binding.so")):
        from paper_2412_06464_amd import build
        build.build_binding()
    has = {f for f in vars(paged._native()) if not f.startswith("__")}
    calls = set(re.findall(r"\b_n\.([a-z_]+)\(", inspect.getsource(paged)))
    assert has == calls
