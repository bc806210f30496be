import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs an MI355X (gfx950) GPU and the built HIP library")


def pytest_collection_modifyitems(items):
    for item in items:
        if item.name == "test_m0_written_only_by_lds_dma_statements":
            # it takes the copy to be the very next instruction behind the write of m0, where
            # gfx950 asks for a wait state; test_lds_dma_waits.py holds the same rules with it
            item.add_marker(pytest.mark.xfail(
                strict=True, reason="a copy right behind its write of m0 may read the old m0"))


@pytest.fixture(scope="session")
def oracle_mod():
    from oracle import oracle
    oracle.build(force=False)
    return oracle
