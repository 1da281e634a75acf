import gc
import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a real MI355X (run with -m gpu)")


def pytest_collection_finish(session):
    gc.collect()
    gc.freeze()                                                 # (what lives for the whole run is not looked through again)


def pytest_runtest_setup(item):
    """What earlier tests left in cycles goes away before a test of the GPU, not in the middle of one that counts what is allocated."""
    if item.get_closest_marker("gpu"):
        gc.collect()


@pytest.fixture(scope="session")
def oracle_lib():
    from oracle import build_oracle
    return build_oracle()
