import gc
import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs an MI355X (gfx950) GPU and the built HIP library")
    config.addinivalue_line("markers", "slow: long-running CPU test")


@pytest.fixture(scope="session")
def _loaded_objects():
    """What is loaded by the first test stays: collections need not go through it."""
    gc.collect()
    gc.freeze()


@pytest.fixture(autouse=True)
def _collector(request):
    """A GPU test runs with the cyclic collector off, and what it leaves in cycles is
    collected behind it: a recorded graph or a handle that the collector destroyed
    while a stream records would break that recording, or end the process."""
    if not request.node.get_closest_marker("gpu"):
        yield
        return
    request.getfixturevalue("_loaded_objects")
    gc.collect()
    gc.disable()
    try:
        yield
    finally:
        gc.enable()
        gc.collect()


@pytest.fixture(scope="session")
def repo_root():
    return ROOT
