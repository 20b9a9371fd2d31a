import gc
import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a real MI355X (run with -m gpu)")


@pytest.fixture(scope="session")
def lib():
    """The HIP library through its Python binding; GPU tests only."""
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2602_04929_amd as tb
    gc.collect()
    gc.freeze()      # what the imports made is not looked through again after every test
    return tb


@pytest.fixture(autouse=True)
def collected(request):
    """A test that keeps an exception (`pytest.raises(...) as e`) leaves its frame in a cycle, with the graphs that it captured.  They go here: a collection in the middle of a later test's capture would
    destroy them there, where the device cannot be synchronised, and a destructor that fails ends the process."""
    yield
    if request.node.get_closest_marker("gpu"):
        gc.collect()
