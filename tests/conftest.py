import gc
import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs an MI355X (gfx950) GPU and the built HIP library")


@pytest.fixture(autouse=True)
def _no_garbage_in_a_capture(request):
    """Graphs and ctxs of earlier tests sit in reference cycles (pytest.raises keeps its frame).
    A collection in the middle of a capture would free them there, and a graph's destructor
    waits for the device, which HIP refuses then: the process ends.  So they go first."""
    if "captur" in request.node.name:
        gc.collect()
