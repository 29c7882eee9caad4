import gc
import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HERE = os.path.dirname(os.path.abspath(__file__))
for p in (ROOT, HERE):
    if p not in sys.path:
        sys.path.insert(0, p)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs an MI355X (gfx950) and the built HIP library")
    config.addinivalue_line("markers", "slow: longer CPU test")


def pytest_collection_finish(session):
    """What the run has loaded lives as long as it: left out of collections, which took some 100 ms each, longer than tests
    that look at a stream while it is busy keep it so."""
    gc.collect()
    gc.freeze()
