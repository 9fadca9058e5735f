import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a CUDA device (run with -m gpu on a B200)")


@pytest.fixture(autouse=True)
def no_wait_ran_out(request):
    """After each GPU test of the layer's operators: no kernel gave up on a bounded wait (its outputs would be incomplete)."""
    yield
    if request.module.__name__.startswith("test_gpu_layer") and request.node.get_closest_marker("gpu"):
        from paper_2505_11157_b200 import sna
        sna.sna_layer_check()
