import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a CUDA GPU (sm_103a) and the built library")


@pytest.fixture(scope="session")
def golden_dir():
    return os.path.join(ROOT, "tests", "golden")


@pytest.fixture(autouse=True)
def no_wait_gave_up(request):
    """After each GPU test of the serving operators: no wait of paged attention ran into its limit."""
    yield
    if request.node.get_closest_marker("gpu") and "serving" in request.node.fspath.basename:
        from paper_2608_28003_gb300 import binding
        binding.paged_attention_check()
