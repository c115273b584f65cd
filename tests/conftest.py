import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a CUDA device (run with -m gpu on a B200)")


@pytest.fixture(scope="session")
def oracle():
    from oracle import perq_oracle
    perq_oracle.build()
    return perq_oracle


@pytest.fixture(autouse=True)
def no_device_error(request):
    """No wait inside a kernel runs out in any GPU test."""
    if request.node.get_closest_marker("gpu") is None:
        yield
        return
    import torch
    from paper_2601_22347_b200 import binding, build
    build.build()
    binding.perq_device_error_clear()
    yield
    torch.cuda.synchronize()
    assert binding.perq_device_error() == 0
