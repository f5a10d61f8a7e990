import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a CUDA device (run on a B200)")


# Tests that hold a wrong value: they stay as they are and have to fail, with what holds the right one.
WRONG = {
    "test_gpu_step.py::test_step_against_autograd": "weighs a factor by d_in / r, which ||A S^T||^2 over ||A||^2 is not on average (that is "
    "(d_in + r + 1) / r): test_gpu_step_edges.py::test_step_against_autograd_with_the_weight_of_the_factors has all of its checks",
}


def pytest_collection_modifyitems(items):
    for item in items:
        for name, reason in WRONG.items():
            if item.nodeid.endswith(name):
                item.add_marker(pytest.mark.xfail(reason=reason, raises=AssertionError, strict=True))


@pytest.fixture(scope="session")
def golden_dir():
    return os.path.join(ROOT, "tests", "golden")
