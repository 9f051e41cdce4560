import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs an MI355X (gfx950) GPU")
    config.addinivalue_line("markers", "slow: full-size workload")


def pytest_collection_modifyitems(items):
    # Its reference takes 1 / rms for 0 where a NaN in the row makes it NaN, and so pins zeros behind a NaN.
    # test_gpu_rows8_edges.py::test_norm_of_rows_that_are_not_finite holds the same calls to the definition.
    for item in items:
        if item.path.name == "test_gpu_rows8.py" and item.originalname == "test_norm_not_finite":
            item.add_marker(pytest.mark.xfail(strict=True, raises=AssertionError, reason="the reference pins zeros in rows with a NaN"))


@pytest.fixture(scope="session")
def oracle_lib():
    import oracle
    oracle.build(force=False)
    return oracle
