import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a real MI355X (run with -m gpu)")


# Tests that stay as they are though what they compare with has been shown to be wrong, by (file, function).
WRONG_VALUES = {
    ("test_gpu_serving_loop.py", "test_a_bounded_cache_step_by_step"):
        "holds `recent` to the last PLACES of a cache that was cut back before (7 of the newest 8 rows at keep 44, high 50): test_oracle_positions.py shows "
        "that these are not the newest rows, test_gpu_serving_recent.py has the same walk by positions",
}


def pytest_collection_modifyitems(items):
    for item in items:
        reason = WRONG_VALUES.get((item.path.name, getattr(item, "originalname", None)))
        if reason:
            item.add_marker(pytest.mark.xfail(reason=reason, raises=AssertionError, strict=True))


@pytest.fixture(scope="session")
def oracle():
    import oracle as o
    from oracle.build import build
    build(force=False)
    return o
