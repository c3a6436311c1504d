import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a CUDA GPU (GB300, sm_103a) and the built library")
    config.addinivalue_line("markers", "slow: long-running CPU test")


# Cases that expect a length of 0 of a sequence that does not fit its table, where the header gives it its start: they
# fail, and run last, so that a run that ends at its first failure has run all the others.
LAST = ("test_a_sequence_past_its_table_is_reported_and_left_out[3--2]",
        "test_a_sequence_past_its_table_is_reported_and_left_out[40-9]")


def pytest_collection_modifyitems(items):
    items.sort(key=lambda item: item.name in LAST)


@pytest.fixture(scope="session")
def golden_dir():
    return os.path.join(ROOT, "tests", "golden")
