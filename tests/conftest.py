import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a real MI355X (run with -m gpu)")


# Tests that hold a wrong value.  They stay as they are, and are expected to fail on it.
HOLDS_A_WRONG_VALUE = {
    f"test_gpu_cache.py::test_a_life_of_sequences[{case}]":
        "its list model lets twins of a sequence with pages left over write to the same page; test_lives_of_sequences in "
        "test_gpu_pages.py is the same life with a model that does not"
    for case in ("17-32-500-20", "70-16-9000-30", "1500-16-70000-25")}


def pytest_collection_modifyitems(items):
    for item in items:
        why = HOLDS_A_WRONG_VALUE.get(item.nodeid.split("/")[-1])
        if why:
            item.add_marker(pytest.mark.xfail(reason=why, raises=AssertionError, strict=True))


@pytest.fixture(scope="session", autouse=True)
def _oracle_built():
    """The C oracle is compiled once per session if its library is missing or stale."""
    from oracle import build
    build.build(force=False)
