import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a real MI355X (run with -m gpu)")


@pytest.fixture(autouse=True)
def _letter_of_the_paper(request, monkeypatch):
    """One pin states which blocks share an identity in the letter of the paper, by the adapter id alone; it is run in that reading of the oracle.  (The
    adopted one tells activation points inside a block apart as well: test_reuse_length_equals_the_flat_definition_with_places.)"""
    if request.node.name == "test_oracle_reuse_length_equals_the_flat_definition":
        from oracle.prefix_cache import PrefixCacheOracle
        monkeypatch.setattr(PrefixCacheOracle, "place", False)
