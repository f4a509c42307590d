"""The wait limit of the recurrence's calls: what it takes, before any device use."""
import pytest

from paper_2608_21308_b200 import binding as E
from paper_2608_21308_b200 import build as libbuild


def test_wait_limit():
    libbuild.build()
    try:
        assert E.e2ttt_selftest_scan_wait_limit(0) == 0 and E.e2ttt_selftest_scan_wait_limit(2_000_000_000) == 0
        with pytest.raises(E.E2TTTError):
            E.e2ttt_selftest_scan_wait_limit(2_000_000_001)
    finally:
        assert E.e2ttt_selftest_scan_wait_limit(-1) == 0
