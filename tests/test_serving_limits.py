"""Refusals, sizes and checks of the serving operators on the CPU, beside those of test_serving_*.py."""
from __future__ import annotations

import pytest

from test_serving_attend import _call as attend


@pytest.mark.parametrize("change", [dict(wait_limit_us=-2), dict(wait_limit_us=-(1 << 31)), dict(reserved2=1)])
def test_attend_wait_limits(change):
    assert attend(**change) == 1
    assert attend(wait_limit_us=-1, n_seqs=0) == 0
