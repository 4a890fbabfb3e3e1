"""The order in which the sequences of an uneven batch are taken: the longest first, equal ones as they come."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import device_checks

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def checks(tmp_path_factory):
    return device_checks.load(tmp_path_factory.mktemp("device_checks"))


@pytest.mark.parametrize("n", [1, 2, 33, 128])
@pytest.mark.parametrize("window,sinks", [(50, 4), (1, 0), (1 << 30, 0), (1 << 30, 4), (1, 1 << 30), (1 << 30, 1 << 30), (1 << 29, 1 << 29), ((1 << 30) - 1, 1 << 30)])
def test_the_longest_first(checks, n, window, sinks):
    rng = np.random.default_rng(n)
    lens = rng.integers(-3, 900, n)
    lens[rng.random(n) < 0.2] = 5000                     # beyond the table: as long as that
    lens[rng.random(n) < 0.2] = 300
    most = np.minimum(np.clip(lens, 0, 60 * 16), window + sinks)
    got = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    own = torch.from_numpy(lens.astype(np.int32)).cuda()
    assert checks.check_order(own.data_ptr(), n, 60, 16, window, sinks, got.data_ptr()) == 0
    assert got.tolist() == np.argsort(-most, kind="stable").tolist()
