"""Bounded waits of the tensor core kernels, by themselves: when they run out, and when another role gives up."""
from __future__ import annotations

import pytest
import torch

import device_checks

pytestmark = pytest.mark.gpu

SLACK_US = 100   # two tries of about 4 us, the timer, a thread that sleeps; far below the 256 us of 64 tries


@pytest.fixture(scope="module")
def checks(tmp_path_factory):
    return device_checks.load(tmp_path_factory.mktemp("device_checks"))


def took(checks, patient, limit_us, give_up_us=0):
    us, result = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    assert checks.check_wait(patient, limit_us * 1000, give_up_us * 1000, us.data_ptr(), result.data_ptr()) == 0
    assert result.item() == 2        # not over, and the others are told
    return us.item() / 1000


@pytest.mark.parametrize("patient", [0, 1])
@pytest.mark.parametrize("limit", [0, 1, 20, 300, 2000, 50000])
def test_a_wait_ends_at_its_limit(checks, patient, limit):
    took(checks, patient, 1)
    assert limit <= took(checks, patient, limit) + 0.1 and took(checks, patient, limit) <= limit + SLACK_US


@pytest.mark.parametrize("patient", [0, 1])
def test_a_wait_ends_when_another_role_gives_up(checks, patient):
    took(checks, patient, 1)
    for after in (10, 60, 500):
        assert after - 0.1 <= took(checks, patient, 3000000, after) <= after + SLACK_US
