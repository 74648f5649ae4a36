"""The check of weights refuses what it must (on the host)."""
import math

import pytest
import torch

import cache_weights_check as check

TABLE = torch.tensor([[1]], dtype=torch.int32)
SUMS = {(0, 0): (torch.full((20,), 0.5, dtype=torch.float64), None, torch.full((20,), 1e-6, dtype=torch.float64))}


def weights(at=None, value=0.0):
    w = torch.full((2, 1, 32), 0.5)
    if at is not None:
        w[1, 0, at] = value
    return w


def test_right_weights_pass():
    used = check.weights(weights(25, math.nan), SUMS, None, TABLE, [0, 20], [20])  # (behind the last key)
    assert int(used.sum()) == 20 and bool(used[1, 0, :20].all())


@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf, 0.5001, 0.0])
@pytest.mark.parametrize("at", [0, 7, 19])
def test_one_wrong_weight_fails(at, value):
    with pytest.raises(AssertionError, match=f"first at {at}"):
        check.weights(weights(at, value), SUMS, None, TABLE, [0, 20], [20])


def test_all_nan_fails():
    with pytest.raises(AssertionError):
        check.weights(weights() * math.nan, SUMS, None, TABLE, [0, 20], [20])
