"""CPU tests of the comparison that the sequence layers' GPU tests are run with a second time."""
import numpy as np
import pytest
import torch

from tests import sequence_strict


def test_results_within_the_tolerance_pass():
    ref = np.array([1.0, -2.0, 0.0, np.inf, np.nan])
    sequence_strict.close(torch.tensor([1.0, -2.0 - 2.0 ** -23, 0.0, -np.inf, np.nan]), ref, np.ones(5), "f32", 2.0 ** -22, "")


@pytest.mark.parametrize("wrong", [float("nan"), float("inf"), -float("inf"), 1.001])
@pytest.mark.parametrize("at", [0, 2])
def test_values_that_are_wrong_or_none_do_not_pass(wrong, at):
    got, ref = np.array([1.0, -2.0, 1.0]), np.array([1.0, -2.0, 1.0])
    got[at] = wrong
    with pytest.raises(AssertionError):
        sequence_strict.close(torch.tensor(got), ref, np.ones(3), "f32", 2.0 ** -22, "")


def test_finite_values_do_not_stand_for_infinities():
    for ref in (np.inf, np.nan):
        with pytest.raises(AssertionError):
            sequence_strict.close(torch.tensor([1.0]), np.array([ref]), np.ones(1), "f32", 1.0, "")


def test_kinds():
    assert sequence_strict.kind(np.array([0.0, -3.0, np.inf, -np.inf, np.nan])).tolist() == [0, 0, 1, -1, 2]
