"""The axis of every pair, as msa_norm_rotate_axes takes it in Python: what is refused does not depend on what was asked for before."""
import numpy as np
import pytest
import torch

import paper_2603_23516_amd as msa


@pytest.fixture
def asked_for():
    """[0] * 32 and its like are known already."""
    msa._axes_arrays.clear()
    for axes in ([0] * 32, [1] * 32, [u % 3 for u in range(32)]):
        assert list(msa._axes_array(axes, 32)) == axes


@pytest.mark.parametrize("bad", [[0.0] * 32, [1.0] * 32, [0] * 31 + [0.0], [0] * 31 + [0.5], [0] * 31 + [4], [0] * 31 + [-1], [0] * 31 + [300],
                                 [0] * 31, [0] * 33, [], ["0"] * 32, [None] * 32, [np.float32(1)] * 32, [0j] * 32])
def test_refused_before_and_after(asked_for, bad):
    for _ in range(2):
        with pytest.raises(ValueError):
            msa._axes_array(bad, 32)
    msa._axes_arrays.clear()
    with pytest.raises(ValueError):
        msa._axes_array(bad, 32)


@pytest.mark.parametrize("good", [[2] * 32, tuple([2] * 32), np.full(32, 2, np.int64), np.full(32, 2, np.uint8), torch.full((32,), 2),
                                  range(2, 3), (2 for _ in range(32)), [np.int32(2)] * 32])
def test_taken_before_and_after(good):
    """Integers of any kind, in any order of calls."""
    n = 1 if isinstance(good, range) else 32
    again = good if not hasattr(good, "__next__") else [2] * 32
    msa._axes_arrays.clear()
    assert list(msa._axes_array(good, n)) == [2] * n
    assert list(msa._axes_array(again, n)) == [2] * n
    msa._axes_arrays.clear()
    assert list(msa._axes_array([2] * n, n)) == [2] * n
    assert list(msa._axes_array(again, n)) == [2] * n


def test_an_array_changed_in_place_is_read_again():
    for axes in (np.zeros(32, np.int64), torch.zeros(32, dtype=torch.int64)):
        assert list(msa._axes_array(axes, 32)) == [0] * 32
        axes[5] = 3
        assert list(msa._axes_array(axes, 32)) == [0] * 5 + [3] + [0] * 26


def test_few_are_kept():
    for i in range(200):
        axes = [int(c) for c in f"{i:032b}"]
        assert list(msa._axes_array(axes, 32)) == axes
    assert len(msa._axes_arrays) <= 64
