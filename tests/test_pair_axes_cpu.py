"""The axis of each pair of columns, as callers hold it: the description that the
library reads is the same for bytes and for any sequence of integers, whatever
their width in memory (no GPU)."""
import array

import numpy as np
import pytest
import torch

import paper_2608_18656_amd as fa

AXES = [0, 1, 2, 1, 0, 2, 2, 1]


def described(pair_axes):
    freq, pos = torch.ones(len(AXES)), torch.zeros((3, 2, 5), dtype=torch.int32)
    r = fa._rotary(fa._runtime(), freq, pos, pair_axes, False, 2, 5, freq.get_device())
    return list(r.pair_axis)[:len(AXES)]


@pytest.mark.parametrize("pair_axes", [
    AXES, tuple(AXES), bytes(AXES), bytearray(AXES), memoryview(bytes(AXES)), range(0), np.array(AXES), np.array(AXES, np.int32),
    np.array(AXES, np.uint8), array.array("i", AXES), array.array("q", AXES), torch.tensor(AXES),
    np.repeat(np.array(AXES), 2)[::2]], ids=lambda a: type(a).__name__ + str(getattr(a, "dtype", "")))
def test_any_sequence_of_integers(pair_axes):
    if len(pair_axes) == 0:
        with pytest.raises(ValueError):
            described(pair_axes)
    else:
        assert described(pair_axes) == AXES


@pytest.mark.parametrize("pair_axes,error", [([0.0] * 8, TypeError), (np.array(AXES, np.float32), TypeError), ([300] * 8, ValueError),
                                             ([-1] * 8, ValueError), (np.array([256] * 8), ValueError), (AXES[:7], ValueError),
                                             (AXES + [0], ValueError)])
def test_refusals(pair_axes, error):
    with pytest.raises(error):
        described(pair_axes)
