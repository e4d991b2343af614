"""Positions that are not [axes, count*m] would be read as if they were: Context.rotate_axes refuses them, without a GPU."""
import numpy as np
import pytest
import torch

from tests.test_attend_call import calls, context  # noqa: F401  (a fixture)


@pytest.mark.parametrize("shape", [(3,), (3, 2), (6, 3), (3, 7), (3, 5), (1, 5), (0, 6), ()])
def test_shapes(calls, shape):  # noqa: F811
    t = torch.zeros(8)
    with pytest.raises(AssertionError, match="positions"):
        context().rotate_axes(t, 3, 2, torch.zeros((5, 2, 64)), torch.zeros(shape, dtype=torch.int32), np.zeros(64, dtype=np.uint8), t, t, t, 64)
    assert not calls


@pytest.mark.parametrize("shape", [(1, 6), (2, 6), (4, 6), (4, 3, 2), (1, 9)])
def test_axes_by_tokens(calls, shape):  # noqa: F811
    t = torch.zeros(8)
    context().rotate_axes(t, 3, 2, torch.zeros((5, 2, 64)), torch.zeros(shape, dtype=torch.int32), np.zeros(64, dtype=np.uint8), t, t, t, 64)
    assert len(calls) == 1 and calls[0][1][7] == shape[0]
