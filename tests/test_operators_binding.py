"""Refusals of the operators' binding that need no device."""
import os

import numpy as np
import pytest
import torch


@pytest.fixture(scope="module")
def ops():
    from paper_1903_12287_amd import operators, pbg
    if not os.path.exists(pbg.LIB_PATH):
        pytest.skip("library not built")
    return operators


@pytest.mark.parametrize("offsets", [None, [0, 1, 3], np.array([0, 1, 3])])
def test_offsets_that_are_no_tensor(ops, offsets):
    z, labels, f = torch.zeros(3, 4), torch.zeros(3, dtype=torch.int32), torch.zeros(2)
    with pytest.raises(TypeError, match="offsets must be a torch.Tensor"):
        ops.pbg_preference_loss(None, z, labels, offsets, None, 0.1, 0.0, None, f, None, torch.zeros(3, 2))
    with pytest.raises(TypeError, match="offsets must be a torch.Tensor"):
        ops.pbg_preference_loss_backward(None, z, labels, offsets, torch.zeros(3, 2), f, z)
