"""Argument checks of the token-block operators' binding that need no GPU."""
import pytest
import torch

import paper_2105_09080_b200 as pkg
from paper_2105_09080_b200 import token_ops


def test_parameters_without_a_dimension_are_refused():
    """A single value is no vector of one column."""
    with pytest.raises(pkg.GpgaError) as err:
        token_ops._params(torch.ones(()), "weight", 1, 1, -1)
    assert err.value.status == pkg.GPGA_ERR_INVALID_ARG and "weight" in str(err.value)
    assert token_ops._params(torch.ones(1), "weight", 1, 1, -1) == 1
    assert token_ops._params(torch.ones((1, 1)), "weight", 1, 1, -1) == 1
