"""loss() and head_loss() record no autograd graph and say so: the warnings come before anything that needs a device."""
import warnings

import pytest
import torch

from paper_2502_05202_b200 import tli


def bare():
    v = tli.Verifier.__new__(tli.Verifier)
    v._index, v.device, v.ctx = 0, torch.device("cuda", 0), 0
    return v


@pytest.mark.parametrize("call", [lambda v, x: v.loss(x, torch.zeros(2, dtype=torch.int32)), lambda v, x: v.head_loss(x, torch.zeros(3, 8), torch.zeros(2, dtype=torch.int32)),
                                  lambda v, x: v.head_loss(torch.zeros(2, 8), x, torch.zeros(2, dtype=torch.int32))])
def test_inputs_that_wait_for_a_gradient(call):
    v = bare()
    with pytest.warns(UserWarning, match="no autograd graph"), pytest.raises(ValueError):      # (CPU tensors are refused afterwards)
        call(v, torch.zeros(2, 8, requires_grad=True))
    with warnings.catch_warnings(), torch.no_grad():
        warnings.simplefilter("error")
        with pytest.raises(ValueError):
            call(v, torch.zeros(2, 8, requires_grad=True))
