"""Verifier.embed() and torch's autograd, without a GPU."""
import warnings

import pytest
import torch

from paper_2502_05202_b200 import tli


def test_a_table_that_waits_for_a_gradient_is_not_passed_over_in_silence():
    v = tli.Verifier.__new__(tli.Verifier)                                    # without a context: the call itself is left out
    v.ctx, v._index, v.device, v.V_t, v.V_d, v._fn_embed, v._call = 0, -1, torch.device("cpu"), 5, 4, None, lambda fn, args: None
    ids, table = torch.zeros(3, dtype=torch.int32), torch.zeros(5, 8, requires_grad=True)
    with pytest.warns(UserWarning, match="embed_grad"):
        assert v.embed(ids, table)["rows"].shape == (3, 8)
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        v.embed(ids, table.detach())
        with torch.no_grad():
            v.embed(ids, table)
