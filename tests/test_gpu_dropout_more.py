"""Dropout's refusals of what is no number."""
import math

import pytest
import torch

from paper_2609_27209_gb300 import erc

from ._gpu import dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("value", [None, math.nan, math.inf, "7", [1], 1.5, 1j])
def test_keys_and_firsts_that_are_no_whole_numbers(value):
    x = torch.randn(8, 8, device=dev())
    for call in (lambda: erc.erc_dropout(x, 0.5, value), lambda: erc.erc_dropout(x, 0.5, 1, first=value)):
        with pytest.raises(erc.ErcError) as e:
            call()
        assert e.value.status == erc.ERC_ERR_INVALID_ARG


def test_whole_numbers_of_any_type():
    x = torch.randn(8, 8, device=dev())
    want = erc.erc_dropout(x, 0.5, 2**63, first=8)
    assert torch.equal(erc.erc_dropout(x, 0.5, 2.0**63, first=8.0), want)
    assert torch.equal(erc.erc_dropout(x, 0.5, 2**63 + 2**64, first=8), want)
    assert torch.equal(erc.erc_dropout(x, 0.5, -(2**63), first=8), want)
