"""Scores at the ends of their ranges."""
import math

import pytest
import torch

from paper_2609_27209_gb300 import erc

from ._gpu import dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("n", [40, 3001, 20001])
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan, 3e38])
def test_masked_entries_have_no_gradient_whatever_comes_from_above(kind, n, value):
    g = torch.Generator(device=dev()).manual_seed(n)
    x = torch.randn(6, n, generator=g, device=dev()).to(kind)
    masked = torch.rand(6, n, generator=g, device=dev()) < 0.3
    masked[:, 0], masked[:, 1] = False, True
    x[masked] = -math.inf
    x[2, masked[2]] = math.nan
    ids = torch.tensor([0, 1, -1, 0, 0, n], dtype=torch.int32, device=dev())
    _, entropy, norm, _, _ = erc.erc_score_rows(x, ids)
    one = torch.ones(6, device=dev())
    for dlogp, dentropy in ((value * one, one), (one, value * one), (value * one, value * one)):
        grad = erc.erc_score_rows_backward(x, ids, norm, dlogp, entropy, dentropy)
        assert not grad[masked].any()
    # and rows beside it are what they are alone
    dlogp = one.clone()
    dlogp[3] = value
    got, want = (erc.erc_score_rows_backward(x, ids, norm, d, entropy, one) for d in (dlogp, one))
    others = [0, 1, 2, 4, 5]
    assert torch.equal(got[others], want[others])
