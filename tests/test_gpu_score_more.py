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


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows", [1, 3])
def test_many_equal_entries_of_rows_that_a_second_kernel_joins(rows, kind):
    """More than 256 candidates among the parts' best: the exact search by key and index."""
    n, k = 1400003, 32
    equal = torch.full((rows, n), 2.5, device=dev()).to(kind)
    ids = erc.erc_score_rows(equal, k=k)[3]
    assert (ids == torch.arange(k, device=dev(), dtype=torch.int32)).all()
    few = equal.clone()
    few[:, : n // 2] = 1.0  # the best are the later half
    best = [n - 1, n // 2 + 70000, n // 2 + 70001]
    few[:, best] = 3.0
    _, _, _, ids, logp = erc.erc_score_rows(few, k=k)
    want = torch.cat([torch.tensor(sorted(best)), torch.arange(n // 2, n // 2 + k - 3)]).to(dev()).int()
    assert torch.equal(ids, want.expand(rows, k))
    assert (logp[:, :3] == logp[:, :1]).all() and (logp[:, 3:] == logp[:, 3:4]).all() and (logp[:, 0] > logp[:, 3]).all()
    zeros = torch.zeros(rows, n, device=dev()).to(kind)
    zeros[:, ::3] = -0.0  # equal to +0
    zeros[:, 5] = -math.inf
    want = [i for i in range(k + 1) if i != 5]
    assert erc.erc_score_rows(zeros, k=k)[3].tolist() == [want] * rows


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,n", [(5, 40), (3000, 40), (5, 9001), (3000, 2500), (2, 60001), (1, 1400003)])
def test_a_types_lowest_value_is_a_score_and_a_mask_beside_others(rows, n, kind):
    low = torch.finfo(kind).min
    x = torch.full((rows, n), low, dtype=kind, device=dev())
    ids = torch.full((rows,), n - 1, dtype=torch.int32, device=dev())
    logp, entropy, norm, _, _ = erc.erc_score_rows(x, ids)
    # equal entries are counted, not summed: log n within its rounding and that of the logarithm
    for v, want in ((logp, -math.log(n)), (entropy, math.log(n)), (norm[:, 1], math.log(n))):
        assert (v - want).abs().max().item() <= 4 * 2.0**-24 * math.log(n)
    assert (norm[:, 0] == low).all()
    x[:, 3] = 0.0
    logp, entropy, norm, _, _ = erc.erc_score_rows(x, ids)
    assert (norm == 0).all() and (entropy == 0).all() and (logp == low).all()
    grad = erc.erc_score_rows_backward(x, ids, norm, torch.ones(rows, device=dev()), entropy, torch.ones(rows, device=dev()))
    want = torch.zeros_like(x)
    want[:, 3], want[:, -1] = -1.0, 1.0
    assert torch.equal(grad, want)
