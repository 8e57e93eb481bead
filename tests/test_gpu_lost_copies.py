"""Failure detection in the operators that do not wait for the GPU: with a limit of one look, a wait for a copy gives up
while the copy is on its way.  Nothing faults or hangs: the blocks wait for their copies before they end, results that were
not reached are NaN, and none is wrong."""
import pytest
import torch

from paper_2609_27209_gb300 import erc

from ._gpu import dev

pytestmark = pytest.mark.gpu
TRIES = 3


@pytest.fixture(autouse=True)
def default_limits_after():
    yield
    erc.erc_set_wait_limit(0)


# a block a row, a cluster a row, rows joined by a second kernel, blocks that take several rows
@pytest.mark.parametrize("rows,n,k", [(700, 9001, 0), (700, 9001, 5), (40, 60001, 0), (40, 60001, 20), (1, 1400003, 0),
                                      (2, 1400003, 32), (10001, 5001, 3), (3000, 60001, 4)])
@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
def test_rows_whose_copy_was_not_waited_for_are_nan(rows, n, k, kind):
    g = torch.Generator(device=dev()).manual_seed(n + k)
    x = torch.randn(rows, n, generator=g, device=dev()).to(kind)
    ids = torch.randint(-1, n, (rows,), generator=g, device=dev(), dtype=torch.int32)
    want = [v for v in erc.erc_score_rows(x, ids, k=k) if v is not None]
    missing = [torch.full_like(v, -1 if v.dtype == torch.int32 else float("nan")) for v in want]
    erc.erc_set_wait_limit(1)
    lost = 0
    for _ in range(TRIES):
        got = [v for v in erc.erc_score_rows(x, ids, k=k) if v is not None]
        gone = torch.isnan(got[1])  # the entropy
        lost += int(gone.sum())
        for v, right, none in zip(got, want, missing):
            expected = torch.where(gone.view(-1, *[1] * (v.dim() - 1)), none, right)
            assert torch.equal(v, expected) if v.dtype == torch.int32 else torch.equal(v.nan_to_num(7e7), expected.nan_to_num(7e7))
    assert lost > 0
    erc.erc_set_wait_limit(0)
    again = [v for v in erc.erc_score_rows(x, ids, k=k) if v is not None]
    assert all(torch.equal(a, b) for a, b in zip(again, want))
