"""Failure detection in the operators that do not wait for the GPU: with a limit of one look, a wait for a copy gives up
while the copy is on its way.  Nothing faults or hangs: the blocks wait for their copies before they end, results that were
not reached are NaN, and none is wrong."""
import numpy as np
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


def block_inputs(seed, counts, width, inner, kind):
    g = torch.Generator(device=dev()).manual_seed(seed)
    mk = lambda *s, scale=1.0: (scale * torch.randn(*s, generator=g, device=dev())).to(kind)  # noqa: E731
    slots, E = sum(counts) + 3, len(counts)
    at = torch.tensor([0, *np.cumsum(counts)], device=dev())
    return at, mk(slots, width), mk(slots, width), mk(E, 2 * inner, width, scale=width**-0.5), mk(E, width, inner, scale=inner**-0.5)


def block_steps(at, x, dy, w_in, w_out, pre, act=0):
    """Forward and gradient, each with its results and the status that it leaves in its workspace."""
    shape = erc._ffn_shape(x, "x", at, w_in, w_out, act)
    out = []
    for size, call in (("erc_expert_ffn_workspace_size", lambda ws: erc.erc_expert_ffn(x, at, w_in, w_out, act, keep=True, ws=ws)),
                       ("erc_expert_ffn_backward_workspace_size",
                        lambda ws: erc.erc_expert_ffn_backward(dy, x, pre, at, w_in, w_out, act, ws=ws))):
        ws = torch.empty(getattr(erc.lib(), size)(shape), dtype=torch.uint8, device=dev())
        results = call(ws)
        start = -ws.data_ptr() % 256
        out.append((results, int(ws[start : start + 4].view(torch.int32))))
    return out


BLOCKS = {"one": ([5000], 512, 256), "ragged": ([300, 0, 1000, 77], 256, 320), "many": ([64] * 70, 128, 64),
          "odd": ([2900], 201, 203), "deep": ([40000], 32, 64)}


@pytest.mark.parametrize("counts,width,inner", BLOCKS.values(), ids=BLOCKS)
@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("polls", [1, 20, 200, 2000])
def test_a_wait_of_the_block_that_gave_up_is_in_its_status(counts, width, inner, kind, polls):
    at, x, dy, w_in, w_out = block_inputs(width + polls, counts, width, inner, kind)
    pre = erc.erc_expert_ffn(x, at, w_in, w_out, keep=True)[1]
    want = block_steps(at, x, dy, w_in, w_out, pre)
    assert [status for _, status in want] == [erc.ERC_OK] * 2
    erc.erc_set_wait_limit(polls)
    for _ in range(TRIES):
        for (got, status), (right, _) in zip(block_steps(at, x, dy, w_in, w_out, pre), want):
            assert status in (erc.ERC_OK, erc.ERC_ERR_TIMEOUT)
            assert polls > 1 or status == erc.ERC_ERR_TIMEOUT
            if status == erc.ERC_OK:
                assert all(torch.equal(a, b) for a, b in zip(got, right))
    erc.erc_set_wait_limit(0)
    for (got, status), (right, _) in zip(block_steps(at, x, dy, w_in, w_out, pre), want):
        assert status == erc.ERC_OK and all(torch.equal(a, b) for a, b in zip(got, right))


@pytest.mark.parametrize("counts,width,inner", BLOCKS.values(), ids=BLOCKS)
@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("act", [0, 1, 2])
@pytest.mark.parametrize("polls", [1, 30, 300])
def test_results_that_a_block_did_not_reach_are_nan(counts, width, inner, kind, act, polls):
    at, x, dy, w_in, w_out = block_inputs(width + polls + act, counts, width, inner, kind)
    pre = erc.erc_expert_ffn(x, at, w_in, w_out, act, keep=True)[1]
    want = block_steps(at, x, dy, w_in, w_out, pre, act)
    erc.erc_set_wait_limit(polls)
    for _ in range(TRIES):
        for (got, status), (right, _) in zip(block_steps(at, x, dy, w_in, w_out, pre, act), want):
            missing = [torch.isnan(a) for a in got]
            for a, b, none in zip(got, right, missing):
                assert torch.equal(torch.where(none, b, a), b)
            # a block that gave up may have had no rows of its own (those from `inner` on), so only one way
            some = any(bool(none.any()) for none in missing)
            assert status == erc.ERC_ERR_TIMEOUT or (status == erc.ERC_OK and not some)
            assert polls > 1 or some
