"""Arrays of more than 2^31 (or 2^32) elements: offsets are 64 bits wide in every operator of training and answering."""
import numpy as np
import pytest
import torch

from oracle import expert_oracle as X
from paper_2609_27209_gb300 import erc

from ._gpu import dev

pytestmark = pytest.mark.gpu

U = 2.0**-24


@pytest.fixture(autouse=True)
def give_memory_back():
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("rows,n,k", [(60001, 40000, 0), (60001, 40000, 3), (9000001, 257, 2)])
def test_scores_past_32_bits(rows, n, k):
    x = torch.zeros(rows, n, dtype=torch.bfloat16, device=dev())
    few = torch.randn(5, n, generator=torch.Generator().manual_seed(n)).to(torch.bfloat16)
    x[-5:] = few.to(dev())
    ids = torch.full((rows,), n - 1, dtype=torch.int32, device=dev())
    logp, entropy, norm, top, _ = erc.erc_score_rows(x, ids, k=k)
    grad = erc.erc_score_rows_backward(x, ids, norm, torch.ones(rows, device=dev()))
    for i in range(5):
        want = X.score_row(few[i].double().numpy(), n - 1, 1.0, k)
        assert abs(logp[rows - 5 + i].item() - want[0]) <= 700 * U + 8 * U * abs(want[0])
        if k:
            assert top[rows - 5 + i].tolist() == want[3].tolist()
        back = X.score_row_backward(few[i].double().numpy(), n - 1, 1.0, 0.0)
        got = grad[rows - 5 + i].double().cpu().numpy()
        assert np.all(np.abs(got - back) <= (2.0**-8 + 800 * U) * np.abs(back))


def test_the_block_past_32_bits():
    slots, width, inner = 1_200_001, 64, 1024
    g = torch.Generator(device=dev()).manual_seed(2)
    mk = lambda *s, scale=1.0: (scale * torch.randn(*s, generator=g, device=dev())).bfloat16()  # noqa: E731
    x, dy = mk(slots, width), mk(slots, width)
    w_in, w_out = mk(2, 2 * inner, width, scale=0.125), mk(2, width, inner, scale=0.03125)
    at = torch.tensor([0, 700_000, slots - 3], device=dev())
    y, pre = erc.erc_expert_ffn(x, at, w_in, w_out, keep=True)
    dx, _, _ = erc.erc_expert_ffn_backward(dy, x, pre, at, w_in, w_out, dw=False)
    assert not y[-3:].any() and not pre[-3:].any() and not dx[-3:].any()
    s = slice(slots - 43, slots - 3)
    f = lambda t: t.double().cpu().numpy()  # noqa: E731
    own = np.array([0, 0, 40])
    want_y, want_pre = X.ffn(f(x[s]), own, f(w_in), f(w_out), 0)
    want_dx, _, _ = X.ffn_backward(f(dy[s]), f(x[s]), f(pre[s]), own, f(w_in), f(w_out), 0)
    # roundings of bfloat16 (2^-8 of a value at most, of h or the gradients of a and b, and of the result), the sums'
    # magnitudes: entries of order 1, 8 times a result's size at most
    for got, want in ((y[s], want_y), (pre[s], want_pre), (dx[s], want_dx)):
        assert np.abs(f(got) - want).max() <= 8 * 2.0**-8 * np.abs(want).max()


def test_dropout_past_32_bits():
    count = 2**32 + 1001
    x = torch.ones(count, dtype=torch.bfloat16, device=dev())
    r = torch.ones(count, dtype=torch.bfloat16, device=dev())
    out = erc.erc_dropout(x, 0.5, 17, residual=r)
    first = count - 1001 - 4096
    keep = torch.from_numpy(X.dropout_keep(1001 + 4096, 0.5, 17, first))
    assert torch.equal(out[first:].float().cpu(), torch.where(keep, 3.0, 1.0))
    del out
    odd = erc.erc_dropout(x[1:], 0.5, 17)  # not aligned: four entries a thread
    tail = torch.from_numpy(X.dropout_keep(1001 + 4096, 0.5, 17, first))[: count - 1 - first]
    assert torch.equal(odd[first:].float().cpu(), torch.where(tail, 2.0, 0.0))
