"""GPU parity of erc_dropout: every step is one rounded float32 operation, so results are bit-exact."""
import numpy as np
import pytest
import torch

from oracle import expert_oracle as X
from paper_2609_27209_gb300 import erc

from ._gpu import dev

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def want(x, p, key, residual=None, first=0):
    r = None if residual is None else residual.float().cpu().numpy()
    return torch.from_numpy(X.dropout(x.float().cpu().numpy(), p, key, r, first)).to(x.dtype)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("count", [1, 3, 4, 7, 8, 9, 1000, 4099, 300007])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 1.0])
def test_against_the_oracle(kind, count, p):
    x = torch.randn(count, device=dev()).to(TYPES[kind])
    r = torch.randn(count, device=dev()).to(TYPES[kind])
    key = 0x9E3779B97F4A7C15 + count
    assert torch.equal(erc.erc_dropout(x, p, key).cpu(), want(x, p, key))
    assert torch.equal(erc.erc_dropout(x, p, key, residual=r).cpu(), want(x, p, key, r))


@pytest.mark.parametrize("kind", TYPES)
def test_misaligned_views_continue_one_stream(kind):
    base = torch.randn(5001, device=dev()).to(TYPES[kind])
    whole = erc.erc_dropout(base, 0.3, 77)
    part = base[1204:4801]  # a view that is not 16-byte aligned for every type
    assert torch.equal(erc.erc_dropout(part, 0.3, 77, first=1204), whole[1204:4801])
    odd = base[3:]
    assert torch.equal(erc.erc_dropout(odd, 0.3, 77).cpu(), want(odd, 0.3, 77))


def test_numbers_beyond_32_bits():
    x = torch.ones(64, device=dev())
    for first in (2**34 - 32, 2**40, 2**61):
        assert torch.equal(erc.erc_dropout(x, 0.5, 3, first=first).cpu(), want(x, 0.5, 3, first=first))


def test_more_than_a_machine_of_entries():
    x = torch.ones(40_000_003, dtype=torch.bfloat16, device=dev())
    out = erc.erc_dropout(x, 0.25, 11)
    tail = want(torch.ones(3 + 4096), 0.25, 11, first=40_000_000 - 4096).to(torch.bfloat16)
    assert torch.equal(out[-4099:].cpu(), tail)
    assert abs(float((out != 0).float().mean()) - 0.75) < 5 * (0.1875 / 4e7) ** 0.5


def test_dropped_entries_are_zero_whatever_they_hold():
    x = torch.full((4096,), float("nan"), device=dev())
    out = erc.erc_dropout(x, 0.5, 9)
    keep = torch.from_numpy(X.dropout_keep(4096, 0.5, 9)).to(dev())
    assert torch.isnan(out[keep]).all() and (out[~keep] == 0).all()


def test_gradient_is_the_same_call():
    x = torch.randn(1000, dtype=torch.float64, requires_grad=True)
    g = torch.randn(1000)
    keep = torch.from_numpy(X.dropout_keep(1000, 0.2, 21))
    torch.where(keep, x * float(np.float32(1 / 0.8)), 0.0).backward(g.double())
    got = erc.erc_dropout(g.to(dev()), 0.2, 21).cpu()
    assert torch.equal(got, x.grad.float())  # one product, rounded once


def test_a_key_on_the_device_is_read_when_a_graph_replays():
    x = torch.randn(10, 333, device=dev())
    key = torch.tensor([5], device=dev())
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        erc.erc_dropout(x, 0.3, key)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = erc.erc_dropout(x, 0.3, key, residual=x)
    for k in (5, -1, 2**62):
        key.fill_(k)
        graph.replay()
        assert torch.equal(out, erc.erc_dropout(x, 0.3, k, residual=x))
        assert torch.equal(out.cpu(), want(x, 0.3, k % 2**64, x))


def test_in_place_through_the_c_entry():
    x, r = torch.randn(2, 999, device=dev())
    for target in (x.clone(), r.clone()):
        a, b = (target, r) if torch.equal(target, x) else (x, target)
        erc.lib().erc_dropout(999, a.data_ptr(), 0, b.data_ptr(), 0.4, 8, None, 0, target.data_ptr(), None)
        torch.cuda.synchronize()
        assert torch.equal(target, erc.erc_dropout(x, 0.4, 8, residual=r))


def test_refusals_and_empty():
    x = torch.randn(8, 8, device=dev())
    assert erc.erc_dropout(x[:0], 0.5, 1).shape == (0, 8)
    for call in (lambda: erc.erc_dropout(x.t(), 0.5, 1), lambda: erc.erc_dropout(x.double(), 0.5, 1), lambda: erc.erc_dropout(x, 2.0, 1),
                 lambda: erc.erc_dropout(x, 0.5, 1, residual=x[:4]), lambda: erc.erc_dropout(x, 0.5, 1, residual=x.half()),
                 lambda: erc.erc_dropout(x, 0.5, torch.tensor([1])), lambda: erc.erc_dropout(x, 0.5, 1, first=2),
                 lambda: erc.erc_dropout(x, 0.5, 1, first=-4), lambda: erc.erc_dropout(x, 0.5, 1.5)):
        with pytest.raises(erc.ErcError) as e:
            call()
        assert e.value.status == erc.ERC_ERR_INVALID_ARG
