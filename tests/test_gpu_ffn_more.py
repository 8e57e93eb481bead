"""The gated feed-forward block at the ends of its ranges: an expert with as many rows as there can be, weights' gradients
over many rows, a handful of rows."""
import numpy as np
import pytest
import torch

from oracle import expert_oracle as X
from paper_2609_27209_gb300 import erc

from ._gpu import dev
from .test_gpu_ffn import TYPES, U, check, f64, inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def give_memory_back():
    yield
    torch.cuda.empty_cache()


def test_an_expert_with_as_many_rows_as_there_can_be():
    slots = 2**31 - 1  # x, y and the hidden rows: 34 GB each
    if torch.cuda.mem_get_info()[0] < 120 << 30:
        pytest.skip("needs 120 GB")
    g = torch.Generator().manual_seed(1)
    w_in = (torch.randn(2, 16, 8, generator=g) / 2).bfloat16().to(dev())
    w_out = (torch.randn(2, 8, 8, generator=g) / 2).bfloat16().to(dev())
    x = torch.zeros(slots, 8, dtype=torch.bfloat16, device=dev())
    at = torch.tensor([0, 300, slots - 3], device=dev())
    places = [0, 2**30, 2**31 - 2**23, slots - 403]  # the last: 400 rows and the 3 behind the experts
    for p in places:
        x[p : p + 400] = torch.randn(400, 8, generator=g).bfloat16().to(dev())
    y, _ = erc.erc_expert_ffn(x, at, w_in, w_out)
    assert not y[-3:].any()
    for p in places:
        own = np.array([0, 300 if p == 0 else 0, 400])
        want, _ = X.ffn(f64(x[p : p + 400]), own, f64(w_in), f64(w_out), 0)
        # roundings of bfloat16: of h (2^-8 of it) and of the result; sums of 8 terms, at most 8 times a result's size
        assert np.abs(f64(y[p : p + 400]) - want).max() <= 8 * 2.0**-8 * np.abs(want).max()
    assert not y[1000:10000].any()


@pytest.mark.parametrize("slots,width,inner", [(20000, 64, 64), (100000, 2048, 2048), (1500000, 96, 128)])
def test_long_float32_sums_over_slots_keep_their_last_bits(slots, width, inner):
    """dw_out sums act(a) b dy over the slots, act(a) b rounded as torch rounds it.  Sums of 256 terms of mixed signs, then of
    n / 256 such sums, then of up to 64 parts: as in the other long sums, squared errors of U^2 / 6 for each term summed."""
    g = torch.Generator(device=dev()).manual_seed(slots)
    mk = lambda *s: torch.randn(*s, generator=g, device=dev())  # noqa: E731
    x, dy, pre = torch.zeros(slots, width, device=dev()), mk(slots, width), mk(slots, 2 * inner)
    w_in, w_out = torch.zeros(1, 2 * inner, width, device=dev()), torch.zeros(1, width, inner, device=dev())
    at = torch.tensor([0, slots], device=dev())
    _, _, got = erc.erc_expert_ffn_backward(dy, x, pre, at, w_in, w_out, act=erc.ERC_ACT_RELU, dxs=False)
    h = pre[:, :inner].clamp(min=0) * pre[:, inner:]
    want = dy.double().T @ h.double()
    error = (got[0].double() - want).norm().item() / want.norm().item()
    assert error <= U * np.sqrt((256 + slots / 256 + 64) / 6), error / U


FEW = {"two": [2], "three": [3], "five": [5], "seven": [7], "eight": [8], "two-each": [1, 3], "none-first": [0, 8, 0],
       "of-three": [4, 2, 5], "past-eight": [9, 1, 2], "of-eight": [1, 0, 6, 2, 8, 3, 7, 5], "all-to-one": [0, 0, 0, 32, 0, 0, 0, 0]}


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("width,inner", [(8, 16), (72, 40), (520, 264)])
@pytest.mark.parametrize("counts", FEW)
def test_a_handful_of_slots(kind, width, inner, counts):
    """Single tokens: every number of rows that a warp takes at once, more than it takes, several experts, rows behind."""
    behind = 1 if sum(FEW[counts]) < 8 else 0
    check(*inputs(width + len(counts), FEW[counts], behind, width, inner, kind), act=(width + len(counts)) % 3)


def test_a_handful_of_slots_repeats_and_replays():
    offsets, x, dy, w_in, w_out = inputs(3, [2, 0, 5, 3], 1, 256, 512, "bf16")
    at = torch.from_numpy(offsets).to(dev())
    first = erc.erc_expert_ffn(x, at, w_in, w_out, keep=True)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = erc.erc_expert_ffn(x, at, w_in, w_out, keep=True)
    graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(first, held))
    at.copy_(torch.tensor([0, 0, 9, 9, 11]))  # more rows of one expert, none behind
    x.copy_(torch.randn(11, 256, generator=torch.Generator().manual_seed(8)))
    graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(held, erc.erc_expert_ffn(x, at, w_in, w_out, keep=True)))
